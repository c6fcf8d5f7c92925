"""Calls on the cache whose outputs would overlap are refused.  No GPU:
validation fails before any pointer is used."""
import ctypes

import pytest

from test_cache_ops_refusals import BIG, FAKE, H, INVALID, desc, packed  # noqa: F401  (H: a fixture)


def buffers(H, **at):
    """A packed cache of 2 x 2 x 10 rows: 2560 bytes of codes and 640 of parameters for K and for V, apart but for ``at``."""
    p = dict(k_codes=FAKE, k_params=FAKE + 4096, v_codes=FAKE + 8192, v_params=FAKE + 12288)
    p.update(at)
    return packed(H, cap=10, **p)


OVERLAPS = [
    dict(v_codes=FAKE, v_params=FAKE + 4096),                  # K and V in the same buffers
    dict(v_codes=FAKE), dict(v_params=FAKE + 4096),
    dict(v_codes=FAKE + 2544), dict(v_codes=FAKE - 2544),      # the last 16 bytes of one, the first of the other
    dict(k_params=FAKE + 2544), dict(k_params=FAKE - 624), dict(v_params=FAKE + 4096 + 624), dict(v_params=FAKE + 8192 + 16),
]


@pytest.mark.parametrize("at", OVERLAPS)
def test_written_caches_hold_k_and_v_apart(H, at):
    lib, p = H.load_library(), buffers(H, **at)
    d = desc(H, n=4, sink=0, recent=0)
    assert lib.hill_pack_kv(ctypes.byref(d), ctypes.byref(p), FAKE, FAKE, None, 0, None) == INVALID
    assert b"overlap" in lib.hill_last_error()
    assert lib.hill_evict(ctypes.byref(d), FAKE, 2, FAKE, None, None, ctypes.byref(p), None, 0, 0, FAKE, BIG, None) == INVALID
    assert b"overlap" in lib.hill_last_error()


@pytest.mark.parametrize("at", [dict(), dict(v_codes=FAKE + 2560, k_params=FAKE + 5120), dict(k_params=FAKE + 2560), dict(k_params=FAKE - 640)])
def test_buffers_that_only_touch_pass(H, at):
    """Seen by the next check's answer: rows outside the cache, an empty workspace."""
    lib, p = H.load_library(), buffers(H, **at)
    d = desc(H, n=4, sink=0, recent=0)
    assert lib.hill_pack_kv(ctypes.byref(d), ctypes.byref(p), FAKE, FAKE, None, 7, None) == INVALID
    assert b"not inside" in lib.hill_last_error()
    assert lib.hill_evict(ctypes.byref(d), FAKE, 2, FAKE, None, None, ctypes.byref(p), None, 0, 0, FAKE, 0, None) == 3
