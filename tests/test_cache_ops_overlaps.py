"""Calls on the cache whose outputs would overlap are refused, as are counts
that 32 bits would wrap around and launches of 2^32 threads.  No GPU: validation fails
before any pointer is used."""
import ctypes
import itertools
import random

import pytest
import torch

from test_cache_ops_refusals import BIG, FAKE, H, INVALID, UNSUPPORTED, WORKSPACE, desc, meta, packed, prefill  # noqa: F401  (H: a fixture)


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
    assert lib.hill_evict(ctypes.byref(d), FAKE, 2, FAKE, None, None, ctypes.byref(p), None, 0, 0, FAKE, 0, None) == WORKSPACE


def layouts(seed):
    """Sizes and strides of rows of 128 elements, [B, heads, tokens], nested in any order, and with gaps too small or none."""
    rng = random.Random(seed)
    for _ in range(400):
        sizes = [rng.choice([1, 2, 3, 5]) for _ in range(3)]
        strides, extent = [0, 0, 0], 128
        for i in rng.sample(range(3), 3):
            strides[i] = max(0, extent + 8 * rng.choice([0, 0, 1, 3, 16, -1, -16]))
            extent = strides[i] * (sizes[i] - 1) + extent
        if rng.random() < 0.3:
            strides[rng.choice([0, 1])] = rng.choice([0, 8, 128, 136, 384])
        strides[2] = max(strides[2], 128)
        yield sizes, strides


def starts(sizes, strides):
    return sorted(sum(i * s for i, s in zip(at, strides)) for at in itertools.product(*map(range, sizes)))


def meet(a, b):
    """Whether a row that starts in a and one that starts in b have an element in common."""
    return any(abs(x - y) < 128 for x in a for y in b)


def test_rows_that_overlap_are_refused_and_no_others(H):
    lib, seen = H.load_library(), [0, 0]
    for (B, heads, n), (sb, sh, sn) in layouts(1):
        at = starts((B, heads, n), (sb, sh, sn))
        bad = any(y - x < 128 for x, y in zip(at, at[1:]))
        seen[bad] += 1
        d = desc(H, B=B, Hq=heads, Hkv=heads, n=n, sink=0, recent=0, k_stride_b=sb, k_stride_h=sh, k_stride_n=sn)
        evict = lambda k, v: lib.hill_evict(ctypes.byref(d), FAKE, 1, FAKE, k, v, None, None, 0, 0, FAKE, 0, None)
        assert evict(FAKE, FAKE + (1 << 30)) == (INVALID if bad else WORKSPACE), (B, heads, n, sb, sh, sn)
        d.k_stride_b, d.k_stride_h, d.k_stride_n, d.v_stride_b, d.v_stride_h, d.v_stride_n = desc(H, B=B, Hkv=heads, n=n).k_stride_b, n * 128, 128, sb, sh, sn
        assert evict(FAKE, FAKE + (1 << 30)) == (INVALID if bad else WORKSPACE), (B, heads, n, sb, sh, sn)
        if sb >= 0 and B == 1:     # [1, heads, tokens] of a prefill's output: without a workspace it needs none, or too little
            p = prefill(H, n_new=n, o_stride_b=sb, o_stride_h=max(sh, 128), o_stride_t=sn, q_stride_t=1024)
            at = starts((1, heads, n), (0, max(sh, 128), sn))
            if any(y - x < 128 for x, y in zip(at, at[1:])):
                assert lib.hill_window_prefill(ctypes.byref(d), ctypes.byref(p), FAKE, FAKE, FAKE, None, FAKE, None, 0, None) == INVALID
                assert b"rows of out overlap" in lib.hill_last_error()
    assert min(seen) > 50


def test_k_and_v_that_overlap_are_refused(H):
    lib, rng, seen = H.load_library(), random.Random(2), [0, 0]
    for (B, heads, n), (sb, sh, sn) in layouts(3):
        at = starts((B, heads, n), (sb, sh, sn))
        if any(y - x < 128 for x, y in zip(at, at[1:])):
            continue
        far = at[-1] // 8 + 16
        shift = 8 * rng.choice([rng.randint(-far, far), 16, -16, 15, sn // 8, far, -far, 1 - far])
        bad = meet([x + shift for x in at], at)
        seen[bad] += 1
        d = desc(H, B=B, Hq=heads, Hkv=heads, n=n, sink=0, recent=0, k_stride_b=sb, k_stride_h=sh, k_stride_n=sn,
                 v_stride_b=sb, v_stride_h=sh, v_stride_n=sn)
        k = FAKE + (1 << 24)
        evict = lib.hill_evict(ctypes.byref(d), FAKE, 1, FAKE, k, k + 2 * shift, None, None, 0, 0, FAKE, 0, None)
        assert evict == (INVALID if bad and shift else WORKSPACE), (B, heads, n, sb, sh, sn, shift)
        p = buffers(H)
        if bad:     # of the reader's outputs
            assert lib.hill_unpack_kv(ctypes.byref(d), ctypes.byref(p), 2, 2 + n, k, k + 2 * shift, None) == INVALID
            assert b"overlap" in lib.hill_last_error()
    assert min(seen) > 30


def test_outputs_with_overlapping_rows(H):
    """The plain ways to make them: an expanded tensor, one buffer for two outputs, a window that slides by less than a row."""
    lib, p = H.load_library(), buffers(H)
    back = lambda k=FAKE, v=FAKE + 4096, **st: lib.hill_unpack_kv(
        ctypes.byref(desc(H, n=8, **st)), ctypes.byref(p), 0, 8, k, v, None)
    for bad in (dict(v=FAKE), dict(v=FAKE + 256), dict(k_stride_b=0), dict(v_stride_b=0), dict(k_stride_h=0), dict(v_stride_h=64)):
        assert back(**bad) == INVALID, bad
        assert b"overlap" in lib.hill_last_error()
    d = desc(H)
    for bad in (dict(o_stride_t=128), dict(o_stride_h=128, o_stride_t=1016), dict(o_stride_b=128), dict(o_stride_h=16 * 128 - 8, o_stride_t=128)):
        q = prefill(H, **bad)
        assert lib.hill_window_prefill(ctypes.byref(d), ctypes.byref(q), FAKE, FAKE, FAKE, None, FAKE, FAKE, BIG, None) == INVALID
        assert b"rows of out overlap" in lib.hill_last_error(), bad


@pytest.fixture
def on_meta(H, monkeypatch):
    """A packed cache of 2 x 2 x 50 rows without memory; calls that pass the binding's checks end in an error of their own."""
    from paper_2602_18750_amd import cache as C
    monkeypatch.setattr(C, "_device_of", lambda *named: torch.device("meta"))
    monkeypatch.setattr(C, "_on", lambda *args: pytest.fail("accepted"))
    monkeypatch.setattr(C, "_ptr", lambda t: pytest.fail("accepted"))
    return H.new_packed_cache(2, 2, 50, "meta")


WRAP = 1 << 32


def test_counts_beyond_32_bits(H, on_meta):
    cache, k = on_meta, meta(2, 2, 5, 128)
    q, kv, s = meta(2, 8, 128), meta(2, 2, 50, 128), meta(2, 1, 52, dtype=torch.float32)
    for call in (lambda x: H.pack_kv(k, k, cache, at=x), lambda x: H.unpack_kv(cache, token_begin=x, token_end=x + 5),
                 lambda x: H.unpack_kv(cache, token_end=x + 5), lambda x: H.unpack_kv(cache, token_begin=x),
                 lambda x: H.hill_window_attn(q, kv, kv, window=4, n_tokens=x + 5),
                 lambda x: H.hill_window_prefill(q[:, :, None], kv, kv, window=4, n_tokens=x + 5),
                 lambda x: H.hill_packed_attn(q, cache, n_tokens=x + 5), lambda x: H.PackedAttnCall(q, cache, n_tokens=x + 5),
                 lambda x: H.hill_evict(s, x + 5, k=kv, v=kv), lambda x: H.hill_evict(s, 3, n_tokens=x + 5, k=kv, v=kv)):
        for x in (WRAP, -WRAP, 7 * WRAP):
            with pytest.raises(ValueError):
                call(x)


def test_ranges_of_the_writer_and_the_reader(H, on_meta):
    cache = on_meta
    rows = lambda n: meta(2, 2, n, 128)
    for n, at in ((5, -1), (5, 46), (51, 0), (0, 51), (0, -1)):
        with pytest.raises(ValueError):
            H.pack_kv(rows(n), rows(n), cache, at=at)
    for a, b in ((-1, 3), (4, 3), (0, 51), (51, 51), (50, 49)):
        with pytest.raises(ValueError):
            H.unpack_kv(cache, token_begin=a, token_end=b)


def test_no_rows_are_written_and_read(H, on_meta, monkeypatch):
    import contextlib
    from paper_2602_18750_amd import cache as C
    monkeypatch.setattr(C, "_on", lambda *args: contextlib.nullcontext())
    cache, none = on_meta, meta(2, 2, 0, 128)
    for at in (0, 17, 50):
        assert H.pack_kv(none, none, cache, at=at) is cache
        assert H.unpack_kv(cache, token_begin=at, token_end=at)[0].shape == (2, 2, 0, 128)
    assert H.pack_kv(none, none, cache, at=meta(2, dtype=torch.int32)) is cache


@pytest.mark.parametrize("B,heads", [(1 << 30, 4), (1 << 29, 8), (1 << 28, 16), ((1 << 31) - 1, 2), ((1 << 31) - 1, 256)])
def test_an_evictions_grid_in_64_bits(H, B, heads):
    """B * heads is a multiple of 2^32, or wraps to something small."""
    d = desc(H, B=B, Hq=heads, Hkv=heads, n=8, sink=0, recent=0, gran=1)
    ask = lambda: H.load_library().hill_evict(ctypes.byref(d), FAKE, 1, FAKE, None, None, None, None, 0, 0, FAKE,
                                                   (1 << 64) - 1, None)
    assert ask() == UNSUPPORTED
    assert b"workgroups" in H.load_library().hill_last_error()


def test_launches_hold_fewer_than_2_to_the_32_threads(H):
    """The last batch that fits passes on to the workspace's check (where it needs one), the next is refused."""
    lib, p = H.load_library(), packed(H, cap=8)
    small = dict(n=8, sink=0, recent=8)

    def evict(B, heads, keep, gran, n=8):
        d = desc(H, B=B, Hq=heads, Hkv=heads, n=n, sink=0, recent=0, gran=gran)
        return lib.hill_evict(ctypes.byref(d), FAKE, keep, FAKE, None, None, None, None, 0, 0, FAKE, 0, None)

    def score(B, heads):
        d = desc(H, B=B, Hq=heads, Hkv=heads, **small)
        return lib.hill_packed_attn(ctypes.byref(d), ctypes.byref(p), FAKE, None, None, 0, FAKE, FAKE, FAKE, 0, None)

    assert evict((1 << 20) - 1, 4, 8, 1) == WORKSPACE and evict(1 << 20, 4, 8, 1) == UNSUPPORTED      # the selection's
    assert evict(1 << 22, 1, 8, 0) == UNSUPPORTED
    assert evict(511, 1, 1 << 21, 0, n=1 << 21) == WORKSPACE                                          # the move's
    assert evict(512, 1, 1 << 21, 0, n=1 << 21) == UNSUPPORTED
    assert score((1 << 21) - 1, 8) == WORKSPACE and score(1 << 21, 8) == UNSUPPORTED
    d = desc(H, B=1 << 21, Hq=8, Hkv=8, **small)
    assert lib.hill_window_attn(ctypes.byref(d), FAKE, FAKE, FAKE, None, FAKE, FAKE, BIG, None) == UNSUPPORTED
    assert lib.hill_packed_attn(ctypes.byref(d), ctypes.byref(p), FAKE, None, None, 0, None, FAKE, FAKE, BIG, None) == UNSUPPORTED
    q = prefill(H, n_new=8, o_stride_b=8 * 8 * 128)
    assert lib.hill_window_prefill(ctypes.byref(d), ctypes.byref(q), FAKE, FAKE, FAKE, None, FAKE, FAKE, BIG, None) == UNSUPPORTED
