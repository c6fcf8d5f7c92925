"""Argument errors of window attention, the 4-bit cache and eviction, at the C
ABI and in the Python binding.  No GPU: every call breaks one rule, and the
pointers are fake (never dereferenced, because validation fails first)."""
import ctypes
import os

import pytest
import torch

FAKE = 0x10000
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def H():
    import paper_2602_18750_amd as H
    if not os.path.exists(H.hill.LIB_PATH):
        from paper_2602_18750_amd import _build
        _build.build()
    H.load_library()
    return H


def desc(H, B=2, Hq=8, Hkv=2, n=1000, sink=4, recent=100, gran=0, **kw):
    d = H.HillDesc(ctypes.sizeof(H.HillDesc), B, Hq, Hkv, 128, n, 1, 0, gran, 0.0, Hq * 128, 128, Hkv * n * 128, n * 128, 128,
                   Hkv * n * 128, n * 128, 128, (n + 3) // 4 * 4 * (Hkv if gran else 1), (n + 3) // 4 * 4, sink, recent)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def packed(H, cap=1000, **kw):
    p = H.hill.PackedDesc(ctypes.sizeof(H.hill.PackedDesc), cap, FAKE, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def prefill(H, n_new=16, **kw):
    p = H.hill.PrefillDesc(ctypes.sizeof(H.hill.PrefillDesc), n_new, 8 * 128, 16 * 8 * 128, 128, 8 * 128)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BIG = 1 << 40


def window_attn(H, d=None, q=FAKE, k=FAKE, v=FAKE, lens=None, out=FAKE, ws=FAKE, ws_bytes=BIG):
    return H.load_library().hill_window_attn(ctypes.byref(d or desc(H)), q, k, v, lens, out, ws, ws_bytes, None)


def window_prefill(H, d=None, p=None, q=FAKE, k=FAKE, v=FAKE, lens=None, out=FAKE, ws=FAKE, ws_bytes=BIG):
    return H.load_library().hill_window_prefill(ctypes.byref(d or desc(H)), ctypes.byref(p or prefill(H)), q, k, v, lens, out,
                                                ws, ws_bytes, None)


def packed_attn(H, d=None, p=None, q=FAKE, lens=None, idx=None, k_sel=0, s=None, out=FAKE, ws=FAKE, ws_bytes=BIG):
    return H.load_library().hill_packed_attn(ctypes.byref(d or desc(H)), ctypes.byref(p or packed(H)), q, lens, idx, k_sel, s,
                                             out, ws, ws_bytes, None)


def evict(H, d=None, s=FAKE, keep=500, idx=FAKE, k=FAKE, v=FAKE, p=None, pos=None, pos_st=(1000, 1000), ws=FAKE, ws_bytes=BIG):
    return H.load_library().hill_evict(ctypes.byref(d or desc(H)), s, keep, idx, k, v, None if p is None else ctypes.byref(p),
                                       pos, *pos_st, ws, ws_bytes, None)


BAD_DESC = [("struct_size", 8, INVALID), ("batch", 0, INVALID), ("n_q_heads", 7, INVALID), ("n_tokens", 0, INVALID),
            ("head_dim", 64, UNSUPPORTED), ("dtype", 2, UNSUPPORTED), ("n_tokens", 1 << 22, UNSUPPORTED),
            ("n_sink", -1, INVALID), ("n_recent", -1, INVALID), ("k_stride_n", 100, INVALID), ("v_stride_n", 64, INVALID),
            ("q_stride_h", 4, INVALID), ("sm_scale", float("inf"), INVALID)]


@pytest.mark.parametrize("field,value,code", BAD_DESC)
def test_descriptor(H, field, value, code):
    for call in (window_attn, window_prefill, packed_attn, evict):
        assert call(H, d=desc(H, **{field: value})) == code, call.__name__
        assert H.load_library().hill_last_error()


@pytest.mark.parametrize("name", ["q", "k", "v", "out"])
@pytest.mark.parametrize("bad", [None, FAKE + 2])
def test_pointers(H, name, bad):
    assert window_attn(H, **{name: bad}) == INVALID
    assert window_prefill(H, **{name: bad}) == INVALID
    if name in ("q", "out"):
        assert packed_attn(H, **{name: bad}) == INVALID
    if name in ("k", "v"):
        assert evict(H, **{name: bad}) == INVALID     # one alone, or misaligned


def test_lens_and_workspaces(H):
    lib = H.load_library()
    for call in (window_attn, window_prefill, packed_attn):
        assert call(H, lens=FAKE + 2) == INVALID
    need = ctypes.c_size_t()
    d = desc(H)
    for call, fn, args in ((window_attn, lib.hill_window_workspace_bytes, (0,)),
                           (window_prefill, lib.hill_window_workspace_bytes, (16,)),
                           (packed_attn, lib.hill_packed_workspace_bytes, (0, 0)),
                           (evict, lib.hill_evict_workspace_bytes, (500,))):
        assert fn(ctypes.byref(d), *args, ctypes.byref(need)) == 0
        if need.value:
            assert call(H, d=d, ws_bytes=need.value - 1) == WORKSPACE
            assert call(H, d=d, ws=None, ws_bytes=need.value) == INVALID
            assert call(H, d=d, ws=FAKE + 8, ws_bytes=need.value) == INVALID
        assert fn(ctypes.byref(d), *args, None) == INVALID
    assert need.value > 0
    assert lib.hill_window_workspace_bytes(ctypes.byref(d), -1, ctypes.byref(need)) == INVALID
    assert lib.hill_window_workspace_bytes(ctypes.byref(d), 1001, ctypes.byref(need)) == INVALID
    assert lib.hill_packed_workspace_bytes(ctypes.byref(d), 1001, 0, ctypes.byref(need)) == INVALID
    assert lib.hill_evict_workspace_bytes(ctypes.byref(d), 0, ctypes.byref(need)) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(n_new=0), INVALID), (dict(n_new=1001), INVALID), (dict(struct_size=4), INVALID), (dict(q_stride_t=12), INVALID),
    (dict(q_stride_t=64), INVALID), (dict(o_stride_t=0), INVALID), (dict(o_stride_h=64), INVALID), (dict(o_stride_b=8), INVALID),
    (dict(o_stride_h=-128), INVALID)])
def test_prefill_descriptor(H, kw, code):
    assert window_prefill(H, p=prefill(H, **kw)) == code


@pytest.mark.parametrize("kw", [dict(struct_size=4), dict(cap=0), dict(cap=999), dict(k_codes=None), dict(k_params=FAKE + 4),
                                dict(v_codes=FAKE + 8), dict(v_params=None)])
def test_packed_descriptor(H, kw):
    assert packed_attn(H, p=packed(H, **kw)) == INVALID
    assert evict(H, k=None, v=None, p=packed(H, **kw)) == INVALID


def test_packed_attn_lists_and_importance(H):
    assert packed_attn(H, k_sel=5) == INVALID                                    # a length without a list
    assert packed_attn(H, idx=FAKE, k_sel=0) == INVALID
    assert packed_attn(H, idx=FAKE, k_sel=1001) == INVALID
    assert packed_attn(H, idx=FAKE + 2, k_sel=5) == INVALID
    assert packed_attn(H, idx=FAKE, k_sel=5, lens=FAKE) == INVALID
    assert packed_attn(H, idx=FAKE, k_sel=5, s=FAKE) == INVALID
    assert packed_attn(H, s=FAKE + 4) == INVALID
    assert packed_attn(H, s=FAKE, d=desc(H, s_stride_r=998)) == INVALID


def test_pack_and_unpack_ranges(H):
    lib = H.load_library()
    d, p = desc(H, n=10), packed(H, cap=12)
    call = lambda at=None, at0=0, k=FAKE, v=FAKE, dd=d: lib.hill_pack_kv(ctypes.byref(dd), ctypes.byref(p), k, v, at, at0, None)
    assert call(at0=-1) == INVALID and call(at0=3) == INVALID and call(at0=0x7fffffff) == INVALID
    assert call(at=FAKE + 1) == INVALID
    assert call(k=None) == INVALID and call(v=FAKE + 2) == INVALID and call(dd=desc(H, n=10, head_dim=96)) == UNSUPPORTED
    back = lambda t0, t1, k=FAKE, v=FAKE: lib.hill_unpack_kv(ctypes.byref(d), ctypes.byref(p), t0, t1, k, v, None)
    assert back(-1, 3) == INVALID and back(4, 3) == INVALID and back(0, 13) == INVALID and back(0, 12) == INVALID
    assert back(0, 5, k=None) == INVALID and back(0, 5, v=FAKE + 4) == INVALID


def test_evict_arguments(H):
    assert evict(H, keep=0) == INVALID and evict(H, keep=1001) == INVALID
    assert evict(H, keep=103) == INVALID                                         # 104 pinned tokens
    assert evict(H, s=None) == INVALID and evict(H, idx=None) == INVALID and evict(H, idx=FAKE + 2) == INVALID
    assert evict(H, pos=FAKE + 1) == INVALID
    assert evict(H, pos=FAKE, pos_st=(999, 1000)) == INVALID                     # two sequences' rows overlap
    assert evict(H, d=desc(H, gran=1), pos=FAKE, pos_st=(2000, 999)) == INVALID
    assert evict(H, p=packed(H)) == INVALID                                      # both kinds of cache
    assert evict(H, d=desc(H, k_stride_h=0)) == INVALID and evict(H, d=desc(H, v_stride_b=0)) == INVALID


def test_grids_beyond_the_launch_limit(H):
    d = desc(H, B=1 << 28, n=1000)
    assert window_attn(H, d=d) == UNSUPPORTED and packed_attn(H, d=d) == UNSUPPORTED
    assert window_prefill(H, d=d) == UNSUPPORTED and evict(H, d=d) == UNSUPPORTED


# ---------------------------------------------------------------- the binding --

def test_binding_refuses_cpu_tensors(H):
    q, k = torch.zeros(1, 4, 128), torch.zeros(1, 2, 8, 128)
    s = torch.zeros(1, 1, 8)
    cache = H.new_packed_cache
    for call in (lambda: H.hill_window_attn(q, k, k, window=4), lambda: H.hill_window_prefill(q[:, :, None], k, k, window=4),
                 lambda: H.hill_evict(s, 4, k=k, v=k), lambda: H.WindowAttnCall(q, k, k, window=4), lambda: cache(1, 2, 8, "cpu")):
        with pytest.raises(ValueError, match="GPU tensors only"):
            call()


def meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_binding_checks_shapes_and_types(H, monkeypatch):
    """The checks before the first pointer is taken, on tensors without memory."""
    from paper_2602_18750_amd import cache as C
    monkeypatch.setattr(C, "_device_of", lambda *named: torch.device("meta"))
    q, k = meta(2, 8, 128), meta(2, 2, 50, 128)
    bad = [
        lambda: H.hill_window_attn(q[0], k, k, window=4),
        lambda: H.hill_window_attn(q, k, meta(2, 2, 49, 128), window=4),
        lambda: H.hill_window_attn(q, k.half(), k.half(), window=4),
        lambda: H.hill_window_attn(q, meta(3, 2, 50, 128), meta(3, 2, 50, 128), window=4),
        lambda: H.hill_window_attn(q, k, k, window=-1),
        lambda: H.hill_window_attn(q, k, k, window=4, n_sink=-1),
        lambda: H.hill_window_attn(q, k, k, window=4, n_tokens=51),
        lambda: H.hill_window_attn(q, k, k, window=4, lens=meta(2)),
        lambda: H.hill_window_attn(q, k, k, window=4, lens=meta(3, dtype=torch.int32)),
        lambda: H.hill_window_attn(meta(2, 128, 8).transpose(1, 2), k, k, window=4),
        lambda: H.hill_window_prefill(q, k, k, window=4),
        lambda: H.hill_evict(meta(2, 1, 50), 5, k=k, v=k),
        lambda: H.hill_evict(meta(2, 1, 50, dtype=torch.float32), 5, k=k),
        lambda: H.hill_evict(meta(2, 1, 50, dtype=torch.float32), 51, k=k, v=k),
        lambda: H.hill_evict(meta(2, 1, 50, dtype=torch.float32), -1, k=k, v=k),
        lambda: H.hill_evict(meta(2, 2, 50, dtype=torch.float32), 5, k=k, v=k),
        lambda: H.hill_evict(meta(2, 1, 50, dtype=torch.float32), 5, k=k, v=k, granularity="kvhead"),
        lambda: H.hill_evict(meta(2, 1, 50, dtype=torch.float32), 5, k=k, v=k, pos=meta(2, 1, 40, dtype=torch.int32)),
        lambda: H.hill_evict(meta(2, 1, 50, dtype=torch.float32), 5, k=k, v=k, pos=meta(2, 1, 50, dtype=torch.int64)),
        lambda: H.hill_evict(meta(2, 1, 60, dtype=torch.float32), 5, k=k, v=k),
        lambda: H.PackedCache(meta(1, 2, 8, 64), meta(1, 2, 8, 4, 2), meta(1, 2, 8, 64), meta(1, 2, 8, 4, 2)),
        lambda: H.PackedCache(meta(1, 2, 8, 64, dtype=torch.uint8), meta(1, 2, 8, 4, 2, dtype=torch.float16),
                              meta(1, 2, 9, 64, dtype=torch.uint8), meta(1, 2, 8, 4, 2, dtype=torch.float16)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was accepted" % i)
