"""Window attention, the 4-bit cache and eviction as a decoding program runs
them: together, captured, on other streams, with whatever a workspace holds,
and with offsets beyond 32 bits."""
import sys

import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128


def H():
    import paper_2602_18750_amd as H
    return H


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, file=sys.stderr, flush=True)


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def test_prefill_pack_decode_evict():
    """A bounded 4-bit cache: a windowed prefill, its K and V packed, decode steps that append a token and add the
    weights to S, an eviction that keeps a third, more steps.  Every output against the 64-bit form on the values
    held and the positions kept."""
    B, Hq, Hkv, T, cap, sink, window, keep = 2, 8, 2, 150, 200, 4, 40, 60
    G = Hq // Hkv
    k, v = randn((B, Hkv, T, D), torch.bfloat16, 1), randn((B, Hkv, T, D), torch.bfloat16, 2)
    q = randn((B, Hq, T, D), torch.bfloat16, 3)
    out = H().hill_window_prefill(q, k, v, window=window, n_sink=sink)
    for b in range(B):
        for g in range(Hkv):
            hs = slice(g * G, (g + 1) * G)
            want, bound, spread, _, _ = R.attend(q[b, hs], k[b, g], v[b, g], R.visible_mask(torch.arange(T), T, sink, window))
            u = 2.0 ** -8     # weights and output rounded to bf16
            assert ((out[b, hs].cpu().double() - want).abs() <= bound + u * spread + u * (1 + u) * want.abs() + 2.0 ** -25).all()
    cache = H().pack_kv(k, v, H().new_packed_cache(B, Hkv, cap, DEV))
    held_k, held_v = R.quantise(k)[3], R.quantise(v)[3]
    s = H().new_importance(B, Hkv, cap, DEV)
    pos = torch.arange(cap, device=DEV, dtype=torch.int32).expand(B, Hkv, cap).contiguous()
    want_s, tol_s = torch.zeros(B, Hkv, cap, dtype=torch.float64), torch.zeros(B, Hkv, cap, dtype=torch.float64)
    n = T
    for step in range(12):
        if step == 6:
            got_s = s.cpu()[..., :n]
            idx = H().hill_evict(s, keep, cache=cache, pos=pos, n_tokens=n, granularity="kvhead", n_sink=sink, n_recent=20)
            want_idx = R.kept(got_s, keep, sink, 20)
            assert torch.equal(idx.cpu().long(), want_idx)
            assert torch.equal(pos.cpu()[..., :keep].long(), want_idx)         # positions were 0, 1, ... until now
            assert torch.equal(s.cpu()[..., :keep], got_s.gather(-1, want_idx)) and (s[..., keep:n] == 0).all()
            rows = want_idx[..., None].expand(B, Hkv, keep, D)
            held_k, held_v = held_k.gather(2, rows), held_v.gather(2, rows)
            want_s[..., :keep], tol_s[..., :keep] = want_s.gather(-1, want_idx), tol_s.gather(-1, want_idx)
            want_s[..., keep:] = tol_s[..., keep:] = 0
            n = keep
        kn, vn, qn = (randn((B, h, 1, D), torch.bfloat16, 100 + 3 * step + i) for i, h in enumerate((Hkv, Hkv, Hq)))
        H().pack_kv(kn, vn, cache, at=n)
        held_k, held_v = torch.cat((held_k, R.quantise(kn)[3]), 2), torch.cat((held_v, R.quantise(vn)[3]), 2)
        n += 1
        out = H().hill_packed_attn(qn[:, :, 0], cache, n_tokens=n, s=s, granularity="kvhead")
        for b in range(B):
            for g in range(Hkv):
                hs = slice(g * G, (g + 1) * G)
                want, bound, _, w, e_w = R.attend(qn[b, hs], held_k[b, g], held_v[b, g], torch.ones(1, n, dtype=torch.bool))
                assert ((out[b, hs].cpu().double() - want[:, 0]).abs() <= bound[:, 0]).all(), step
                want_s[b, g, :n] += w.sum((0, 1))
                tol_s[b, g, :n] += (w * (2 * e_w + (n / 32 + 64 + Hq) * 2 * R.F32)).sum((0, 1)) + want_s[b, g, :n] * 2 * R.F32
        assert ((s.cpu().double() - want_s).abs() <= tol_s + 1e-30).all(), step


def step_inputs(B=3, Hq=16, Hkv=4, cap=700):
    k, v = randn((B, Hkv, cap, D), torch.float16, 1), randn((B, Hkv, cap, D), torch.float16, 2)
    q = randn((B, Hq, D), torch.float16, 3)
    lens = torch.tensor([300, 1, 650], dtype=torch.int32, device=DEV)[:B].contiguous()
    return k, v, q, lens


def test_captured_steps_equal_eager_ones():
    """A captured step (append at the lengths, lengths + 1, window attention, packed attention with S, the last
    tokens' prefill) replayed with eager work between, against eager steps, bit for bit."""
    k, v, q, lens0 = step_inputs()
    kn, vn = randn((3, 4, 1, D), torch.float16, 7), randn((3, 4, 1, D), torch.float16, 8)

    def fresh():
        st = dict(lens=lens0.clone(), cache=H().pack_kv(k, v, H().new_packed_cache(3, 4, 700, DEV)), s=H().new_importance(3, 1, 700, DEV))
        st["w"] = H().WindowAttnCall(q, k, v, window=90, n_sink=4, lens=st["lens"])
        st["p"] = H().PackedAttnCall(q, st["cache"], lens=st["lens"], s=st["s"])
        return st

    def step(st):
        H().pack_kv(kn, vn, st["cache"], at=st["lens"])
        st["lens"].add_(1)
        st["w"](q.data_ptr())
        st["p"](q.data_ptr())
        st["f"] = H().hill_window_attn(q, k, v, window=90, n_sink=4, lens=st["lens"])
        st["c"] = H().hill_window_prefill(q[:, :, None], k, v, window=90, n_sink=4, lens=st["lens"])

    eager, graph = fresh(), fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph["w"] = H().WindowAttnCall(q, k, v, window=90, n_sink=4, lens=graph["lens"])
        graph["p"] = H().PackedAttnCall(q, graph["cache"], lens=graph["lens"], s=graph["s"])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(graph)
    torch.cuda.synchronize()
    for t in range(4):
        step(eager)
        junk = torch.randn(1 << 20, device=DEV).sort().values.sum()       # other work between the replays
        g.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(junk)
        assert torch.equal(eager["lens"], graph["lens"]) and int(graph["lens"][1]) == 2 + t
        for name in ("f", "c"):
            assert torch.equal(eager[name], graph[name]), (t, name)
        assert torch.equal(eager["w"].out, graph["w"].out) and torch.equal(eager["w"].out, eager["f"])
        assert torch.equal(eager["p"].out, graph["p"].out) and torch.equal(eager["s"], graph["s"])
        assert torch.equal(eager["cache"].k_codes, graph["cache"].k_codes)


@pytest.mark.parametrize("n", [3000, 40000])
def test_captured_eviction(n):
    """An eviction in a graph, replayed over new importance each time."""
    keep = n // 3
    k, v = randn((1, 2, n, D), torch.bfloat16, 1), randn((1, 2, n, D), torch.bfloat16, 2)
    s = H().new_importance(1, 1, n, DEV)
    ke, ve, se = k.clone(), v.clone(), s.clone()
    s.uniform_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        idx = H().hill_evict(s, keep, k=k, v=v)
    for t in range(3):
        x = torch.rand((1, 1, n), generator=torch.Generator().manual_seed(t)).to(DEV)
        s.copy_(x)
        se.copy_(x)
        g.replay()
        want = H().hill_evict(se, keep, k=ke, v=ve)
        torch.cuda.synchronize()
        assert torch.equal(idx, want) and torch.equal(s, se) and torch.equal(k, ke) and torch.equal(v, ve)


def test_other_streams_and_two_at_once():
    """Calls given a stream (an object or its pointer) run there, and two at a time do not share scratch."""
    n = 6000
    k, v = randn((1, 8, n, D), torch.bfloat16, 1), randn((1, 8, n, D), torch.bfloat16, 2)
    q = randn((2, 1, 32, D), torch.bfloat16, 3)
    cache = H().pack_kv(k, v, H().new_packed_cache(1, 8, n, DEV))
    want = [(H().hill_window_attn(x, k, v, window=n), H().hill_packed_attn(x, cache)) for x in q]
    kk = [(k.clone(), v.clone(), torch.rand((1, 1, n), generator=torch.Generator().manual_seed(i)).to(DEV)) for i in range(2)]
    ref = [(a.clone(), b.clone(), s.clone()) for a, b, s in kk]
    for a, b, s in ref:
        H().hill_evict(s, 2000, k=a, v=b)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for x, st in zip(q, streams):
            given = st.cuda_stream if x is q[0] else st
            got.append((H().hill_window_attn(x, k, v, window=n, stream=given), H().hill_packed_attn(x, cache, stream=given)))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for (a, b, s), st in zip(kk, streams):
        H().hill_evict(s, 2000, k=a, v=b, stream=st)
    torch.cuda.synchronize()
    for x, y in zip(kk, ref):
        assert all(torch.equal(a, b) for a, b in zip(x, y))


def test_workspace_contents_and_repeats():
    """A workspace of the exact size full of NaN bits gives what the call's own gives, and repeats are equal."""
    import ctypes
    from paper_2602_18750_amd import cache as C
    lib = H().load_library()
    k, v, q, lens = step_inputs()
    cache = H().pack_kv(k, v, H().new_packed_cache(3, 4, 700, DEV))

    def full(fn, d, *args):
        need = ctypes.c_size_t()
        assert fn(ctypes.byref(d), *args, ctypes.byref(need)) == 0
        return torch.full((need.value,), 0xff, dtype=torch.uint8, device=DEV)

    d, _ = C._window_desc(q, k, v, lens, None, 400, 4, 0.0, 3)
    a = H().hill_window_attn(q, k, v, window=400, n_sink=4, lens=lens)
    for _ in range(2):
        assert torch.equal(a, H().hill_window_attn(q, k, v, window=400, n_sink=4, lens=lens, ws=full(lib.hill_window_workspace_bytes, d, 0)))
    a = H().hill_window_prefill(q[:, :, None], k, v, window=400, n_sink=4, lens=lens)
    b = H().hill_window_prefill(q[:, :, None], k, v, window=400, n_sink=4, lens=lens, ws=full(lib.hill_window_workspace_bytes, d, 1))
    assert torch.equal(a, b)
    ss = [H().new_importance(3, 4, 700, DEV) for _ in range(2)]
    d, _ = C._packed_desc(q, cache, None, lens, 0, None, None, ss[0], "kvhead", 0.0)
    a = H().hill_packed_attn(q, cache, lens=lens, s=ss[0], granularity="kvhead")
    b = H().hill_packed_attn(q, cache, lens=lens, s=ss[1], granularity="kvhead", ws=full(lib.hill_packed_workspace_bytes, d, 0, 1))
    assert torch.equal(a, b) and torch.equal(ss[0], ss[1])
    s0 = torch.rand((3, 4, 700), device=DEV)
    s1, k1, v1 = s0.clone(), k.clone(), v.clone()
    d = C._desc(3, 4, 4, D, 700, torch.float16, s_st=(2800, 700), granularity="kvhead")
    i0 = H().hill_evict(s0, 333, k=k, v=v, granularity="kvhead")
    i1 = H().hill_evict(s1, 333, k=k1, v=v1, granularity="kvhead", ws=full(lib.hill_evict_workspace_bytes, d, 333))
    assert torch.equal(i0, i1) and torch.equal(s0, s1) and torch.equal(k, k1) and torch.equal(v, v1)


@pytest.mark.parametrize("stride,n", [(1 << 21, 1100), (1 << 25, 70)])
def test_rows_beyond_32_bit_offsets(stride, n):
    """Caches whose token stride puts the last rows past 2^31 elements."""
    kv = [torch.empty_strided((1, 1, n, D), (n * stride, n * stride, stride, 1), dtype=torch.float16, device=DEV) for _ in range(2)]
    flat = [randn((1, 1, n, D), torch.float16, i) for i in range(2)]
    for x, y in zip(kv, flat):
        x.copy_(y)
    q = randn((1, 4, D), torch.float16, 5)
    args = dict(window=n - 40, n_sink=3)
    assert torch.equal(H().hill_window_attn(q, *kv, **args), H().hill_window_attn(q, *flat, **args))
    qq = randn((1, 4, n, D), torch.float16, 6)
    assert torch.equal(H().hill_window_prefill(qq, *kv, **args), H().hill_window_prefill(qq, *flat, **args))
    a, b = (H().pack_kv(*x, H().new_packed_cache(1, 1, n, DEV)) for x in (kv, flat))
    assert torch.equal(a.k_codes, b.k_codes) and torch.equal(a.v_params, b.v_params)
    back = H().unpack_kv(a, k_out=torch.empty_like(flat[0]), v_out=torch.empty_strided(kv[0].shape, kv[0].stride(), dtype=torch.float16, device=DEV))
    assert torch.equal(back[1], H().unpack_kv(b)[1])
    s = H().new_importance(1, 1, n, DEV).copy_(torch.rand((1, 1, n), device=DEV))
    s2 = s.clone()
    i, j = H().hill_evict(s, n // 2, k=kv[0], v=kv[1]), H().hill_evict(s2, n // 2, k=flat[0], v=flat[1])
    assert torch.equal(i, j) and torch.equal(kv[0], flat[0]) and torch.equal(kv[1], flat[1])


def test_packed_cache_beyond_4_gib():
    B, Hkv, cap, n = 1, 36, 1 << 21, 90
    cache = H().PackedCache(*(torch.empty((B, Hkv, cap) + s, dtype=t, device=DEV)
                              for s, t in (((64,), torch.uint8), ((4, 2), torch.float16)) * 2))
    small = H().new_packed_cache(B, Hkv, n, DEV)
    k, v = randn((B, Hkv, n, D), torch.bfloat16, 1), randn((B, Hkv, n, D), torch.bfloat16, 2)
    at = cap - n
    H().pack_kv(k, v, cache, at=at)
    H().pack_kv(k, v, cache)
    H().pack_kv(k, v, small)
    q = randn((B, Hkv, D), torch.bfloat16, 3)
    want = H().hill_packed_attn(q, small)
    assert torch.equal(H().hill_packed_attn(q, cache, n_tokens=n), want)
    idx = torch.arange(at, cap, device=DEV, dtype=torch.int32).view(1, 1, n)
    far = H().hill_packed_attn(q, cache, idx=idx)
    assert torch.equal(far, H().hill_packed_attn(q, small, idx=idx - at))
    assert all(torch.equal(x, y) for x, y in zip(H().unpack_kv(cache, token_begin=at), H().unpack_kv(small)))
