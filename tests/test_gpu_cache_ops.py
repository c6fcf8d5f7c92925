"""Window attention, the 4-bit cache and eviction on the GPU against their
plain 64-bit forms (tests/cache_ref.py, where the bounds are derived)."""
import math
import sys

import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}     # half a step, relative


def H():
    import paper_2602_18750_amd as H
    return H


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, file=sys.stderr, flush=True)


def draw(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def check_decode(got, q, k, v, lens, sink, window, scale=None):
    """got [B, Hq, D] against the 64-bit attention of q over k, v [B, Hkv, m, D] (values as held)."""
    B, Hq, _ = q.shape
    G = Hq // k.shape[1]
    got = got.cpu().double()
    for b in range(B):
        n = lens[b]
        mask = R.visible_mask([n - 1], n, sink, window)
        for g in range(k.shape[1]):
            hs = slice(g * G, (g + 1) * G)
            out, bound, _, _, _ = R.attend(q[b, hs, None], k[b, g, :n], v[b, g, :n], mask, scale)
            err = (got[b, hs] - out[:, 0]).abs()
            assert (err <= bound[:, 0]).all(), (b, g, err.max(), bound.min())


WINDOW_CASES = [  # B, Hq, Hkv, n, sink, window, lens
    (1, 1, 1, 1, 0, 1, None),
    (1, 4, 2, 1, 4, 16, None),
    (2, 8, 2, 31, 4, 7, None),
    (1, 8, 8, 33, 0, 33, None),
    (2, 28, 4, 517, 4, 100, (517, 3)),
    (3, 6, 2, 300, 64, 64, (0, 1, 300)),
    (2, 8, 8, 1000, 1, 31, (999, 40)),
    (1, 40, 2, 700, 5, 300, None),          # 20 heads per KV head: two head tiles
    (1, 128, 1, 200, 3, 90, None),
    (2, 4, 2, 260, 0, 0, None),             # nothing visible
    (1, 4, 2, 260, 17, 0, None),            # sinks alone
    (1, 8, 2, 5000, 4, 4096, None),         # several shares, an odd window
    (4, 8, 2, 4097, 31, 2 ** 31 - 1, (4097, 4096, 33, 2)),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("case", WINDOW_CASES)
def test_window_attn(case, dtype):
    B, Hq, Hkv, n, sink, window, lens = case
    q, k, v = draw((B, Hq, D), dtype, n), draw((B, Hkv, n, D), dtype, n + 1), draw((B, Hkv, n, D), dtype, n + 2)
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = H().hill_window_attn(q.to(DEV), k.to(DEV), v.to(DEV), window=window, n_sink=sink, lens=dl)
    check_decode(out, q, k, v, lens or [n] * B, sink, window)


def plain_decode(q, k, v, lens, sink, window):
    """64-bit decode on the GPU, all rows at once: q [B, Hq, D], k, v [B, Hkv, n, D]."""
    B, Hq, _ = q.shape
    Hkv, n = k.shape[1], k.shape[2]
    j = torch.arange(n, device=DEV)
    m = torch.as_tensor(lens, device=DEV).view(B, 1)
    seen = ((j < m) & ((j < sink) | (j >= m - window))).view(B, 1, 1, n)
    x = torch.matmul(q.double().view(B, Hkv, Hq // Hkv, D), k.double().transpose(2, 3).contiguous()) * D ** -0.5
    e = torch.where(seen, torch.exp(x - x.masked_fill(~seen, -1e300).amax(-1, keepdim=True)), torch.zeros_like(x))
    w = e / e.sum(-1, keepdim=True)
    return torch.matmul(w, v.double()).view(B, Hq, D), w


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("held", ["16-bit", "packed"])
@pytest.mark.parametrize("sink,window", [(4, 700), (40, 612), (33, 900), (0, 0x7fffffff), (64, 64)])
def test_many_tiles_per_wave(sink, window, held, dtype):
    """Enough sequences that every wave walks several tiles: the first one across the sinks' end, the last one
    partial, ragged lengths between."""
    B, Hq, Hkv, n = 33, 16, 8, 1001
    g = torch.Generator(device=DEV).manual_seed(sink + 7)
    q = torch.randn((B, Hq, D), generator=g, device=DEV).to(dtype)
    k, v = (torch.randn((B, Hkv, n, D), generator=g, device=DEV).to(dtype) for _ in range(2))
    lens = torch.randint(1, n + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    lens[0], lens[1], lens[2] = n, 1, 33
    if held == "packed":
        cache = H().pack_kv(k, v, H().new_packed_cache(B, Hkv, n, DEV))
        out = H().hill_packed_attn(q, cache, lens=lens, n_sink=sink, window=window)
        k, v = H().unpack_kv(cache)
    else:
        out = H().hill_window_attn(q, k, v, window=window, n_sink=sink, lens=lens)
    want, w = plain_decode(q, k, v, lens, sink, window)
    # as check_decode's bound, with the largest row's products for all and sum w |V| <= max |V|
    size = torch.matmul(q.double().abs().view(B, Hkv, 2, D), k.double().abs().transpose(2, 3).contiguous()).amax(-1) * D ** -0.5
    bound = (2 * (size * (D * R.F32 + 4 * R.F32 * 1.4427) + 8 * R.F32) + 2 * (n / 32 + 64) * R.F32).view(B, Hq, 1) * v.abs().max()
    assert ((out.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("scale", [0.0, 0.5, -0.2])
def test_window_attn_strides_scales_and_unseen_rows(scale):
    """A [B, n, 2, Hkv, D] cache (K and V interleaved), more rows than tokens, a view of q, rows that no query sees
    full of NaN and infinities."""
    B, Hq, Hkv, n, cap = 2, 6, 3, 333, 400
    kv = draw((B, cap, 2, Hkv, D), torch.bfloat16, 1)
    q = draw((B, Hq, 3, D), torch.bfloat16, 2)
    lens = [333, 150]
    bad = kv.clone()
    for b, m in enumerate(lens):
        bad[b, m:] = float("nan")
        bad[b, 5:m - 60, 0] = float("inf")
        bad[b, 5:m - 60, 1] = float("nan")
    x = bad.to(DEV)
    out = H().hill_window_attn(q.to(DEV)[:, :, 1], x[:, :, 0].transpose(1, 2), x[:, :, 1].transpose(1, 2), window=60, n_sink=5,
                               n_tokens=n, lens=torch.tensor(lens, dtype=torch.int32, device=DEV), sm_scale=scale)
    check_decode(out, q[:, :, 1], kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2), lens, 5, 60,
                 scale or None)


def test_window_attn_large_logits():
    """Logits over hundreds, both signs, and a row whose largest comes last."""
    n = 700
    q, k, v = draw((1, 4, D), torch.float16, 1, 6.0), draw((1, 2, n, D), torch.float16, 2, 6.0), draw((1, 2, n, D), torch.float16, 3)
    k[:, :, -1] = k[:, :, 0] * 3
    out = H().hill_window_attn(q.to(DEV), k.to(DEV), v.to(DEV), window=n)
    assert torch.isfinite(out).all()
    check_decode(out, q, k, v, [n], 0, n)


PREFILL_CASES = [  # B, Hq, Hkv, n, T, sink, window, lens
    (1, 1, 1, 1, 1, 0, 1, None),
    (1, 4, 2, 65, 65, 0, 65, None),
    (2, 8, 2, 200, 200, 4, 50, None),
    (1, 28, 4, 131, 37, 3, 20, None),
    (1, 8, 8, 300, 300, 64, 64, None),
    (2, 6, 2, 400, 129, 70, 130, (400, 400)),
    (3, 4, 1, 257, 100, 2, 40, (257, 60, 0)),     # shorter than the chunk, and empty
    (1, 5, 1, 500, 3, 9, 444, None),
    (1, 4, 4, 300, 150, 0, 0, None),              # nothing visible
    (1, 4, 4, 300, 290, 33, 0, None),             # sinks alone, most of them after some queries
    (1, 2, 2, 640, 640, 0, 1, None),              # itself alone
    (1, 8, 2, 1500, 1, 4, 1024, None),
    (1, 4, 2, 900, 900, 0, 2 ** 31 - 1, None),    # causal
]


def check_prefill(got, q, k, v, lens, sink, window, scale=None):
    B, Hq, T, _ = q.shape
    G = Hq // k.shape[1]
    u = HALF[q.dtype]
    got = got.cpu().double()
    for b in range(B):
        n = lens[b]
        mask = R.visible_mask(torch.arange(n - T, n), n, sink, window)
        for g in range(k.shape[1]):
            hs = slice(g * G, (g + 1) * G)
            out, bound, spread, _, _ = R.attend(q[b, hs], k[b, g, :n], v[b, g, :n], mask, scale)
            # weights rounded to 16 bits, the output too; fp16 weights below 2^-14 lose 2^-25 each, out of a total >= 1
            tol = bound + u * spread + u * out.abs() * (1 + u) + 2.0 ** -25
            if q.dtype == torch.float16 and n:
                tol = tol + mask.sum(-1).reshape(1, -1, 1) * 2.0 ** -25 * v[b, g, :n].double().abs().max()
            err = (got[b, hs] - out).abs()
            assert (err <= tol).all(), (b, g, (err - tol).max(), err.max())
            assert (got[b, hs][:, ~mask.any(-1)] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("case", PREFILL_CASES)
def test_window_prefill(case, dtype):
    B, Hq, Hkv, n, T, sink, window, lens = case
    q, k, v = draw((B, Hq, T, D), dtype, n), draw((B, Hkv, n, D), dtype, n + 1), draw((B, Hkv, n, D), dtype, n + 2)
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = H().hill_window_prefill(q.to(DEV), k.to(DEV), v.to(DEV), window=window, n_sink=sink, lens=dl)
    assert out.dtype == dtype and out.shape == q.shape
    check_prefill(out, q, k, v, lens or [n] * B, sink, window)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,Hq,Hkv,n,T,sink,window", [
    (33, 16, 8, 500, 150, 5, 170),       # eight-wave workgroups, two blocks of 256 rows
    (20, 8, 8, 400, 130, 40, 100),       # four-wave workgroups, one share
    (2, 8, 2, 3000, 5, 9, 2500),         # few rows: many shares
    (1, 12, 4, 2100, 100, 0, 2100),
])
def test_window_prefill_block_forms(B, Hq, Hkv, n, T, sink, window, dtype):
    """Every form of a block and its shares, ragged lengths (some below the chunk) among them."""
    g = torch.Generator(device=DEV).manual_seed(n)
    q = torch.randn((B, T, Hq, D), generator=g, device=DEV).to(dtype).transpose(1, 2)
    k, v = (torch.randn((B, Hkv, n, D), generator=g, device=DEV).to(dtype) for _ in range(2))
    lens = torch.randint(1, n + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    lens[0] = n
    if B > 2:
        lens[1], lens[2] = T // 2, 0
    out = H().hill_window_prefill(q, k, v, window=window, n_sink=sink, lens=lens)
    assert out.stride() == q.stride()
    j = torch.arange(n, device=DEV)
    p = lens.view(B, 1, 1) - T + torch.arange(T, device=DEV).view(1, T, 1)
    seen = ((j <= p) & ((j < sink) | (p - j < window))).view(B, 1, 1, T, n)
    x = torch.matmul(q.double().reshape(B, Hkv, Hq // Hkv * T, D), k.double().transpose(2, 3).contiguous()) * D ** -0.5
    x = x.view(B, Hkv, Hq // Hkv, T, n).masked_fill(~seen, -1e300)
    e = torch.where(seen, torch.exp(x - x.amax(-1, keepdim=True)), torch.zeros_like(x))
    w = e / e.sum(-1, keepdim=True).clamp_min(1e-300)
    want, spread = (torch.matmul(w.view(B, Hkv, -1, n), y.double()).view(B, Hq, T, D) for y in (v, v.abs()))
    size = torch.matmul(q.double().abs().reshape(B, Hkv, -1, D), k.double().abs().transpose(2, 3).contiguous()).amax() * D ** -0.5
    u = HALF[dtype]
    # as check_prefill's, the largest products for every row
    tol = (2 * (size * (D * R.F32 + 4 * R.F32 * 1.4427) + 8 * R.F32) + 2 * (n / 32 + 64) * R.F32 + u) * spread
    tol = tol + u * (1 + u) * want.abs() + 2.0 ** -25 + (n * 2.0 ** -25 * v.abs().max().double() if dtype == torch.float16 else 0)
    assert ((out.double() - want).abs() <= tol).all(), ((out.double() - want).abs() - tol).max()
    assert (out.double()[~seen.any(-1).expand(B, Hkv, Hq // Hkv, T).reshape(B, Hq, T)] == 0).all()


@pytest.mark.parametrize("scale", [0.0, 0.4, -0.3])
def test_window_prefill_strides_scales_and_unseen_rows(scale):
    """Token-major q, out and cache; rows that no query sees full of NaN; what lies between out's rows is left."""
    B, Hq, Hkv, n, T, cap = 2, 6, 2, 300, 70, 320
    q, kv = draw((B, T, Hq, D), torch.bfloat16, 1), draw((B, cap, 2, Hkv, D), torch.bfloat16, 2)
    lens = [300, 180]
    bad = kv.clone()
    for b, m in enumerate(lens):
        bad[b, m:] = float("nan")
        bad[b, 6:m - T - 30] = float("nan")
    x = bad.to(DEV)
    buf = torch.full((B, T, Hq, D + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    out = buf[..., :D].transpose(1, 2)
    H().hill_window_prefill(q.to(DEV).transpose(1, 2), x[:, :, 0].transpose(1, 2), x[:, :, 1].transpose(1, 2), window=30, n_sink=6,
                            n_tokens=n, lens=torch.tensor(lens, dtype=torch.int32, device=DEV), sm_scale=scale, out=out)
    check_prefill(out, q.transpose(1, 2), kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2), lens, 6, 30, scale or None)
    assert (buf[..., D:] == 7.0).all()


def test_prefill_of_one_token_is_the_decode():
    n = 777
    q, k, v = (draw(s, torch.float16, i).to(DEV) for i, s in enumerate([(2, 8, D), (2, 2, n, D), (2, 2, n, D)]))
    a = H().hill_window_attn(q, k, v, window=100, n_sink=4)
    b = H().hill_window_prefill(q[:, :, None], k, v, window=100, n_sink=4)[:, :, 0]
    assert (a - b.float()).abs().max() <= 2.0 ** -10 * v.abs().max()


# --------------------------------------------------------------- 4-bit cache --

def odd_rows(shape, dtype, seed):
    """Rows with outlier channels, constant groups, zeros, large offsets and tiny spreads."""
    x = draw(shape, torch.float32, seed) * torch.exp(draw((D,), torch.float32, seed + 1))
    flat = x.view(-1, D)
    flat[0] = 0.0
    if flat.shape[0] > 4:
        flat[1, :32] = 3.75
        flat[2, 32:64] = 500.0 + flat[2, 32:64] * 0.25
        flat[3, 64:96] *= 1e-6
        flat[4, 96:] *= 1e-3
        flat[4, 96] = 60000.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,Hkv,T,cap,at", [(1, 1, 1, 1, 0), (2, 3, 65, 80, 7), (1, 2, 257, 257, 0), (2, 1, 5, 12, (3, 9))])
def test_pack_and_unpack(B, Hkv, T, cap, at, dtype):
    """Codes, scales, zeros and values bit for bit; rows outside the written ones, and rows dropped, stay."""
    k, v = odd_rows((B, Hkv, T, D), dtype, T), odd_rows((B, Hkv, T, D), dtype, T + 9)
    cache = H().new_packed_cache(B, Hkv, cap, DEV)
    for t in (cache.k_codes, cache.v_codes):
        t.fill_(0x5a)
    dat = at if isinstance(at, int) else torch.tensor(at, dtype=torch.int32, device=DEV)
    H().pack_kv(k.to(DEV), v.to(DEV), cache, at=dat)
    ku, vu = H().unpack_kv(cache)
    kb, vb = H().unpack_kv(cache, dtype=torch.bfloat16)
    for x, codes, params, back, back16 in ((k, cache.k_codes, cache.k_params, ku, kb), (v, cache.v_codes, cache.v_params, vu, vb)):
        code, scale, zero, value = R.quantise(x)
        for b in range(B):
            a0 = at if isinstance(at, int) else at[b]
            m = min(T, cap - a0)
            rows = slice(a0, a0 + m)
            assert torch.equal(R.codes_of(codes[b, :, rows]), code[b, :, :m])
            assert torch.equal(params[b, :, rows, :, 0].cpu(), scale[b, :, :m])
            assert torch.equal(params[b, :, rows, :, 1].cpu(), zero[b, :, :m])
            assert torch.equal(back[b, :, rows].cpu(), value[b, :, :m])
            assert torch.equal(back16[b, :, rows].cpu(), value[b, :, :m].bfloat16())
            rest = [j for j in range(cap) if not a0 <= j < a0 + m]
            assert (codes[b, :, rest] == 0x5a).all() and (params[b, :, rest] == 0).all()


def test_pack_out_of_range_and_unpack_into_views():
    cache = H().new_packed_cache(2, 2, 10, DEV)
    k = draw((2, 2, 4, D), torch.float16, 1).to(DEV)
    H().pack_kv(k, k, cache, at=torch.tensor([-2, 8], dtype=torch.int32, device=DEV))
    value = R.quantise(k)[3]
    buf = torch.full((2, 10, 2, 2, D), -1.0, dtype=torch.float16, device=DEV)
    ko, vo = buf[:, 1:9, 0].transpose(1, 2), buf[:, 1:9, 1].transpose(1, 2)
    H().unpack_kv(cache, token_begin=2, token_end=10, k_out=ko, v_out=vo)
    assert torch.equal(cache.k_codes[0, :, 2:].cpu(), torch.zeros(2, 8, 64, dtype=torch.uint8))
    assert torch.equal(ko[1, :, 6:].cpu(), value[1, :, :2]) and torch.equal(vo[1, :, 6:].cpu(), value[1, :, :2])
    assert (buf[:, 0] == -1).all() and (buf[:, 9] == -1).all()
    full = H().unpack_kv(cache, token_begin=0, token_end=2)[0]
    assert torch.equal(full[0].cpu(), value[0, :, 2:])
    assert H().unpack_kv(cache, token_begin=3, token_end=3)[0].shape == (2, 2, 0, D)


def packed(B, Hkv, n, dtype, seed):
    k, v = odd_rows((B, Hkv, n, D), dtype, seed), odd_rows((B, Hkv, n, D), dtype, seed + 5)
    k[k.abs() > 100] = 1.0
    v[v.abs() > 100] = 1.0
    cache = H().new_packed_cache(B, Hkv, n + 3, DEV)
    H().pack_kv(k.to(DEV), v.to(DEV), cache)
    return cache, R.quantise(k)[3], R.quantise(v)[3]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("case", [c for c in WINDOW_CASES if c[3] < 6000])
def test_packed_attn(case, dtype):
    B, Hq, Hkv, n, sink, window, lens = case
    cache, kv, vv = packed(B, Hkv, n, dtype, n)
    q = draw((B, Hq, D), dtype, 3)
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = H().hill_packed_attn(q.to(DEV), cache, n_tokens=n, lens=dl, n_sink=sink, window=window)
    check_decode(out, q, kv, vv, lens or [n] * B, sink, window)
    if lens is None:
        check_decode(H().hill_packed_attn(q.to(DEV), cache, n_tokens=n), q, kv, vv, [n] * B, 0, n)


@pytest.mark.parametrize("rows", ["token", "kvhead"])
@pytest.mark.parametrize("B,Hq,Hkv,n,k", [(1, 4, 2, 50, 1), (2, 28, 4, 777, 200), (2, 8, 8, 3000, 999)])
def test_packed_attn_over_a_selection(B, Hq, Hkv, n, k, rows):
    cache, kv, vv = packed(B, Hkv, n, torch.bfloat16, n)
    rr = 1 if rows == "token" else Hkv
    q = draw((B, Hq, D), torch.bfloat16, 3)
    g = torch.Generator().manual_seed(k)
    idx = torch.stack([torch.randperm(n, generator=g)[:k] for _ in range(B * rr)]).view(B, rr, k)   # any order
    out = H().hill_packed_attn(q.to(DEV), cache, n_tokens=n, idx=idx.to(torch.int32).to(DEV), granularity=rows)
    G = Hq // Hkv
    for b in range(B):
        for h in range(Hkv):
            j = idx[b, h if rr > 1 else 0]
            hs = slice(h * G, (h + 1) * G)
            want, bound, _, _, _ = R.attend(q[b, hs, None], kv[b, h, j], vv[b, h, j], torch.ones(1, k, dtype=torch.bool))
            assert ((out[b, hs].cpu().double() - want[:, 0]).abs() <= bound[:, 0]).all()


@pytest.mark.parametrize("rows", ["token", "kvhead"])
@pytest.mark.parametrize("case", WINDOW_CASES)
def test_packed_attn_adds_the_weights(case, rows):
    B, Hq, Hkv, n, sink, window, lens = case
    cache, kv, vv = packed(B, Hkv, n, torch.float16, n)
    q = draw((B, Hq, D), torch.float16, 3)
    G, rr = Hq // Hkv, 1 if rows == "token" else Hkv
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    s = H().new_importance(B, rr, n, DEV)
    s.copy_(draw((B, rr, n), torch.float32, 8).abs())
    want, tol = s.cpu().double(), torch.full((B, rr, n), 1e-30, dtype=torch.float64)
    out = H().hill_packed_attn(q.to(DEV), cache, n_tokens=n, lens=dl, n_sink=sink, window=window, s=s, granularity=rows)
    check_decode(out, q, kv, vv, lens or [n] * B, sink, window)
    for b in range(B):
        m = n if lens is None else lens[b]
        mask = R.visible_mask([m - 1], m, sink, window)
        for h in range(Hkv):
            _, _, _, w, e_w = R.attend(q[b, h * G:(h + 1) * G, None], kv[b, h, :m], vv[b, h, :m], mask)
            row = h if rr > 1 else 0
            want[b, row, :m] += w.sum((0, 1))
            # weight: exponential, its sum and the division; then one addition per head
            tol[b, row, :m] += (w * (2 * e_w + (m / 32 + 64 + Hq) * 2 * R.F32)).sum((0, 1))
    got = s.cpu().double()
    assert ((got - want).abs() <= tol + want.abs() * 2 * R.F32).all(), ((got - want).abs() - tol).max()
    for b in range(B):       # what no head sees is not touched
        m = n if lens is None else lens[b]
        unseen = torch.ones(n, dtype=torch.bool)
        unseen[:m] = ~R.visible_mask([m - 1], m, sink, window)[0] if m else unseen[:m]
        assert torch.equal(got[b][:, unseen], want[b][:, unseen])


# ------------------------------------------------------------------ eviction --

EVICT_CASES = [  # B, Hkv, n, keep, sink, recent
    (1, 1, 1, 1, 0, 0),
    (2, 2, 5, 1, 0, 0),
    (1, 2, 64, 64, 0, 0),
    (2, 3, 129, 128, 0, 0),
    (2, 2, 1000, 999, 4, 100),
    (2, 4, 777, 300, 4, 32),
    (1, 8, 5000, 2500, 0, 0),
    (3, 2, 4097, 65, 1, 64),
    (1, 2, 40000, 20001, 4, 1000),      # beyond the selection's one-launch rows
]


def evict_inputs(B, Hkv, n, rows, seed, ties=False):
    g = torch.Generator().manual_seed(seed)
    rr = 1 if rows == "token" else Hkv
    s = torch.exp(torch.randn((B, rr, n), generator=g))
    if ties:
        s = torch.randint(0, 3, s.shape, generator=g).float()
    si = H().new_importance(B, rr, n, DEV)
    si.copy_(s)
    pos = torch.randint(0, 1 << 30, (B, rr, (n + 3) // 4 * 4), generator=g, dtype=torch.int32).to(DEV)
    return s, si, pos[:, :, :n] if n % 2 else pos[:, :, :n].contiguous()


@pytest.mark.parametrize("rows", ["token", "kvhead"])
@pytest.mark.parametrize("case", EVICT_CASES)
@pytest.mark.parametrize("held", ["16-bit", "packed", "s"])
def test_evict(case, rows, held):
    B, Hkv, n, keep, sink, recent = case
    s, si, pos = evict_inputs(B, Hkv, n, rows, n + keep, ties=n == 777)
    want = R.kept(s, keep, sink, recent)
    pos0 = pos.cpu()
    g = torch.Generator(device=DEV).manual_seed(n)
    if held == "16-bit":
        k, v = (torch.randn((B, Hkv, n + 2, D), generator=g, device=DEV).half() for _ in range(2))
        bufs, args = [k, v], dict(k=k, v=v)
    elif held == "packed":
        bits = [torch.randint(0, 256, (B, Hkv, n + 1, m), generator=g, device=DEV, dtype=torch.uint8) for m in (64, 16, 64, 16)]
        cache = H().PackedCache(bits[0], bits[1].view(torch.float16).view(B, Hkv, n + 1, 4, 2), bits[2],
                                bits[3].view(torch.float16).view(B, Hkv, n + 1, 4, 2))
        bufs, args = bits, dict(cache=cache)
    else:
        bufs, args = [], dict(n_kv_heads=Hkv)
    before = [x.clone() for x in bufs]
    idx = H().hill_evict(si, keep, pos=pos, granularity=rows, n_sink=sink, n_recent=recent, **args)
    assert torch.equal(idx.cpu().long(), want)
    got = si.cpu()
    assert torch.equal(got[..., :keep], s.gather(-1, want)) and (got[..., keep:] == 0).all()
    assert torch.equal(pos.cpu()[..., :keep], pos0.gather(-1, want)) and torch.equal(pos.cpu()[..., keep:], pos0[..., keep:])
    for x, x0 in zip(bufs, before):
        j = want.to(DEV)[:, :, :, None].expand(B, Hkv, keep, x.shape[3])
        assert torch.equal(x[:, :, :keep], x0.gather(2, j))
        assert torch.equal(x[:, :, keep:], x0[:, :, keep:])


def test_evict_views_and_odd_rows():
    """A token-major cache whose rows are 264 elements apart: neighbours of the rows stay as they were."""
    B, Hkv, n, keep = 2, 3, 900, 411
    s, si, pos = evict_inputs(B, Hkv, n, "kvhead", 5)
    buf = torch.randn((B, n, Hkv, 264), device=DEV).bfloat16()
    before = buf.clone()
    k, v = buf[..., :D].transpose(1, 2), buf[..., D:2 * D].transpose(1, 2)
    idx = H().hill_evict(si, keep, k=k, v=v, granularity="kvhead").long()
    want = before.clone()
    for b in range(B):
        for h in range(Hkv):
            want[b, :keep, h, :2 * D] = before[b, idx[b, h], h, :2 * D]
    assert torch.equal(buf, want)


@pytest.mark.parametrize("held", ["16-bit", "packed"])
def test_evict_many_chunks_waits(held):
    """Long in-place moves over many workgroups: dense ends, so that late chunks read what early ones overwrite."""
    n, keep = 65536, 40000
    s = torch.rand((1, 1, n), generator=torch.Generator().manual_seed(1))
    s[..., :30000] -= 0.6              # the front loses most, the end keeps all
    s[..., -20000:] += 1.0
    want = R.kept(s, keep, 0, 0).to(DEV)
    for _ in range(3):
        si = H().new_importance(1, 1, n, DEV)
        si.copy_(s)
        if held == "16-bit":
            k, v = (torch.randint(-30000, 30000, (1, 4, n, D), device=DEV, dtype=torch.int16).view(torch.float16) for _ in range(2))
            bufs, args = [k.view(torch.int16), v.view(torch.int16)], dict(k=k, v=v)
        else:
            cache = H().new_packed_cache(1, 4, n, DEV)
            cache.k_codes.random_(0, 256)
            cache.v_codes.random_(0, 256)
            bufs, args = [cache.k_codes, cache.v_codes], dict(cache=cache)
        before = [x.clone() for x in bufs]
        H().hill_evict(si, keep, **args)
        for x, x0 in zip(bufs, before):
            assert torch.equal(x[:, :, :keep], x0[:, :, want[0, 0]]) and torch.equal(x[:, :, keep:], x0[:, :, keep:])


# every token kept, or all but the lowest; numbers, NaN (below every number) and -inf at the threshold; rows that end with
# a group of 64 tokens and within one; pins that leave the selection nothing to choose
@pytest.mark.parametrize("n,k,sink,recent", [(64, 64, 0, 0), (256, 256, 0, 0), (300, 300, 0, 0), (8192, 8191, 0, 0),
                                             (8193, 8193, 4, 64), (20032, 20032, 0, 0), (32768, 32768, 0, 0),
                                             (1000, 68, 4, 64), (1000, 1000, 500, 500), (32768, 1028, 4, 1024),
                                             (16384, 300, 0, 300), (1, 1, 0, 0), (4096, 4095, 0, 0),
                                             (4097, 2000, 0, 0), (24576, 24576, 0, 1), (24577, 12000, 3, 0)])
@pytest.mark.parametrize("low", ["nan", "-inf", "number"])
def test_selection_writes_its_own_rows(n, k, sink, recent, low):
    g = torch.Generator().manual_seed(n + k)
    s = torch.rand((2, 1, n), generator=g)
    s[:, :, torch.randperm(n, generator=g)[:n // 2]] = float(low) if low != "number" else -1.0
    si = H().new_importance(2, 1, n, DEV)
    si.copy_(s)
    guard = torch.full((64 + 2 * k + 40000,), -7, dtype=torch.int32, device=DEV)
    idx = H().hill_topk(si, k, n_sink=sink, n_recent=recent, idx_out=guard[64:64 + 2 * k].view(2, 1, k))
    assert torch.equal(idx.cpu().long(), R.kept(s, k, sink, recent))
    assert (guard[:64] == -7).all() and (guard[64 + 2 * k:] == -7).all()


# two shares, some, dozens, hundreds; in the last sequence most of them are empty
@pytest.mark.parametrize("n,B,Hq,Hkv", [(385, 2, 8, 2), (900, 2, 6, 3), (9001, 2, 4, 1), (70001, 2, 4, 1)])
@pytest.mark.parametrize("held", ["16-bit", "packed"])
def test_shares_of_one_token(n, B, Hq, Hkv, held):
    q, k, v = draw((B, Hq, D), torch.float16, n), draw((B, Hkv, n, D), torch.float16, n + 1), draw((B, Hkv, n, D), torch.float16, n + 2)
    lens = [n, 37]
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if held == "packed":
        cache = H().pack_kv(k.to(DEV), v.to(DEV), H().new_packed_cache(B, Hkv, n, DEV))
        k, v = (x.cpu() for x in H().unpack_kv(cache))
        out = H().hill_packed_attn(q.to(DEV), cache, lens=dl)
    else:
        out = H().hill_window_attn(q.to(DEV), k.to(DEV), v.to(DEV), window=n, lens=dl)
    check_decode(out, q, k, v, lens, 0, n)


@pytest.mark.parametrize("n,T,Hq,Hkv", [(700, 3, 8, 2), (1500, 33, 6, 3), (9001, 20, 4, 1), (40001, 2, 4, 1)])
def test_shares_of_a_chunk(n, T, Hq, Hkv):
    q, k, v = draw((2, Hq, T, D), torch.bfloat16, n), draw((2, Hkv, n, D), torch.bfloat16, n + 1), draw((2, Hkv, n, D), torch.bfloat16, n + 2)
    lens = [n, 45]
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = H().hill_window_prefill(q.to(DEV), k.to(DEV), v.to(DEV), window=n, n_sink=2, lens=dl)
    check_prefill(out, q, k, v, lens, 2, n)
