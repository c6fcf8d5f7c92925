"""Window prefill at its edges: rows that nothing sees, and fp16 weights over
many binary orders."""
import sys

import pytest
import torch

import cache_ref as R
from test_gpu_cache_ops import D, DEV, H, check_prefill, draw

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, file=sys.stderr, flush=True)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,Hq,Hkv,n,T,sink,lens", [
    (1, 4, 4, 300, 150, 0, None),             # nothing visible
    (2, 4, 2, 300, 290, 33, (300, 200)),      # sinks alone, some of them inside the chunk, and a padded sequence
    (1, 8, 2, 400, 3, 70, None),
    (40, 14, 7, 200, 130, 20, None),          # blocks of 256 rows
    (1, 4, 2, 1500, 20, 1400, None),          # several shares of the sinks
])
def test_window_zero_does_not_read_unseen_rows(B, Hq, Hkv, n, T, sink, lens, dtype):
    """Without a window only the sinks are visible: the others hold NaN and infinities."""
    q, k, v = draw((B, Hq, T, D), dtype, n), draw((B, Hkv, n, D), dtype, n + 1), draw((B, Hkv, n, D), dtype, n + 2)
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[:, :, sink:], bad_v[:, :, sink::2], bad_v[:, :, sink + 1::2] = float("nan"), float("nan"), float("inf")
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = H().hill_window_prefill(q.to(DEV), bad_k.to(DEV), bad_v.to(DEV), window=0, n_sink=sink, lens=dl)
    check_prefill(out, q, k, v, lens or [n] * B, sink, 0)


# An fp16 weight is held with 11 bits down to 2^-25 of the reference that a row's exponentials have, and as a multiple of
# 2^-35 below: off by 2^-36 of the reference, which is at most the row's largest weight.
HELD = 2.0 ** -36


def check_small_weights(got, q, k, v, n, sink, window, scale):
    """got [B, Hq, T, D], the last T of n tokens, within the bounds of check_prefill but for HELD per visible token."""
    B, Hq, T, _ = q.shape
    G, u, got = Hq // k.shape[1], 2.0 ** -11, got.cpu().double()
    mask = R.visible_mask(torch.arange(n - T, n), n, sink, window)
    for b in range(B):
        for g in range(k.shape[1]):
            hs = slice(g * G, (g + 1) * G)
            out, bound, spread, _, _ = R.attend(q[b, hs], k[b, g], v[b, g], mask, scale)
            tol = bound + u * spread + u * out.abs() * (1 + u) + 2.0 ** -25
            tol = tol + mask.sum(-1).reshape(1, -1, 1) * HELD * v[b, g].double().abs().max()
            err = (got[b, hs] - out).abs()
            assert (err <= tol).all(), (b, g, (err - tol).max(), err.max())


@pytest.mark.parametrize("nats", [9.0, 13.0, 17.6])
@pytest.mark.parametrize("B,Hq,Hkv,n,T", [(8, 32, 8, 700, 300),      # one share, 256-row blocks
                                          (1, 4, 2, 400, 150),       # one share of 128
                                          (1, 4, 2, 4096, 3), (1, 8, 2, 9000, 20)])   # several
def test_a_sink_that_takes_nearly_all_weight(B, Hq, Hkv, n, T, nats):
    """The first token's logit lies ``nats`` above the others', and its V is zero: the others' small weights make
    the output."""
    q, k, v = draw((B, Hq, T, D), torch.float16, n, 0.2), draw((B, Hkv, n, D), torch.float16, n + 1, 0.2), draw((B, Hkv, n, D), torch.float16, n + 2)
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    k[:, :, 0] = 0.0
    k[:, :, 0, 0] = nats * D ** 0.5 / 8.0
    v = v * 0.25 + 1.0
    v[:, :, 0] = 0.0
    out = H().hill_window_prefill(q.to(DEV), k.to(DEV), v.to(DEV), window=n - 1, n_sink=1)
    check_small_weights(out, q, k, v, n, 1, n - 1, None)


@pytest.mark.parametrize("scale", [0.9, -0.6])
@pytest.mark.parametrize("B,Hq,Hkv,n,T", [(1, 4, 2, 500, 200), (1, 4, 2, 2000, 9)])
def test_fp16_logits_in_the_tens(B, Hq, Hkv, n, T, scale):
    q, k, v = draw((B, Hq, T, D), torch.float16, n), draw((B, Hkv, n, D), torch.float16, n + 1), draw((B, Hkv, n, D), torch.float16, n + 2)
    out = H().hill_window_prefill(q.to(DEV), k.to(DEV), v.to(DEV), window=n, sm_scale=scale)
    check_small_weights(out, q, k, v, n, 0, n, scale)


@pytest.mark.parametrize("B,Hq,Hkv,n,T", [(1, 4, 2, 700, 150), (1, 4, 2, 3000, 5)])
def test_maxima_that_grow_from_tile_to_tile(B, Hq, Hkv, n, T):
    """Logits that rise along the sequence by steps below and above what the running reference lets pass, and fall
    again: weights of the largest size that is held, and rescaled sums."""
    q, k, v = draw((B, Hq, T, D), torch.float16, n, 0.1), draw((B, Hkv, n, D), torch.float16, n + 1, 0.1), draw((B, Hkv, n, D), torch.float16, n + 2)
    q[..., 1] = 4.0
    j = torch.arange(n)
    for g in range(Hkv):     # in units of ln 2: slow and fast growth, then down
        x = 3.9 * (j // 64) + 4.0 * torch.rand(n, generator=torch.Generator().manual_seed(g)) * (g == 0)
        x = torch.where(j < n * 3 // 4, x, 3.9 * ((n - j) // 64)) if g else x.clamp_max(60.0)
        k[:, g, :, 1] = (x.clamp_max(70.0) * 0.6931 * D ** 0.5 / 4.0).half()
    out = H().hill_window_prefill(q.to(DEV), k.to(DEV), v.to(DEV), window=n)
    check_small_weights(out, q, k, v, n, 0, n, None)
