"""Finite rows whose logits lie below fp32's range weigh nothing, wherever in the
cache they are, and leave the others their weights."""
import sys

import pytest
import torch

import cache_ref as R
from test_gpu_cache_ops import D, DEV, H, draw

pytestmark = pytest.mark.gpu
N = 700
# which of 700 tokens lie far below: whole tiles of a wave, its first one, one wave's all, the last tokens, all but one
FAR = {"first tiles": lambda j: j < 200, "a wave's first": lambda j: j < 32, "every second tile": lambda j: j // 32 % 2 == 0,
       "the end": lambda j: j >= 400, "scattered": lambda j: j % 3 == 1, "all but one": lambda j: j != 555}


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, file=sys.stderr, flush=True)


def rows(far, q_far, k_far, dtype):
    """q, k, v and the far tokens: heads alternate between those that see them at -infinity in fp32 and those that see
    them as any other (their q is 0 where the far keys reach)."""
    q, k, v = draw((1, 8, D), dtype, 1), draw((1, 2, N, D), dtype, 2), draw((1, 2, N, D), dtype, 3)
    mask = FAR[far](torch.arange(N))
    q[..., 0], k[..., 0] = 0.0, 0.0
    q[:, ::2, 0] = q_far
    k[:, :, mask, 0] = k_far
    return q, k, v, mask


def want_of(q, k, v, mask, h, window=N):
    """Head h's tokens (the odd heads': all that are visible; else the near ones), output, bound and weights."""
    near = torch.nonzero((torch.arange(N) >= N - window) & ~(mask & (h % 2 == 0))).flatten()
    kk = k[0, h // 4, near].clone()
    kk[:, 0] = 0.0          # met by a query's 0, or one of the near tokens' zeros
    out, bound, _, w, e_w = R.attend(q[0, h:h + 1, None], kk, v[0, h // 4, near], torch.ones(1, len(near), dtype=torch.bool))
    return near, out[0, 0], bound[0, 0], w[0, 0], e_w[0, 0]


@pytest.mark.parametrize("far,window", [(f, N) for f in FAR] + [(f, 90) for f in FAR if not FAR[f](torch.arange(N - 90, N)).all()])
def test_16_bit_rows(far, window):
    q, k, v, mask = rows(far, 1e20, -1e20, torch.bfloat16)
    got = H().hill_window_attn(q.to(DEV), k.to(DEV), v.to(DEV), window=window).cpu().double()
    chunk = H().hill_window_prefill(q[:, :, None].to(DEV), k.to(DEV), v.to(DEV), window=window)[:, :, 0].cpu().double()
    for h in range(8):
        _, out, bound, w, _ = want_of(q, k, v, mask, h, window)
        assert ((got[0, h] - out).abs() <= bound).all(), (h, got[0, h, :4], out[:4])
        # the prefill's weights and outputs are bf16: half a step of sum w |V| <= max |V|, and of the output
        assert ((chunk[0, h] - out).abs() <= bound + 2.0 ** -8 * (v.double().abs().max() + 1.01 * out.abs())).all()


@pytest.mark.parametrize("far", FAR)
def test_packed_rows_and_their_importance(far):
    """A bf16 query of 1e38 over fp16 values of -30000: the logit, -2.7e41, is below fp32's range."""
    q, k, v, mask = rows(far, 1e38, -30000.0, torch.bfloat16)
    k, v = k.half(), v.half()
    k[..., 1:32] = 0.0       # the far group holds 0 and -30000, exactly
    cache = H().pack_kv(k.to(DEV), v.to(DEV), H().new_packed_cache(1, 2, N, DEV))
    held_k, held_v = R.quantise(k)[3], R.quantise(v)[3]
    qq = q.clone()
    qq[:, ::2, 1:] = 0.0     # beside 1e38 the others lose their bits in fp16: they are 0
    s = H().new_importance(1, 1, N, DEV)
    got = H().hill_packed_attn(qq.to(DEV), cache, s=s).cpu().double()
    want_s, tol_s = torch.zeros(N, dtype=torch.float64), torch.zeros(N, dtype=torch.float64)
    for h in range(8):
        near, out, bound, w, e_w = want_of(qq, held_k, held_v, mask, h)
        assert ((got[0, h] - out).abs() <= bound).all(), (h, got[0, h, :4], out[:4])
        want_s[near] += w
        tol_s[near] += w * (2 * e_w + (N / 32 + 72) * 2 * R.F32)
    assert ((s.cpu().double()[0, 0] - want_s).abs() <= tol_s + want_s * 2 * R.F32 + 1e-30).all()


def test_nothing_but_far_tokens():
    """Then no weight is known, and S stays a number."""
    q, k, v, _ = rows("first tiles", 1e38, -30000.0, torch.bfloat16)
    k, v = k.half(), v.half()
    k[..., 1:32], k[..., 0] = 0.0, -30000.0
    cache = H().pack_kv(k.to(DEV), v.to(DEV), H().new_packed_cache(1, 2, N, DEV))
    s = H().new_importance(1, 1, N, DEV)
    q[..., 0], q[..., 1:] = 1e38, 0.0
    out = H().hill_packed_attn(q.to(DEV), cache, s=s)
    assert (out == 0).all() and (s == 0).all()
