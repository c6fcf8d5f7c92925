"""Plain 64-bit forms of the cache operators, and the bounds that their fp32
kernels keep: every term counts roundings of half a step.

Attention.  A logit is an fp32 sum of 128 exact products: off by at most
128 * 2^-24 * scale * sum |q_d K_d|, plus one rounding of the scaled value and of the
exponential's argument (|x| * 2^-23, |x| <= scale * sum |q_d K_d| * log2 e).  A
weight is then off by that and the exponential's ulp, relatively (e_w); out
= sum w V / sum w by at most 2 e_w sum w |V|, plus the fp32 sums' roundings."""
import math

import torch

D = 128
F32 = 2.0 ** -24


def visible_mask(p, m, sink, window):
    """[T, m]: which of m tokens queries at positions p see."""
    p = torch.as_tensor(p).reshape(-1, 1)
    j = torch.arange(m).reshape(1, -1)
    return (j <= p) & ((j < sink) | (p - j < window))


def attend(q, k, v, mask, scale=None):
    """q [G, T, D], k, v [m, D], mask [T, m] -> out, bound of the fp32 form's error, sum w |V|, weights."""
    scale = D ** -0.5 if scale is None else scale
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    x = torch.einsum("gtd,md->gtm", q, k) * scale
    x = x.masked_fill(~mask, -math.inf)
    top = x.amax(-1, keepdim=True) if x.shape[-1] else torch.zeros(x.shape[:-1] + (1,))
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    w = torch.where(total > 0, e / total.clamp_min(1e-300), torch.zeros_like(e))
    out, spread = torch.einsum("gtm,md->gtd", w, v), torch.einsum("gtm,md->gtd", w, v.abs())
    size = (torch.einsum("gtd,md->gtm", q.abs(), k.abs()) * abs(scale)).masked_fill(~mask, 0.0)
    size = size.amax(-1, keepdim=True) if x.shape[-1] else torch.zeros(x.shape[:-1] + (1,))
    e_w = size * (D * F32 + 4 * F32 * 1.4427) + 8 * F32
    sums = (mask.sum(-1).double() / 32 + 64).reshape(1, -1, 1) * F32     # 32 products to an fp32 addition, then the merges
    return out, (2 * e_w + 2 * sums) * spread + 1e-30, spread, w, e_w


def quantise(x):
    """Codes [..., 128], (scale, zero) [..., 4] and fp16 values of the 4-bit format, by its definition: fp32 steps are
    fp32 operations, the value is rounded once from 64 bits."""
    g = x.detach().cpu().float().clamp(-65504.0, 65504.0).unflatten(-1, (4, 32))
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    scale, zero = ((hi - lo) * torch.tensor(1.0 / 15.0)).half(), lo.half()
    inv = torch.where(scale > 0, 1.0 / scale.float(), torch.zeros_like(lo))
    code = torch.round((g - zero.float()) * inv).clamp(0, 15)
    exact = code.double() * scale.double() + zero.double()
    value = torch.from_numpy(exact.numpy().astype("float16"))
    return code.flatten(-2).to(torch.uint8), scale.squeeze(-1), zero.squeeze(-1), value.flatten(-2)


def codes_of(by):
    """[..., 64] bytes -> [..., 128] codes (element 2i of a 4-byte word in bits 4i.., element 2i+1 in bits 16+4i..)."""
    by = by.cpu().to(torch.int64).unflatten(-1, (16, 4))
    word = by[..., 0] | by[..., 1] << 8 | by[..., 2] << 16 | by[..., 3] << 24
    at = [4 * (e // 2) + 16 * (e % 2) for e in range(8)]
    return torch.stack([(word >> s) & 15 for s in at], -1).flatten(-2).to(torch.uint8)


def kept(s, k_keep, sink, recent):
    """Former indices of what an eviction keeps, ascending."""
    x = s.detach().cpu().double().clone()
    n = x.shape[-1]
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    x[..., :sink] = math.inf
    if recent:
        x[..., max(0, n - recent):] = math.inf
    return torch.sort(torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :k_keep], -1).values
