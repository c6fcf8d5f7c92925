"""The 4-bit cache where fp16 ends: groups that reach its largest value come
back finite."""
import sys

import pytest
import torch

import cache_ref as R
from test_gpu_cache_ops import D, DEV, H, check_decode, draw

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, file=sys.stderr, flush=True)


def quantise(x):
    """As R.quantise, with the smaller scale that a group takes whose largest code would be infinite; and which did."""
    code, scale, zero, value = R.quantise(x)
    top = torch.from_numpy((15.0 * scale.double() + zero.double()).numpy().astype("float16"))
    over = torch.isinf(top)
    scale = torch.where(over, (scale.view(torch.int16) - 1).view(torch.float16), scale)
    g = x.detach().cpu().float().clamp(-65504.0, 65504.0).unflatten(-1, (4, 32))
    lower = torch.round((g - zero.float()[..., None]) * (1.0 / scale.float())[..., None]).clamp(0, 15)
    code = torch.where(over[..., None], lower.to(torch.uint8), code.unflatten(-1, (4, 32)))
    exact = code.double() * scale.double()[..., None] + zero.double()[..., None]
    return code.flatten(-2), scale, zero, torch.from_numpy(exact.numpy().astype("float16")).flatten(-2), over


def far_rows(n, dtype, seed):
    """Groups with a largest element of 65504 or near it, and a smallest anywhere; bf16 elements beyond fp16 too."""
    x = draw((1, 2, n, D), torch.float32, seed, 100.0).unflatten(-1, (4, 32))
    g = torch.Generator().manual_seed(seed)
    edge = lambda: 65504.0 - 32.0 * torch.randint(0, 8, x.shape[:-1], generator=g).float() * (torch.rand(x.shape[:-1], generator=g) < 0.5)
    x[..., 3], x[..., 7] = edge(), edge() * (torch.rand(x.shape[:-1], generator=g) * 2 - 1)
    x[:, :, 0] = 1.0
    x[:, :, 0, :, 3] = 65504.0
    x[:, :, 0, 0, 7], x[:, :, 0, 1, 7], x[:, :, 0, 2, 7] = 0.0, -65504.0, 65472.0
    x = x.flatten(-2)
    if dtype == torch.bfloat16:
        x[:, :, 1::3] *= 1e6
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_rows_at_the_end_of_fp16_come_back_finite(dtype):
    n = 400
    k, v = far_rows(n, dtype, 1), far_rows(n, dtype, 2)
    cache = H().pack_kv(k.to(DEV), v.to(DEV), H().new_packed_cache(1, 2, n, DEV))
    for x, codes, params, back in zip((k, v), (cache.k_codes, cache.v_codes), (cache.k_params, cache.v_params), H().unpack_kv(cache)):
        code, scale, zero, value, over = quantise(x)
        assert 0.02 < over.float().mean() < 0.9 and torch.isfinite(value).all()
        assert torch.equal(params[..., 0].cpu(), scale) and torch.equal(params[..., 1].cpu(), zero)
        assert torch.equal(R.codes_of(codes), code) and torch.equal(back.cpu(), value)
        # no element is further off than a step: the scale is at most one fp16 step below (max - min) / 15
        far = (back.cpu().float() - x.float().clamp(-65504.0, 65504.0)).abs().unflatten(-1, (4, 32))
        assert (far <= scale.float()[..., None]).all()


def test_attention_over_such_rows():
    n = 300
    k, v = draw((1, 2, n, D), torch.float16, 1), far_rows(n, torch.float16, 5)
    q = draw((1, 4, D), torch.float16, 3)
    cache = H().pack_kv(k.to(DEV), v.to(DEV), H().new_packed_cache(1, 2, n, DEV))
    out = H().hill_packed_attn(q.to(DEV), cache)
    check_decode(out, q, R.quantise(k)[3], quantise(v)[3], [n], 0, n)
