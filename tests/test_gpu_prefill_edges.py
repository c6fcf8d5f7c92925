"""Window prefill at its edges: rows that nothing sees."""
import sys

import pytest
import torch

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
