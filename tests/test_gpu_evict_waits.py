"""What an eviction's move does when a wait finds no end: it leaves rows as they
are and says so, and otherwise its status is 0."""
import ctypes
import sys

import pytest
import torch

from test_gpu_cache_ops import D, DEV, H

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, file=sys.stderr, flush=True)


def test_a_wait_without_end_leaves_the_rows():
    """Every second of 512 tokens kept, in four chunks of 64 for each of two KV heads.  The first head's first chunk is
    marked as taken, and nobody will say that its rows have been read: its second chunk, over whose rows they lie, gives
    up (after tens of milliseconds) and moves nothing; what does not depend on it moves."""
    from paper_2602_18750_amd import _build
    lib = ctypes.CDLL(_build.MOVE_LIB)
    P, I = ctypes.c_void_p, ctypes.c_int32
    lib.hill_move.argtypes = [P, I, I, I, P, P, P, P, P, P, P]
    lib.hill_move_flag_words.argtypes, lib.hill_move_flag_words.restype = [I], ctypes.c_int64
    heads, n, keep = 2, 512, 256
    idx = torch.arange(0, n, 2, dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    k0, v0 = (torch.randn((heads, n, D), generator=g, device=DEV).half() for _ in range(2))
    s0, pos0 = torch.rand(n, generator=g, device=DEV) + 1.0, torch.arange(n, dtype=torch.int32, device=DEV) + 7
    words = lib.hill_move_flag_words(keep)
    assert words >= 1 + keep // 64
    for taken in (0, 1):
        k, v, s, pos = k0.clone(), v0.clone(), s0.clone(), pos0.clone()
        flags = torch.zeros((heads, words), dtype=torch.int32, device=DEV)
        flags[0, 0] = taken
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        assert lib.hill_move(*(x.data_ptr() if isinstance(x, torch.Tensor) else x
                               for x in (idx, heads, n, keep, s, pos, k, v, flags, status)),
                             torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert int(status) == 2 * taken        # the chunk that gave up, and a workgroup that found no chunk left
        for x, x0 in ((k, k0), (v, v0)):
            want = x0.clone()
            want[:, :keep] = x0[:, idx.long()]
            if taken:
                want[0, :128] = x0[0, :128]
            assert torch.equal(x, want)
        for x, x0 in ((s, s0), (pos, pos0)):   # moved beside the first head
            want = x0.clone()
            want[:keep] = x0[idx.long()]
            if taken:
                want[:128] = x0[:128]
            if x is s:
                want[keep:] = 0
            assert torch.equal(x, want)


@pytest.mark.parametrize("n,keep,rows", [(700, 300, "token"), (4097, 4096, "kvhead"), (50000, 20000, "token")])
def test_the_status_word_of_a_call(n, keep, rows):
    from paper_2602_18750_amd import cache as C
    rr = 1 if rows == "token" else 2
    s = H().new_importance(1, rr, n, DEV)
    s.copy_(torch.rand((1, rr, n), generator=torch.Generator().manual_seed(n)))
    k, v = (torch.randn((1, 2, n, D), device=DEV).half() for _ in range(2))
    d = C._desc(1, 2, 2, D, n, torch.float16, s_st=s.stride()[:2], granularity=rows)
    need = ctypes.c_size_t()
    assert H().load_library().hill_evict_workspace_bytes(ctypes.byref(d), keep, ctypes.byref(need)) == 0
    ws = torch.full((need.value + 512,), 0xff, dtype=torch.uint8, device=DEV)
    H().hill_evict(s, keep, k=k, v=v, granularity=rows, ws=ws)
    status = ws[need.value - 256:need.value].view(torch.int32)
    assert int(status[0]) == 0 and (ws[need.value:] == 0xff).all()
