// The move of hill_evict without its selection, built as a small library of its
// own (libhill_move.so) for the tests; not part of libhill or its ABI.  A test
// hands it flags in a state that no call leaves behind.
#include <hip/hip_runtime.h>

#include "hill_internal.h"

// One sequence, one importance row, contiguous k and v [heads, n, 128], s and
// pos [n]; idx [keep] ascending.  flags: heads * hill_move_flag_words(keep)
// words, per KV head its ticket counter, then its chunks' flags.  Returns 0, 1
// for an invalid argument (nothing launched), or 2 if the launch failed.
extern "C" __attribute__((visibility("default"))) int64_t hill_move_flag_words(int32_t keep)
{
    return keep < 1 ? 0 : hill::evict_flag_words((keep + hill::kEvictChunk - 1) / hill::kEvictChunk);
}

extern "C" __attribute__((visibility("default"))) int hill_move(const int32_t* idx, int32_t heads, int32_t n, int32_t keep,
                                                                float* s, int32_t* pos, void* k, void* v, uint32_t* flags,
                                                                uint32_t* status, void* stream)
{
    if (!idx || !s || !pos || !k || !v || !flags || !status || heads < 1 || heads > 256 || keep < 1 || keep > n) return 1;
    hill::EvictArgs a{};
    a.idx = idx;
    a.B = a.R = 1;
    a.Hkv = a.heads = heads;
    a.n = n;
    a.keep = keep;
    a.s = s;
    a.pos = pos;
    a.s_sb = a.s_sr = a.p_sb = a.p_sr = n;
    a.k = static_cast<uint16_t*>(k);
    a.v = static_cast<uint16_t*>(v);
    a.k_sb = a.v_sb = (int64_t)heads * n * hill::kHeadDim;
    a.k_sh = a.v_sh = (int64_t)n * hill::kHeadDim;
    a.k_sn = a.v_sn = hill::kHeadDim;
    a.flags = flags;
    a.flag_words = hill_move_flag_words(keep);
    a.status = status;
    a.chunks = (keep + hill::kEvictChunk - 1) / hill::kEvictChunk;
    return hill::launch_evict(a, static_cast<hipStream_t>(stream)) == hipSuccess ? 0 : 2;
}
