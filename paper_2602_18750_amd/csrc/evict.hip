// Eviction's second half: the kept rows of K, V (16-bit or packed), S and the
// positions move to the front of their buffers, in place and in order.
//
// Row i of the result is row idx[i] of the cache, and idx[i] >= i.  A workgroup
// takes kEvictChunk result rows of one (sequence, KV head): it reads their
// sources into registers, says so in a flag, waits until every chunk whose
// sources lie in its own destination rows has said so, and writes.  Those are
// chunks before it (a source never lies before its destination), and a group's chunks are
// handed out by its counter in ascending order, so every chunk waited for is held by a
// workgroup that runs or has ended and sets its flag without waiting: each
// wait ends.  Each kept row is read once and written once, past the caches; the
// bound is a copy's: 16384 of 32768 rows of 8 KV heads, 134 MB, in 31 us (4.3 TB/s; a
// 2 GiB copy reaches 5.0), 131072 of 4 x 65536 tokens, 1.07 GB, in 206 us (5.2 TB/s).
#include "hill_device.h"
#include "hill_internal.h"

namespace hill {

namespace {

constexpr int kLoads = kEvictChunk / 16;   // 16-bit rows per lane group (16 lanes a row)

// A wait lasts a few microseconds; the limit (tens of milliseconds) ends it where
// two calls share one workspace at a time, against the contract.  The workgroup then
// leaves its rows as they are and says so in the status word.
constexpr int kMaxSpins = 1 << 16;

// Stores wait for the flag seen before them, loads for the flag set after them.
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <bool ROWS, bool PACKED>
__global__ __launch_bounds__(256) void evict_kernel(EvictArgs a)
{
    __shared__ int32_t src[kEvictChunk];
    __shared__ int ticket, late;
    const int tid = threadIdx.x;
    const int groups = a.B * a.heads;
    const int bg = blockIdx.x % groups;
    uint32_t* flags = a.flags + (int64_t)bg * a.flag_words;
    if (tid == 0) {
        ticket = (int)atomicAdd(flags, 1u);
        late = 0;
    }
    ++flags;
    __syncthreads();
    const int c = ticket;
    if ((unsigned)c >= (unsigned)a.chunks) {                 // only where two calls share a workspace
        if (tid == 0) atomicAdd(a.status, 1u);
        return;
    }
    const int b = bg / a.heads, g = bg % a.heads;
    const int r = a.R > 1 ? g : 0;
    const int32_t* idx = a.idx + ((int64_t)b * a.R + r) * a.keep;
    const int d0 = c * kEvictChunk, cnt = min(kEvictChunk, a.keep - d0);
    if (tid < kEvictChunk) src[tid] = min(max(idx[d0 + min(tid, cnt - 1)], 0), a.n - 1);
    __syncthreads();
    const bool own_s = a.R > 1 || g == 0;                    // this group moves the row's S and positions
    const bool moves = src[cnt - 1] != d0 + cnt - 1;         // ascending: else no row of the chunk moves
    float* srow = a.s + (int64_t)b * a.s_sb + (int64_t)r * a.s_sr;
    int32_t* prow = a.pos ? a.pos + (int64_t)b * a.p_sb + (int64_t)r * a.p_sr : nullptr;

    float sv = 0.0f;
    int32_t pv = 0;
    u32x4_t kr[kLoads], vr[kLoads], cr[2];
    uint32_t pr[2];
    const int l16 = tid & 15, rg = tid >> 4;
    const int64_t packed0 = ((int64_t)b * a.Hkv + g) * a.cap;
    if (moves) {
        if constexpr (ROWS) {
            const uint16_t* k = a.k + (int64_t)b * a.k_sb + (int64_t)g * a.k_sh + l16 * 8;
            const uint16_t* v = a.v + (int64_t)b * a.v_sb + (int64_t)g * a.v_sh + l16 * 8;
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const int j = src[min(16 * u + rg, cnt - 1)];
                kr[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(k + (int64_t)j * a.k_sn));
                vr[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(v + (int64_t)j * a.v_sn));
            }
        }
        if constexpr (PACKED) {                              // a row's codes by four lanes, its parameters by four
            const int64_t row = packed0 + src[min(tid >> 2, cnt - 1)];
            cr[0] = *reinterpret_cast<const u32x4_t*>(a.kc + row * 64 + (tid & 3) * 16);
            cr[1] = *reinterpret_cast<const u32x4_t*>(a.vc + row * 64 + (tid & 3) * 16);
            pr[0] = a.kp[row * 4 + (tid & 3)];
            pr[1] = a.vp[row * 4 + (tid & 3)];
        }
        if (own_s && tid < cnt) {
            sv = srow[src[tid]];
            if (prow) pv = prow[src[tid]];
        }
    }
    loads_done();
    __syncthreads();
    if (tid == 0) __hip_atomic_store(flags + c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // S past the kept tokens is zero: the tokens from this chunk's first source to the next chunk's are read by
    // no other chunk
    if (own_s) {
        const int from = max(c == 0 ? 0 : src[0], a.keep), to = d0 + cnt < a.keep ? idx[d0 + cnt] : a.n;
        for (int j = from + tid; j < to; j += 256) srow[j] = 0.0f;
    }
    if (!moves) return;
    // chunks with a source among rows [d0, d0 + cnt): each thread looks among a 256th of those before this one (the
    // sources ascend), in one that has any for its first
    const int per = (c + 255) / 256, e1 = min(per * (tid + 1), c);
    int e = per * tid;
    if (e < e1 && idx[e1 * kEvictChunk - 1] >= d0 && idx[e * kEvictChunk] < d0 + cnt) {
        for (int hi = e1 - 1; e < hi;) {
            const int mid = (e + hi) / 2;
            if (idx[mid * kEvictChunk + kEvictChunk - 1] >= d0) hi = mid;
            else e = mid + 1;
        }
        for (int spins = kMaxSpins; e < e1 && idx[e * kEvictChunk] < d0 + cnt; ++e) {
            while (__hip_atomic_load(flags + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0u && --spins > 0)
                __builtin_amdgcn_s_sleep(1);
            if (spins <= 0) {
                late = 1;
                break;
            }
        }
    }
    asm volatile("" ::: "memory");
    __syncthreads();
    if (late) {
        if (tid == 0) atomicAdd(a.status, 1u);
        return;
    }
    if constexpr (ROWS) {
        uint16_t* k = a.k + (int64_t)b * a.k_sb + (int64_t)g * a.k_sh + l16 * 8;
        uint16_t* v = a.v + (int64_t)b * a.v_sb + (int64_t)g * a.v_sh + l16 * 8;
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int i = 16 * u + rg;
            if (i < cnt && src[i] != d0 + i) {
                __builtin_nontemporal_store(kr[u], reinterpret_cast<u32x4_t*>(k + (int64_t)(d0 + i) * a.k_sn));
                __builtin_nontemporal_store(vr[u], reinterpret_cast<u32x4_t*>(v + (int64_t)(d0 + i) * a.v_sn));
            }
        }
    }
    if constexpr (PACKED) {
        const int i = tid >> 2;
        if (i < cnt && src[i] != d0 + i) {
            const int64_t row = packed0 + d0 + i;
            *reinterpret_cast<u32x4_t*>(a.kc + row * 64 + (tid & 3) * 16) = cr[0];
            *reinterpret_cast<u32x4_t*>(a.vc + row * 64 + (tid & 3) * 16) = cr[1];
            a.kp[row * 4 + (tid & 3)] = pr[0];
            a.vp[row * 4 + (tid & 3)] = pr[1];
        }
    }
    if (own_s && tid < cnt) {
        srow[d0 + tid] = sv;
        if (prow) prow[d0 + tid] = pv;
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t st)
{
    const int64_t groups = (int64_t)a.B * a.heads * a.chunks;
    const dim3 grid((unsigned)groups);
    if (a.k) hipLaunchKernelGGL((evict_kernel<true, false>), grid, dim3(256), 0, st, a);
    else if (a.kc) hipLaunchKernelGGL((evict_kernel<false, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((evict_kernel<false, false>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace hill
