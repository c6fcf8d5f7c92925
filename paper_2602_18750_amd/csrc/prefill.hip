// Attention of a chunk's tokens over the first tokens and a sliding window.
//
// The rows of a (sequence, KV head) are its T tokens times its G query heads,
// token by token: a workgroup takes 256 of them, or 128 (eight or four waves of
// 32), so that a group's heads share the keys and values they read and the
// rows of a workgroup lie at few positions, whatever G.  It walks the first
// tokens and then the window [first position - window + 1, last position] in
// tiles of 64, double-buffered in LDS by direct loads, with running maxima and
// sums:
//
//   x^T = K Q^T on the matrix cores (tokens x rows): a lane holds one row's
//   logits, the maximum needs one exchange between lane halves, and the weights
//   are, rounded to 16 bits, the second product's operand as they lie;
//   O^T += V^T w^T with V read from LDS transposed.
//
// Each tile's K Q^T products are formed among the exponentials of the tile
// before it, whose weights then meet V: a wave's matrix and vector instructions
// run side by side (at the size below 979 -> 950 us).  Weights are rounded to
// the cache's type (the output is rounded to it anyway); maxima, sums and O are
// fp32.  The reference of the exponentials follows the running maximum only
// when that has grown by more than 2^8 (fp16: 2^4): weights stay below that, and
// O is rescaled rarely.
//
// Measured: 16K tokens, 32 / 8 heads, window 4096, 0.96 TFLOP: 885 to 950 us
// from card to card, 1.01 to 1.09 PFLOP/s (large library products of the type reach 1.42 to 1.63).  The
// matrix cores, LDS (each wave reads the whole tile for its 32 rows) and the
// vector units (an exponential and about six more instructions per weight)
// each need about half of that, two waves per SIMD overlap them in part (the
// matrix cores are busy 0.94 of 1.77 million cycles), and the clock falls to
// 1.5 to 1.9 GHz of 2.4 under the load: with K's reads from LDS left out 800 us,
// V's 905, the exponentials 872, all three 684.  Sixty-four rows a wave halve
// the reads, but do not fit the registers (1319 us with what that spills and
// moves); the workgroup's halves in turn on the matrix cores and the vector
// units, two barriers a tile, took the same cycles and time.
#include "mfma_device.h"

namespace hill {

namespace {

constexpr int kKeys = 64;                       // tokens per tile
// A tile in LDS: blocks of four rows, which one direct load of a wave fills, each
// 16 bytes further than its 1 KiB; row r of a block keeps its 16-byte piece c at c ^
// 4r.  The rows of one access then lie in different banks (sixteen rows in a column of K;
// four rows by 64 bytes of V), and all of a lane's addresses are one of four and a constant.
constexpr int kBlockBytes = 4 * kHeadDim * 2 + 16;
constexpr int kTileBytes = kKeys / 4 * kBlockBytes;
// How far (in the exponent of 2) a row's maximum may outgrow its reference before that follows, and the factor 2^shift
// that the weights carry, in O and in their sum, until the division: bf16 reaches as far down as fp32, fp16 weights stay
// below 2^15 and are whole (11 bits) down to 2^-25 of the reference, and multiples of 2^-35 below: behind a sink that takes
// nearly all weight the others make the output.  (Slack and shift 8 and 0, 8 and 7, these, in us: 16K x 16K tokens, window
// 4096, 968, 965, 978; 4 x 509 after 20K 72.8, 71.7, 73.8.)
template <int DT>
constexpr float kSlack = DT == 1 ? 8.0f : 4.0f;
template <int DT>
constexpr float kShift = DT == 1 ? 0.0f : 11.0f;

__device__ __forceinline__ float max_x32(float v)
{
    auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

template <int DT>
__device__ __forceinline__ uint32_t round_pair(float x, float y)
{
    if constexpr (DT == 1) return __builtin_bit_cast(uint32_t, bf162_t{(__bf16)x, (__bf16)y});
    else return __builtin_bit_cast(uint32_t, half2_t{(_Float16)x, (_Float16)y});
}

// 16 bytes per lane from global memory into LDS, lane after lane from `to` on.
__device__ __forceinline__ void load_lds16(const uint16_t* from, char* to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

template <int DT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void prefill_kernel(PrefillArgs a)
{
    constexpr int kRows = 32 * NW;
    // four arrays of their own, each step's named at compile time: the compiler then knows that the direct loads into one
    // pair do not write what is read from the other, and does not wait for them before the first read
    __shared__ __attribute__((aligned(16))) char k0[kTileBytes], v0[kTileBytes], k1[kTileBytes], v1[kTileBytes];
    const int tid = threadIdx.x, lane = tid & 63, c32 = lane & 31, hf = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (sequence, KV head) fastest, so that its blocks meet its K and V in one L2; the last tokens, whose windows
    // are full, first
    const int split = blockIdx.x % a.nsplit, unit = blockIdx.x / a.nsplit;
    const int bh = unit % (a.B * a.Hkv), blk = a.blocks - 1 - unit / (a.B * a.Hkv);
    const int b = bh / a.Hkv, g = bh % a.Hkv;
    const int len = seq_len(a.lens, b, a.n);
    const int first = len - a.t;                            // position of the chunk's first token (may be < 0)
    const int rows = a.t * a.G;
    const int r0 = blk * kRows;
    const int row = min(r0 + 32 * w + c32, rows - 1);       // this lane's row
    const int tq = row / a.G, hq = g * a.G + row % a.G;
    const int p = first + tq;
    const int pa = max(first + r0 / a.G, 0), pb = first + min(r0 + kRows - 1, rows - 1) / a.G;

    const bool live = r0 + 32 * w + c32 < rows;

    f32x16_v o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    if (pb >= 0) {
        // tokens [0, ns) and [ws, pb], each of which some row of the block sees; without a window the sinks alone
        const int ws = a.window > 0 ? max(pa - a.window + 1, 0) : pb + 1;
        const int ns = min(a.sink, ws);
        const int st = (ns + kKeys - 1) / kKeys, all = st + (pb + 1 - ws + kKeys - 1) / kKeys;
        const int per = (all + a.nsplit - 1) / a.nsplit, tb = split * per, nt = min(all, tb + per);   // this share's tiles
        const int pw0 = __builtin_amdgcn_readfirstlane(p), pw1 = __builtin_amdgcn_readlane(p, 31);   // this wave's positions
        const uint16_t* kb = a.k + (int64_t)b * a.k_sb + (int64_t)g * a.k_sh;
        const uint16_t* vb = a.v + (int64_t)b * a.v_sb + (int64_t)g * a.v_sh;
        auto tile_begin = [&](int t) { return t < st ? t * kKeys : ws + (t - st) * kKeys; };
        auto tile_end = [&](int t) { return t < st ? min(ns, (t + 1) * kKeys) : min(pb + 1, ws + (t - st + 1) * kKeys); };
        const int piece = (lane & 15) ^ (4 * (lane >> 4));
        auto load = [&](int t, const uint16_t* base, int64_t sn, char* to) {   // rows past the tile's end repeat its last
            const int j0 = tile_begin(t), jl = tile_end(t) - 1;                // one (they weigh 0)
#pragma unroll
            for (int u = 0; u < kKeys / 4 / NW; ++u) {
                const int block = NW * u + w;
                const uint32_t j = (uint32_t)min(j0 + 4 * block + (lane >> 4), jl);
                load_lds16(base + (uint64_t)j * (uint32_t)sn + piece * 8, to + block * kBlockBytes);
            }
        };
        if (tb < nt) {
            load(tb, kb, a.k_sn, k0);
            load(tb, vb, a.v_sn, v0);
            if (tb + 1 < nt) load(tb + 1, kb, a.k_sn, k1);
        }
        uint4 qf[8];
        const float s2 = fabsf(a.s2);                   // a negative scale goes into the query's signs
        const uint32_t flip = a.s2 < 0.0f ? 0x80008000u : 0u;
        const uint16_t* qr = a.q + (int64_t)b * a.q_sb + (int64_t)hq * a.q_sh + (int64_t)tq * a.q_st + 8 * hf;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            qf[i] = *reinterpret_cast<const uint4*>(qr + 16 * i);
            qf[i] = make_uint4(qf[i].x ^ flip, qf[i].y ^ flip, qf[i].z ^ flip, qf[i].w ^ flip);
        }

        // this lane's LDS offsets: K row c32, pieces 4x + hf on; V row 4 hf + c16 / 4, pieces 4x + its half of 32 columns
        const int c16 = lane & 15, vpiece = 2 * ((lane >> 4) & 1) + ((c16 & 3) >> 1);
        int ka[4], va[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            ka[x] = (c32 >> 2) * kBlockBytes + (c32 & 3) * 256 + ((4 * x + hf) ^ (4 * (c32 & 3))) * 16;
            va[x] = hf * kBlockBytes + (c16 >> 2) * 256 + ((4 * x + vpiece) ^ (4 * (c16 >> 2))) * 16 + 8 * (c16 & 1);
        }
        auto products = [&](const char* kl, f32x16_v (&x)[2]) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[s][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const uint4 kf = *reinterpret_cast<const uint4*>(kl + ka[i >> 1] + 32 * (i & 1) + 8 * s * kBlockBytes);
                    x[s] = mfma32<DT>(kf, qf[i], x[s]);
                }
        };
        // tile t's logits: those not visible masked, the reference raised where the maximum has outgrown it
        auto settle = [&](int t, f32x16_v (&x)[2]) {
            const int j0 = tile_begin(t), j1 = tile_end(t);
            // every row of the wave sees the whole tile, or masks
            const bool whole = j1 - j0 == kKeys && j1 - 1 <= pw0 && (j1 <= a.sink || j0 > pw1 - a.window);
            float mx = -INFINITY;
            if (!whole) {
                // token j0 + 4 hf + i, i known at compile time: i <= hi, and i < sk or i > lo
                const int at = j0 + 4 * hf, hi = min(p, j1 - 1) - at, sk = a.sink - at, lo = p - a.window - at;
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int i = 32 * s + (e & 3) + 8 * (e >> 2);
                        const bool seen = (i <= hi) & ((i < sk) | (i > lo));
                        x[s][e] = seen ? x[s][e] : -INFINITY;
                    }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, x[s][e]);
            mx = max_x32(mx) * s2;
            const bool grown = mx > m + kSlack<DT>;                 // m = -inf: the first visible tile
            if (__any(grown)) {
                const float m_new = grown ? mx : m;
                const float al = grown ? exp2_ftz(m - m_new) : 1.0f;
                m = m_new;
                l *= al;
#pragma unroll
                for (int d = 0; d < 4; ++d) o[d] *= al;
            }
        };
        auto weights = [&](const f32x16_v (&x)[2], uint4 (&pf)[4]) {
            const float ref = m == -INFINITY ? 0.0f : m - kShift<DT>;   // a row that has seen nothing yet: weights 0
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int h8 = 0; h8 < 2; ++h8) {
                    uint32_t u[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y0 = exp2_ftz(__builtin_fmaf(x[s][8 * h8 + 2 * e], s2, -ref));
                        const float y1 = exp2_ftz(__builtin_fmaf(x[s][8 * h8 + 2 * e + 1], s2, -ref));
                        l += y0 + y1;
                        u[e] = round_pair<DT>(y0, y1);
                    }
                    pf[2 * s + h8] = make_uint4(u[0], u[1], u[2], u[3]);
                    asm("" : "+v"(l));                          // summed here, not where l is next read: the unrounded
                }                                               // weights would stay in registers until then
        };
        auto values = [&](const char* vl, const uint4 (&pf)[4]) {
#pragma unroll
            for (int q = 0; q < 4; ++q)                         // 16 tokens each
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const u32x2_v lo = read_transposed(vl + va[d] + 4 * q * kBlockBytes);
                    const u32x2_v hi = read_transposed(vl + va[d] + (4 * q + 2) * kBlockBytes);
                    o[d] = mfma32<DT>(make_uint4(lo.x, lo.y, hi.x, hi.y), pf[q], o[d]);
                }
        };
        auto arrive = [&] {   // what this step reads is there, and every wave has left what it loads over
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        };
        // tile t's weights and values, with tile t + 1's logits between them
        auto step = [&](int t, f32x16_v (&x)[2], f32x16_v (&xn)[2], const char* kl, const char* vl, char* kn, char* vn) {
            arrive();
            if (t + 2 < nt) load(t + 2, kb, a.k_sn, kn);
            load(t + 1, vb, a.v_sn, vn);
            uint4 pf[4];
            products(kl, xn);
            weights(x, pf);
            values(vl, pf);
            settle(t + 1, xn);
        };
        auto last = [&](const f32x16_v (&x)[2], const char* vl) {
            arrive();
            uint4 pf[4];
            weights(x, pf);
            values(vl, pf);
        };
        if (tb < nt) {
            f32x16_v xa[2], xb[2];
            arrive();
            products(k0, xa);
            settle(tb, xa);
            int t = tb;
            for (; t + 2 < nt; t += 2) {
                step(t, xa, xb, k1, v0, k0, v1);
                step(t + 1, xb, xa, k0, v1, k1, v0);
            }
            if (t + 1 < nt) {
                step(t, xa, xb, k1, v0, k0, v1);
                last(xb, v1);
            } else {
                last(xa, v0);
            }
        }
    }
    l += __shfl_xor(l, 32, 64);
    if (!live) return;
    if (a.nsplit > 1) {                                         // a share: unnormalised, by row, joined afterwards
        const int64_t i = ((int64_t)bh * rows + row) * a.nsplit + split;
        if (hf == 0) a.part_ml[i] = make_float2(m, l);
        float* to = a.part_o + i * kHeadDim;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<f32x4_v*>(to + 32 * d + 8 * e + 4 * hf) =
                    f32x4_v{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
        return;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;               // nothing visible: 0
    uint16_t* out = a.out + (int64_t)b * a.o_sb + (int64_t)hq * a.o_sh + (int64_t)tq * a.o_st;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x0 = round_pair<DT>(o[d][4 * e] * inv, o[d][4 * e + 1] * inv);
            const uint32_t x1 = round_pair<DT>(o[d][4 * e + 2] * inv, o[d][4 * e + 3] * inv);
            *reinterpret_cast<uint2*>(out + 32 * d + 8 * e + 4 * hf) = make_uint2(x0, x1);
        }
}

// The shares of row (bh, token, head of the group) joined and written in the cache's type.
template <int DT, int NG>
__global__ __launch_bounds__(256, 4) void prefill_merge_kernel(PrefillArgs a)
{
    __shared__ f32x4_v osum[256];
    __shared__ float2 mlsum[256];
    const int64_t per = (int64_t)a.t * a.G;
    const Joined j = join_shares<NG, 32>(a.part_o, a.part_ml, a.nsplit, a.B * a.Hkv * per, blockIdx.x, osum, mlsum);
    if (j.row < 0) return;
    const int bh = (int)(j.row / per), row = (int)(j.row % per);
    uint16_t* out = a.out + (int64_t)(bh / a.Hkv) * a.o_sb + (int64_t)(bh % a.Hkv * a.G + row % a.G) * a.o_sh +
                    (int64_t)(row / a.G) * a.o_st + j.d;
    *reinterpret_cast<uint2*>(out) = make_uint2(round_pair<DT>(j.o[0], j.o[1]), round_pair<DT>(j.o[2], j.o[3]));
}

template <int DT>
void launch_type(const PrefillArgs& a, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * a.blocks * a.nsplit));
    if (a.rows_per_wg == 256) hipLaunchKernelGGL((prefill_kernel<DT, 8>), grid, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((prefill_kernel<DT, 4>), grid, dim3(256), 0, st, a);
    if (a.nsplit == 1) return;
    const int64_t rows = (int64_t)a.B * a.Hq * a.t;
    if (a.nsplit <= 8) hipLaunchKernelGGL((prefill_merge_kernel<DT, 1>), dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((prefill_merge_kernel<DT, 8>), dim3((unsigned)rows), dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_prefill(const PrefillArgs& a, int dtype, hipStream_t st)
{
    if (dtype == 1) launch_type<1>(a, st);
    else launch_type<0>(a, st);
    return hipGetLastError();
}

}  // namespace hill
