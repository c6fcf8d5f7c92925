// Matrix-core building blocks of the dense attention kernels: the tile
// products, the transposing LDS read that feeds the values, the splits of
// fp32 weights into 16-bit terms and the 4-bit decoding.
#pragma once

#include "hill_device.h"
#include "hill_internal.h"

namespace hill {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf168_t __attribute__((ext_vector_type(8)));
typedef float f32x2_v __attribute__((ext_vector_type(2)));
typedef float f32x4_v __attribute__((ext_vector_type(4)));
typedef float f32x16_v __attribute__((ext_vector_type(16)));
typedef short short4_v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_v __attribute__((ext_vector_type(2)));

// 16x16 (32 deep) and 32x32 (16 deep) products of packed 16-bit operands,
// DT 0 fp16, 1 bf16.  Lane l holds row / column l % 16 (l % 32) of its
// operand and eight consecutive depth elements, 8 * (l / 16) (8 * (l / 32))
// on; the result's column is the same, its rows 4 * (l / 16) + r (r % 4 +
// 8 * (r / 4) + 4 * (l / 32)).  The sum does not depend on which depth element
// is called which, as long as both operands agree.
template <int DT>
__device__ __forceinline__ f32x4_v mfma16(uint4 a, uint4 b, f32x4_v c)
{
    if constexpr (DT == 1)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf168_t, a), __builtin_bit_cast(bf168_t, b), c, 0,
                                                       0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0,
                                                      0);
}

template <int DT>
__device__ __forceinline__ f32x16_v mfma32(uint4 a, uint4 b, f32x16_v c)
{
    if constexpr (DT == 1)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf168_t, a), __builtin_bit_cast(bf168_t, b), c, 0,
                                                       0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0,
                                                      0);
}

// Transposing LDS read: the sixteen lanes of a group point at four rows of
// sixteen 16-bit elements, lane i at elements 4 * (i % 4) on of row i / 4, and
// lane i receives element i of the four rows.
__device__ __forceinline__ u32x2_v read_transposed(const void* p)
{
    typedef __attribute__((address_space(3))) short4_v* lds_ptr;
    return __builtin_bit_cast(u32x2_v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p));
}

// Softmax weights are split exactly enough for the 32-bit result: bf16 terms
// by truncation (3 x 8 bits: all 24), fp16 terms by rounding (2 x 11 bits).
// fp16 weights carry a factor 2^kWeightShift, so that a weight of 2^-28 of the
// largest still is a normal number and its second term keeps 2^-38.
template <int DT>
constexpr float kWeightShift = DT == 1 ? 0.0f : 14.0f;
template <int DT>
constexpr int kWeightTerms = DT == 1 ? 3 : 2;

// 16-bit pair from the upper halves of two words (lo, hi).
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi)
{
    return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}

__device__ __forceinline__ uint32_t lower_halves(uint32_t lo, uint32_t hi)
{
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// Eight weights as kWeightTerms<DT> operands.
template <int DT>
__device__ __forceinline__ void split_weights(const float (&p)[8], uint4 (&t)[kWeightTerms<DT>])
{
    uint32_t w[kWeightTerms<DT>][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = p[2 * i], y = p[2 * i + 1];
        if constexpr (DT == 1) {
#pragma unroll
            for (int u = 0; u < 3; ++u) {
                const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
                w[u][i] = upper_halves(xb, yb);
                x -= __uint_as_float(xb & 0xffff0000u);
                y -= __uint_as_float(yb & 0xffff0000u);
            }
        } else {
            const half2_t h = __builtin_convertvector(f32x2_v{x, y}, half2_t);
            const half2_t r = __builtin_convertvector((f32x2_v{__builtin_fmaf((float)h[0], -1.0f, x), __builtin_fmaf((float)h[1], -1.0f, y)}),
                                                      half2_t);
            w[0][i] = __builtin_bit_cast(uint32_t, h);
            w[1][i] = __builtin_bit_cast(uint32_t, r);
        }
    }
#pragma unroll
    for (int u = 0; u < kWeightTerms<DT>; ++u) t[u] = make_uint4(w[u][0], w[u][1], w[u][2], w[u][3]);
}

// Eight 4-bit codes of a word (element 2i in bits 4i.., element 2i+1 in bits
// 16+4i..) as the fp16 values code * scale + zero, one rounding each.  A code
// becomes a number by its bits under an exponent: 1024 + c (low nibble of a
// byte) or 1024 + 16 c, both exact, from which c follows exactly.
__device__ __forceinline__ uint4 decode8(uint32_t x, half2_t scale, half2_t zero)
{
    const half2_t k1024 = {(_Float16)1024.0f, (_Float16)1024.0f};
    const half2_t k16th = {(_Float16)0.0625f, (_Float16)0.0625f}, k64 = {(_Float16)-64.0f, (_Float16)-64.0f};
    uint32_t exponent = 0x64006400u;
    asm("" : "+v"(exponent));   // in a vector register: one v_and_or_b32 takes one constant
    uint32_t r[4];
#pragma unroll
    for (int s = 0; s < 4; s += 2) {
        const uint32_t y = x >> (4 * s);
        const half2_t lo = __builtin_bit_cast(half2_t, (y & 0x000f000fu) | exponent) - k1024;
        const half2_t hi = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, (y & 0x00f000f0u) | exponent), k16th, k64);
        r[s] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(lo, scale, zero));
        r[s + 1] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(hi, scale, zero));
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// The same values in the order (0, 4), (1, 5), (2, 6), (3, 7), two operations in
// thirteen fewer: a byte that holds a code is, read as fp8 e4m3, exactly code * 2^-9 (its
// subnormals and first binade), and one conversion makes two fp16 numbers of them.
__device__ __forceinline__ uint4 decode8_split(uint32_t x, half2_t scale, half2_t zero)
{
    const uint32_t y[2] = {x & 0x0f0f0f0fu, (x >> 4) & 0x0f0f0f0fu};
    uint32_t r[4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const half2_t c0 = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y[s], 512.0f, false));
        const half2_t c1 = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y[s], 512.0f, true));
        r[2 * s] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c0, scale, zero));
        r[2 * s + 1] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c1, scale, zero));
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// (scale, zero) of a group, broadcast to pairs.
__device__ __forceinline__ void group_params(uint32_t par, half2_t& scale, half2_t& zero)
{
    const half2_t p = __builtin_bit_cast(half2_t, par);
    scale = half2_t{p[0], p[0]};
    zero = half2_t{p[1], p[1]};
}

// Four dimensions (from d on) of a row's output; row < 0: nothing to write.
struct Joined {
    int64_t row;
    int d;
    f32x4_v o;
};

// Joins the shares of attention rows (unnormalised outputs part_o [rows, nsplit,
// 128], (max, sum) part_ml [rows, nsplit]) in a workgroup of 256 threads:
// LANES lanes of four dimensions each (32: a whole row) in NG groups make a row, or
// a quarter of one; group i takes shares i, i + NG, ... with up to eight loads in
// flight.  Empty shares have sum 0, and a row without any gives 0.
template <int NG, int LANES>
__device__ __forceinline__ Joined join_shares(const float* part_o, const float2* part_ml, int nsplit, int64_t rows, int64_t block,
                                              f32x4_v* osum, float2* mlsum)
{
    constexpr int kParts = 32 / LANES, kPerWg = 256 / (NG * LANES);   // parts of a row; (row, part) pairs per workgroup
    const int tid = threadIdx.x, grp = tid / LANES % NG;
    const int64_t pairs = rows * kParts, mine = block * kPerWg + tid / (NG * LANES);
    const int64_t rp = mine < pairs ? mine : pairs - 1;               // past the last: it again
    Joined r;
    r.d = 4 * (tid % LANES + LANES * (int)(rp % kParts));
    r.row = rp / kParts;
    const float2* ml = part_ml + r.row * nsplit;
    const float* po = part_o + r.row * nsplit * kHeadDim + r.d;
    if (mine >= pairs) r.row = -1;
    float m = -INFINITY, l = 0.0f;
    f32x4_v o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = grp; s0 < nsplit; s0 += 8 * NG) {
        float2 v[8];
        f32x4_v x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {                                 // past the last share: it again, with weight 0
            const int s = min(s0 + i * NG, nsplit - 1);
            v[i] = ml[s];
            x[i] = *reinterpret_cast<const f32x4_v*>(po + (int64_t)s * kHeadDim);
            if (s0 + i * NG >= nsplit) v[i].y = 0.0f;
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, v[i].y > 0.0f ? v[i].x : -INFINITY);
        const float al = l > 0.0f ? exp2_ftz(m - top) : 0.0f;
        o *= al;
        l *= al;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float f = v[i].y > 0.0f ? exp2_ftz(v[i].x - top) : 0.0f;
            o += f * x[i];
            l += f * v[i].y;
        }
        m = top;
    }
    if constexpr (NG > 1) {
        osum[tid] = o;
        mlsum[tid] = make_float2(m, l);
        __syncthreads();
        if (grp != 0) r.row = -1;
        float top = m;
#pragma unroll 8
        for (int i = 1; i < NG; ++i) top = fmaxf(top, mlsum[(tid + LANES * i) & 255].x);
        const float al = l > 0.0f ? exp2_ftz(m - top) : 0.0f;
        o *= al;
        l *= al;
#pragma unroll 8
        for (int i = 1; i < NG; ++i) {
            const float2 v = mlsum[(tid + LANES * i) & 255];          // (groups other than 0 add to no avail)
            const float f = v.y > 0.0f ? exp2_ftz(v.x - top) : 0.0f;
            o += f * osum[(tid + LANES * i) & 255];
            l += f * v.y;
        }
    }
    r.o = l > 0.0f ? o * (1.0f / l) : o * 0.0f;
    return r;
}

// Which tokens a query sees: the first ns and, gap tokens further, the last
// nw of a sequence of `len`.  Position i of the ns + nw visible ones is token
// i + (i < ns ? 0 : gap).
struct Visible {
    int ns, nv, gap;
    __device__ __forceinline__ int token(int i) const { return i + (i < ns ? 0 : gap); }
};

__device__ __forceinline__ Visible visible(int len, int sink, int window)
{
    Visible x;
    x.ns = min(sink, len);
    x.nv = x.ns + min(window, len - x.ns);
    x.gap = len - x.nv;
    return x;
}

// Length of sequence b, taken into [0, n].
__device__ __forceinline__ int seq_len(const int32_t* lens, int b, int n)
{
    return lens ? min(max(lens[b], 0), n) : n;
}

}  // namespace hill
