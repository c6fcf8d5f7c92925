// Writer and reader of the 4-bit cache (the format is hill.h's).  Sixteen
// lanes take a row, eight elements each, four lanes a group of 32; a lane makes
// one word of eight codes.  Both directions are copies in effect: 256 B of 16-bit
// row against 80 B of codes and parameters, four rows per lane group in flight.
// Measured: 32768 rows of 8 KV heads, K and V, 176 MB each way: 39 us to write
// them (4.5 TB/s), 27 to read them back (6.5); a copy of a GiB reaches 5.0.
#include "mfma_device.h"

namespace hill {

namespace {

constexpr int kBatch = 4;                  // rows per lane group
constexpr int kRows = 16 * kBatch;         // rows per workgroup

// Min and max over aligned groups of four lanes.
__device__ __forceinline__ float min4(float v)
{
    v = fminf(v, dpp<0xB1>(v));
    return fminf(v, dpp<0x4E>(v));
}

__device__ __forceinline__ float max4(float v)
{
    v = fmaxf(v, dpp<0xB1>(v));
    return fmaxf(v, dpp<0x4E>(v));
}

template <int DT>
__global__ __launch_bounds__(256) void pack_kernel(PackArgs a)
{
    const bool is_v = blockIdx.z != 0;
    const uint16_t* src = is_v ? a.v : a.k;
    const int64_t sb = is_v ? a.v_sb : a.k_sb, sh = is_v ? a.v_sh : a.k_sh, sn = is_v ? a.v_sn : a.k_sn;
    uint8_t* codes = is_v ? a.vc : a.kc;
    uint32_t* par = is_v ? a.vp : a.kp;
    const int l16 = threadIdx.x & 15;
    const int i0 = blockIdx.x * kRows + (threadIdx.x >> 4);   // then + 16, ...
    for (int bg = blockIdx.y; bg < a.B * a.Hkv; bg += gridDim.y) {
        const int b = bg / a.Hkv, g = bg % a.Hkv;
        const uint16_t* rows = src + (int64_t)b * sb + (int64_t)g * sh + l16 * 8;
        const int64_t at = a.at ? a.at[b] : a.at0;
        uint4 w[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) w[u] = load_stream16(rows + (int64_t)min(i0 + 16 * u, a.rows - 1) * sn);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const uint32_t pw[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
            float x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) widen2<DT>(pw[i], x[2 * i], x[2 * i + 1]);
            float lo = INFINITY, hi = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = fminf(fmaxf(x[i], -65504.0f), 65504.0f);   // fp16's range
                lo = fminf(lo, x[i]);
                hi = fmaxf(hi, x[i]);
            }
            lo = min4(lo);
            hi = max4(hi);
            float step = (hi - lo) * (1.0f / 15.0f);
            asm("" : "+v"(step));   // an fp32 value before it becomes fp16: not one rounding of the product
            _Float16 scale = (_Float16)step;
            const _Float16 zero = (_Float16)lo;
            // rounded up, a scale can carry the largest code past fp16's range: then the one below it
            if (__builtin_elementwise_fma((_Float16)15.0f, scale, zero) == (_Float16)INFINITY)
                scale = __builtin_bit_cast(_Float16, (uint16_t)(__builtin_bit_cast(uint16_t, scale) - 1));
            const float inv = (float)scale > 0.0f ? 1.0f / (float)scale : 0.0f;
            uint32_t word = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = fminf(fmaxf(rintf((x[i] - (float)zero) * inv), 0.0f), 15.0f);
                word |= (uint32_t)t << (4 * (i >> 1) + 16 * (i & 1));
            }
            const int64_t j = at + i0 + 16 * u;
            if (i0 + 16 * u < a.rows && j >= 0 && j < a.cap) {
                const int64_t row = (int64_t)bg * a.cap + j;
                *reinterpret_cast<uint32_t*>(codes + row * 64 + l16 * 4) = word;
                if ((l16 & 3) == 0) par[row * 4 + (l16 >> 2)] = __builtin_bit_cast(uint32_t, half2_t{scale, zero});
            }
        }
    }
}

// fp16 pair -> bf16 pair, to nearest.
__device__ __forceinline__ uint32_t half2_to_bf162(uint32_t x)
{
    const half2_t h = __builtin_bit_cast(half2_t, x);
    const bf162_t r = {(__bf16)(float)h[0], (__bf16)(float)h[1]};
    return __builtin_bit_cast(uint32_t, r);
}

template <int DT>
__global__ __launch_bounds__(256) void unpack_kernel(PackArgs a)
{
    const bool is_v = blockIdx.z != 0;
    uint16_t* dst = is_v ? a.v : a.k;
    const int64_t sb = is_v ? a.v_sb : a.k_sb, sh = is_v ? a.v_sh : a.k_sh, sn = is_v ? a.v_sn : a.k_sn;
    const uint8_t* codes = is_v ? a.vc : a.kc;
    const uint32_t* par = is_v ? a.vp : a.kp;
    const int l16 = threadIdx.x & 15;
    const int i0 = blockIdx.x * kRows + (threadIdx.x >> 4);
    for (int bg = blockIdx.y; bg < a.B * a.Hkv; bg += gridDim.y) {
        const int b = bg / a.Hkv, g = bg % a.Hkv;
        uint16_t* rows = dst + (int64_t)b * sb + (int64_t)g * sh + l16 * 8;
        uint32_t w[kBatch], p[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t row = (int64_t)bg * a.cap + a.at0 + min(i0 + 16 * u, a.rows - 1);
            w[u] = *reinterpret_cast<const uint32_t*>(codes + row * 64 + l16 * 4);
            p[u] = par[row * 4 + (l16 >> 2)];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            half2_t scale, zero;
            group_params(p[u], scale, zero);
            uint4 x = decode8(w[u], scale, zero);
            if constexpr (DT == 1)
                x = make_uint4(half2_to_bf162(x.x), half2_to_bf162(x.y), half2_to_bf162(x.z), half2_to_bf162(x.w));
            if (i0 + 16 * u < a.rows) *reinterpret_cast<uint4*>(rows + (int64_t)(i0 + 16 * u) * sn) = x;
        }
    }
}

dim3 pack_grid(const PackArgs& a)
{
    const int64_t bg = (int64_t)a.B * a.Hkv;
    return dim3((a.rows + kRows - 1) / kRows, (unsigned)(bg < 65535 ? bg : 65535), 2);
}

}  // namespace

hipError_t launch_pack(const PackArgs& a, int dtype, hipStream_t st)
{
    if (dtype == 1) hipLaunchKernelGGL(pack_kernel<1>, pack_grid(a), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(pack_kernel<0>, pack_grid(a), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_unpack(const PackArgs& a, int dtype, hipStream_t st)
{
    if (dtype == 1) hipLaunchKernelGGL(unpack_kernel<1>, pack_grid(a), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(unpack_kernel<0>, pack_grid(a), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace hill
