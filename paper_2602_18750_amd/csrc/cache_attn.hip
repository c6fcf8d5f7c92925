// One token's dense attention over a cache: over the first tokens and a
// sliding window of 16-bit rows, over the same or all rows of a cache held in
// 4 bits, or over a list of the latter's rows; optionally with the logits kept
// for the importance S.
//
//   x_i = s2 * q.K_j(i),  m = max x,  l = sum 2^(x - m),  out = sum 2^(x - m) V / l
//
//  cache_attn   one (sequence, KV head, 16 query heads, share of the visible
//               positions) per workgroup of four waves, one pass with running
//               m and l
//  cache_merge  the shares of a head joined, and S += the weights
//
// The bound is memory: 512 B (16-bit) or 160 B (4-bit) per token and KV head
// against 16 heads' products on the matrix cores.  A wave takes 32 tokens at a time,
// without barriers: K rows come in the operand's layout (lane: one token,
// 16-byte pieces) and give x^T (tokens x heads), whose lanes hold exactly what
// the second product's weights operand needs; V rows go through a private 9
// KiB of LDS and come back transposed.  The rows of the next 32 tokens are
// requested before the weights of these are formed.  Products are exact in the matrix
// cores' fp32 sums: the weights are split into 16-bit terms (split_weights), a
// bf16 query over fp16 values is scaled by a power of two into fp16's range
// (elements below 2^-29 of its largest lose bits).
//
// Measured: 32 x 16K tokens, window 4096, 8 KV heads, bf16 rows, 554 MB: 80 to
// 87 us, 6.4 to 6.9 TB/s (reading alone reaches 6.7; with rows kept out of the
// caches, since each is read once: 104.8 -> 87.1).  4-bit: 32K tokens, 42 MB,
// 12 us and 2.4 to 4 for the join, of 8 to 10 for reading them; 4 x 131K, 671 MB,
// 133 us without S; with it 138, and 14 for the join, which reads again the
// logits that the first launch wrote (67 MB each way).  There the instructions count as
// much as the bytes: eleven per word of eight codes, whose results meet at most 16
// heads.
#include "mfma_device.h"

namespace hill {

namespace {

constexpr int kTile = 32;        // tokens per wave and step
constexpr int kVRow = 144;       // 16-bit elements per V row in LDS: 288 bytes, so that the rows of a transposing
                                 // read lie in different banks
constexpr int kHeads = 16;       // query heads per workgroup

enum Rows : int { kRowsF16 = 0, kRowsBf16 = 1, kRowsPacked = 2 };

// What a lane holds of a tile before it is used.
template <int KT>
struct TileRegs {
    uint4 k[KT == kRowsPacked ? 2 : 8];
    uint4 v[KT == kRowsPacked ? 2 : 8];
    uint32_t kp[2], vp[2];       // packed: (scale, zero) of the codes above
};

// Where the rows of a tile lie: bases of the (sequence, KV head) for every lane,
// and each lane's offsets from a tile's first row, which are the same in every
// tile of consecutive tokens.
template <int KT>
struct RowBase {
    const char* k;
    const char* v;
    const char* kp;
    const char* vp;
    uint32_t ko, vo;                                // bytes from the tile's first row
    bool near;                                      // the offsets fit 32 bits
};

template <int KT>
__device__ __forceinline__ RowBase<KT> row_base(const CacheAttnArgs& a, int b, int g)
{
    const int lane = threadIdx.x & 63, c = lane & 15, qd = lane >> 4;
    RowBase<KT> r;
    if constexpr (KT == kRowsPacked) {
        const int64_t row0 = ((int64_t)b * a.Hkv + g) * a.cap;
        r.k = reinterpret_cast<const char*>(a.kc) + row0 * 64;
        r.v = reinterpret_cast<const char*>(a.vc) + row0 * 64;
        r.kp = reinterpret_cast<const char*>(a.kp) + row0 * 16;
        r.vp = reinterpret_cast<const char*>(a.vp) + row0 * 16;
        r.ko = c * 64 + qd * 16;
        r.vo = lane * 16;
        r.near = true;
    } else {
        r.k = reinterpret_cast<const char*>(a.k + (int64_t)b * a.k_sb + (int64_t)g * a.k_sh);
        r.v = reinterpret_cast<const char*>(a.v + (int64_t)b * a.v_sb + (int64_t)g * a.v_sh);
        r.ko = c * 2 * (uint32_t)a.k_sn + qd * 16;
        r.vo = qd * 2 * (uint32_t)a.v_sn + c * 16;
        r.near = max(a.k_sn, a.v_sn) < (1 << 25);
    }
    return r;
}

__device__ __forceinline__ uint32_t load_word(const char* p) { return *reinterpret_cast<const uint32_t*>(p); }

// Positions [i0, i0 + 32): consecutive tokens from uniform bases, or (at the
// ends of the visible ranges, and over lists) a token per row; positions past
// the last repeat it.  tok: a list's tokens, taken into [0, n).
template <int KT, bool IDX>
__device__ __forceinline__ void load_tile(const CacheAttnArgs& a, const RowBase<KT>& r, const Visible& vis, int i0, int tok,
                                          TileRegs<KT>& t)
{
    const int lane = threadIdx.x & 63, c = lane & 15, qd = lane >> 4;
    // One branch on one value: as a chain of conditions the compiler joined the paths with registers that one of
    // them had not set.
    const bool plain = !IDX & r.near & (i0 + kTile <= vis.nv) & ((i0 >= vis.ns) | (i0 + kTile <= vis.ns));
    if (plain) {
        const uint64_t j0 = (uint64_t)vis.token(i0);
        if constexpr (KT == kRowsPacked) {
            const char *k = r.k + j0 * 64, *v = r.v + j0 * 64, *kp = r.kp + j0 * 16, *vp = r.vp + j0 * 16;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                t.k[u] = load_stream16(k + r.ko + 1024 * u);
                t.kp[u] = load_word(kp + (r.ko >> 2) + 256 * u);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                t.v[u] = load_stream16(v + r.vo + 1024 * u);
                t.vp[u] = load_word(vp + (r.vo >> 2) + 256 * u);
            }
        } else {
            const uint64_t kn = 2 * (uint64_t)(uint32_t)a.k_sn, vn = 2 * (uint64_t)(uint32_t)a.v_sn;
            const char *k = r.k + j0 * kn, *v = r.v + j0 * vn;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) t.k[4 * u + i] = load_stream16(k + 16 * u * kn + r.ko + 64 * i);
#pragma unroll
            for (int u = 0; u < 8; ++u) t.v[u] = load_stream16(v + 4 * u * vn + r.vo);
        }
        return;
    }
    auto token = [&](int i) -> uint64_t {   // of position i0 + i
        if constexpr (IDX) return (uint64_t)__shfl(tok, i, 64);
        return (uint64_t)vis.token(min(i0 + i, vis.nv - 1));
    };
    if constexpr (KT == kRowsPacked) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t at = 64u * (uint32_t)token(16 * u + c) + 16u * qd;   // n < 2^22
            t.k[u] = load_stream16(r.k + at);
            t.kp[u] = load_word(r.kp + (at >> 2));
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t at = 64u * (uint32_t)token(16 * u + (lane >> 2)) + 16u * (lane & 3);
            t.v[u] = load_stream16(r.v + at);
            t.vp[u] = load_word(r.vp + (at >> 2));
        }
    } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const char* k = r.k + token(16 * u + c) * 2 * (uint32_t)a.k_sn + 16 * qd;
#pragma unroll
            for (int i = 0; i < 4; ++i) t.k[4 * u + i] = load_stream16(k + 64 * i);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) t.v[u] = load_stream16(r.v + token(4 * u + qd) * 2 * (uint32_t)a.v_sn + 16 * c);
    }
}

// The V rows of a tile into LDS as 16-bit rows.
template <int KT>
__device__ __forceinline__ void stage_values(const TileRegs<KT>& t, uint16_t* vl)
{
    const int lane = threadIdx.x & 63, c = lane & 15, qd = lane >> 4;
    if constexpr (KT == kRowsPacked) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            half2_t scale, zero;
            group_params(t.vp[u], scale, zero);
            uint4* to = reinterpret_cast<uint4*>(vl + (16 * u + (lane >> 2)) * kVRow + (lane & 3) * 32);
            to[0] = decode8_split(t.v[u].x, scale, zero);
            to[1] = decode8_split(t.v[u].y, scale, zero);
            to[2] = decode8_split(t.v[u].z, scale, zero);
            to[3] = decode8_split(t.v[u].w, scale, zero);
        }
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) *reinterpret_cast<uint4*>(vl + (4 * u + qd) * kVRow + c * 8) = t.v[u];
    }
}

// x^T of the tile: lane (c, qd) gets tokens 16 u + 4 qd + r of head c.
template <int KT>
__device__ __forceinline__ void tile_logits(const TileRegs<KT>& t, const uint4 (&qf)[4], f32x4_v (&x)[2])
{
    constexpr int DT = KT == kRowsBf16 ? 1 : 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        x[u] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (KT == kRowsPacked) {
            half2_t scale, zero;
            group_params(t.kp[u], scale, zero);
            const uint32_t w[4] = {t.k[u].x, t.k[u].y, t.k[u].z, t.k[u].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) x[u] = mfma16<DT>(decode8_split(w[i], scale, zero), qf[i], x[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[u] = mfma16<DT>(t.k[4 * u + i], qf[i], x[u]);
        }
    }
}

// A query row (lane's 8-element pieces) as fp16: bf16 elements times 2^-e with
// the row's largest in [2^14, 2^15); returns 2^e.
__device__ __forceinline__ float bf16_query_to_half(uint4 (&qf)[4])
{
    float x[32], m = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {qf[i].x, qf[i].y, qf[i].z, qf[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            widen2<1>(w[j], x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
            m = fmaxf(m, fmaxf(fabsf(x[8 * i + 2 * j]), fabsf(x[8 * i + 2 * j + 1])));
        }
    }
    m = max_x16_x32(m);
    int e = 0;
    if (m > 0.0f && m < INFINITY) {
        frexpf(m, &e);
        e = max(e - 15, -100);   // 2^e times the softmax scale stays a normal number
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const half2_t h = {(_Float16)ldexpf(x[8 * i + 2 * j], -e), (_Float16)ldexpf(x[8 * i + 2 * j + 1], -e)};
            w[j] = __builtin_bit_cast(uint32_t, h);
        }
        qf[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return ldexpf(1.0f, e);
}

template <int KT, bool IDX, bool LOG>
__global__ __launch_bounds__(256, KT == kRowsPacked ? 4 : 3) void cache_attn_kernel(CacheAttnArgs a)
{
    constexpr int DT = KT == kRowsBf16 ? 1 : 0;
    constexpr int kTerms = kWeightTerms<DT>;
    __shared__ __attribute__((aligned(16))) uint16_t vlds[4 * kTile * kVRow];   // then the waves' outputs
    __shared__ float2 ml[4][kHeads];
    __shared__ float inv_l[kHeads];
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, qd = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int split = blockIdx.x % a.nsplit;
    int y = blockIdx.x / a.nsplit;
    const int ht = y % a.head_tiles;
    y /= a.head_tiles;
    const int g = y % a.Hkv, b = y / a.Hkv;
    const int h0 = ht * kHeads;                        // first head of the group
    const int h = g * a.G + min(h0 + c, a.G - 1);      // heads past the group repeat its last
    Visible vis;
    const int32_t* idx = nullptr;
    if constexpr (IDX) {
        idx = a.idx + ((int64_t)b * a.R + (a.R > 1 ? g : 0)) * a.ksel;
        vis.ns = vis.nv = a.ksel;
        vis.gap = 0;
    } else {
        vis = visible(seq_len(a.lens, b, a.n), a.sink, a.window);
    }
    const int tiles = (vis.nv + kTile - 1) / kTile, per = (tiles + a.nsplit - 1) / a.nsplit;
    const int t1 = min(tiles, (split + 1) * per);
    int t = split * per + w;

    uint4 qf[4];
    float s2 = fabsf(a.s2);                            // a negative scale goes into the query's signs
    const uint32_t flip = a.s2 < 0.0f ? 0x80008000u : 0u;
    {
        const uint16_t* qr = a.q + (int64_t)b * a.q_sb + (int64_t)h * a.q_sh;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            qf[i] = *reinterpret_cast<const uint4*>(qr + (KT == kRowsPacked ? 32 * qd + 8 * i : 32 * i + 8 * qd));
    }

    uint16_t* vl = vlds + w * kTile * kVRow;
    const uint16_t* vr = vl + (4 * qd + (c >> 2)) * kVRow + 4 * (c & 3);
    f32x4_v o[8];
#pragma unroll
    for (int d = 0; d < 8; ++d) o[d] = f32x4_v{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;

    // tokens of a list tile: lane i (and i + 32) holds that of position i; loaded a tile ahead of its rows
    auto list_tokens = [&](int tile) {
        int tok = 0;
        if constexpr (IDX) tok = min(max(idx[min(tile * kTile + (lane & 31), vis.nv - 1)], 0), a.n - 1);
        return tok;
    };
    const RowBase<KT> base = row_base<KT>(a, b, g);
    TileRegs<KT> regs;
    int tok = 0;
    if (t < t1) {
        load_tile<KT, IDX>(a, base, vis, t * kTile, list_tokens(t), regs);
        tok = list_tokens(min(t + 4, t1 - 1));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) qf[i] = make_uint4(qf[i].x ^ flip, qf[i].y ^ flip, qf[i].z ^ flip, qf[i].w ^ flip);
    if constexpr (KT == kRowsPacked)   // with the first rows on their way
        if (a.q_bf16) s2 *= bf16_query_to_half(qf);
    if constexpr (KT == kRowsPacked) {   // the order in which decode8_split gives a key's elements
#pragma unroll
        for (int i = 0; i < 4; ++i)
            qf[i] = make_uint4(lower_halves(qf[i].x, qf[i].z), upper_halves(qf[i].x, qf[i].z),
                               lower_halves(qf[i].y, qf[i].w), upper_halves(qf[i].y, qf[i].w));
    }
    for (; t < t1; t += 4) {
        f32x4_v x[2];
        stage_values<KT>(regs, vl);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // other lanes read what this one wrote
        tile_logits<KT>(regs, qf, x);
        if (t + 4 < t1) {
            load_tile<KT, IDX>(a, base, vis, (t + 4) * kTile, tok, regs);
            tok = list_tokens(min(t + 8, t1 - 1));
        }
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = x[e >> 2][e & 3];
        const int i0 = t * kTile + 4 * qd;             // this lane's positions: i0 + r and i0 + 16 + r
        if ((t + 1) * kTile > vis.nv) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i0 + 16 * (e >> 2) + (e & 3) >= vis.nv) p[e] = -INFINITY;
        }
        if constexpr (LOG) {
            if (h0 + c < a.G) {
                float* to = a.logits + ((int64_t)b * a.Hq + h) * a.ld + i0;   // ld holds whole tiles
                *reinterpret_cast<float4*>(to) = make_float4(p[0] * s2, p[1] * s2, p[2] * s2, p[3] * s2);
                *reinterpret_cast<float4*>(to + 16) = make_float4(p[4] * s2, p[5] * s2, p[6] * s2, p[7] * s2);
            }
        }
        float mx = p[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, p[e]);
        const float m_new = fmaxf(m, max_x16_x32(mx) * s2);
        if (__any(m_new > m)) {
            const float al = m_new > m ? exp2_ftz(m - m_new) : 1.0f;
            l *= al;
#pragma unroll
            for (int d = 0; d < 8; ++d) o[d] *= al;
        }
        m = m_new;
        const float ref = m == -INFINITY ? 0.0f : m - kWeightShift<DT>;   // logits below fp32's range alone so far: weights 0
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = exp2_ftz(__builtin_fmaf(p[e], s2, -ref));
            l += p[e];
        }
        uint4 pt[kTerms];
        split_weights<DT>(p, pt);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const u32x2_v lo = read_transposed(vr + 16 * d), hi = read_transposed(vr + 16 * kVRow + 16 * d);
            const uint4 vf = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
            for (int u = 0; u < kTerms; ++u) o[d] = mfma16<DT>(vf, pt[u], o[d]);
        }
    }

    // the four waves' outputs: (m, l) first, then the weighted sums
    l = sum_x16_x32(l);
    if (qd == 0) ml[w][c] = make_float2(m, l);
    __syncthreads();
    float M = -INFINITY, L = 0.0f;
#pragma unroll
    for (int u = 0; u < 4; ++u) M = fmaxf(M, ml[u][c].x);
#pragma unroll
    for (int u = 0; u < 4; ++u) L += ml[u][c].y > 0.0f ? ml[u][c].y * exp2_ftz(ml[u][c].x - M) : 0.0f;
    const float mine = l > 0.0f ? exp2_ftz(m - M) : 0.0f;
    float* ol = reinterpret_cast<float*>(vlds);        // [4][kHeads][kHeadDim]
    const int heads = min(kHeads, a.G - h0);
    if (c < heads) {
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const f32x4_v x = o[d] * mine;
            if constexpr (KT == kRowsPacked) {   // a value's elements lie in decode8_split's order
                float* to = ol + (w * kHeads + c) * kHeadDim + 16 * d + 8 * (qd >> 1) + 2 * (qd & 1);
                *reinterpret_cast<f32x2_v*>(to) = f32x2_v{x[0], x[2]};
                *reinterpret_cast<f32x2_v*>(to + 4) = f32x2_v{x[1], x[3]};
            } else {
                *reinterpret_cast<f32x4_v*>(ol + (w * kHeads + c) * kHeadDim + 16 * d + 4 * qd) = x;
            }
        }
    }
    if (tid < kHeads) {                                // lane c of wave 0 holds head c
        inv_l[tid] = L > 0.0f ? 1.0f / L : 0.0f;       // nothing visible: 0
        if (a.part_ml && h0 + tid < a.G)
            a.part_ml[((int64_t)b * a.Hq + g * a.G + h0 + tid) * a.nsplit + split] = make_float2(M, L);
    }
    __syncthreads();
    for (int e = tid; e < heads * (kHeadDim / 4); e += 256) {
        const int hh = e / (kHeadDim / 4), d = e % (kHeadDim / 4) * 4;
        f32x4_v s = *reinterpret_cast<const f32x4_v*>(ol + hh * kHeadDim + d);
#pragma unroll
        for (int u = 1; u < 4; ++u) s += *reinterpret_cast<const f32x4_v*>(ol + (u * kHeads + hh) * kHeadDim + d);
        const int64_t bh = (int64_t)b * a.Hq + g * a.G + h0 + hh;
        if (a.nsplit > 1) *reinterpret_cast<f32x4_v*>(a.part_o + (bh * a.nsplit + split) * kHeadDim + d) = s;
        else *reinterpret_cast<f32x4_v*>(a.out + bh * kHeadDim + d) = s * inv_l[hh];
    }
}

template <int NG, int LANES>
__device__ __forceinline__ void merge_shares(const CacheAttnArgs& a, int64_t block, f32x4_v* osum, float2* mlsum)
{
    const Joined j = join_shares<NG, LANES>(a.part_o, a.part_ml, a.nsplit, (int64_t)a.B * a.Hq, block, osum, mlsum);
    if (j.row >= 0) *reinterpret_cast<f32x4_v*>(a.out + j.row * kHeadDim + j.d) = j.o;
}

// S[b, r, j(i)] += the weights of the row's heads, 256 * SP positions per
// workgroup: the heads' (m, l) from the shares first, then each thread SP
// positions of every head, in head order.
template <int SP>
__device__ __forceinline__ void add_weights(const CacheAttnArgs& a, int64_t block, float2* red, float2* stat)
{
    const int tid = threadIdx.x;
    const int chunk = (int)(block % a.s_chunks);
    const int64_t row = block / a.s_chunks;
    const int b = (int)(row / a.R), r = (int)(row % a.R);
    const int heads = a.R > 1 ? a.G : a.Hq;
    const int64_t bh0 = (int64_t)b * a.Hq + (int64_t)r * a.G;
    const Visible vis = visible(seq_len(a.lens, b, a.n), a.sink, a.window);
    const int i = chunk * 256 * SP + SP * tid;
    if (chunk * 256 * SP >= vis.nv) return;              // the same for the whole workgroup
    const int tph = 256 / heads;                         // threads per head (heads <= 256)
    {
        const int hh = tid / tph, sub = tid % tph;
        float m = -INFINITY, l = 0.0f;
        if (hh < heads) {
            const float2* ml = a.part_ml + (bh0 + hh) * a.nsplit;
#pragma unroll 8
            for (int s = sub; s < a.nsplit; s += tph) {
                const float2 v = ml[s];
                if (v.y > 0.0f) {
                    const float M = fmaxf(m, v.x);
                    l = l * exp2_ftz(m - M) + v.y * exp2_ftz(v.x - M);
                    m = M;
                }
            }
        }
        red[tid] = make_float2(m, l);
    }
    __syncthreads();
    if (tid < heads) {
        float M = -INFINITY, L = 0.0f;
        for (int u = 0; u < tph; ++u) M = fmaxf(M, red[tid * tph + u].x);
        for (int u = 0; u < tph; ++u) {
            const float2 v = red[tid * tph + u];
            L += v.y > 0.0f ? v.y * exp2_ftz(v.x - M) : 0.0f;
        }
        // the shares' l carry the weights' factor; nothing but logits below fp32's range: weights 0
        stat[tid] = L > 0.0f ? make_float2(M - kWeightShift<0>, 1.0f / L) : make_float2(0.0f, 0.0f);
    }
    __syncthreads();
    if (i >= vis.nv) return;
    typedef float vec __attribute__((ext_vector_type(SP)));
    vec acc = 0.0f;
    const float* x = a.logits + bh0 * a.ld + i;
#pragma unroll 8
    for (int hh = 0; hh < heads; ++hh) {
        const vec v = *reinterpret_cast<const vec*>(x + (int64_t)hh * a.ld);
        const float2 st = stat[hh];
#pragma unroll
        for (int e = 0; e < SP; ++e) acc[e] += exp2_ftz(v[e] - st.x) * st.y;
    }
    float* s = a.s + (int64_t)b * a.s_sb + (int64_t)r * a.s_sr;
#pragma unroll
    for (int e = 0; e < SP; ++e)
        if (i + e < vis.nv) s[vis.token(i + e)] += acc[e];
}

// The first merge_blocks workgroups join shares, the others add weights.
template <int NG, int LANES, int SP>
__global__ __launch_bounds__(256, 4) void cache_merge_kernel(CacheAttnArgs a, int64_t merge_blocks)
{
    __shared__ f32x4_v buf[256 + 128];
    float2* two = reinterpret_cast<float2*>(buf + 256);
    if ((int64_t)blockIdx.x < merge_blocks) merge_shares<NG, LANES>(a, blockIdx.x, buf, two);
    else add_weights<SP>(a, (int64_t)blockIdx.x - merge_blocks, two, reinterpret_cast<float2*>(buf));
}

template <int KT>
void launch_rows(const CacheAttnArgs& a, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * a.head_tiles * a.nsplit));
    if constexpr (KT == kRowsPacked) {
        if (a.idx) hipLaunchKernelGGL((cache_attn_kernel<KT, true, false>), grid, dim3(256), 0, st, a);
        else if (a.s) hipLaunchKernelGGL((cache_attn_kernel<KT, false, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((cache_attn_kernel<KT, false, false>), grid, dim3(256), 0, st, a);
    } else {
        hipLaunchKernelGGL((cache_attn_kernel<KT, false, false>), grid, dim3(256), 0, st, a);
    }
}

// Few shares: eight heads a workgroup; more: one head, its shares over eight
// groups; many: a quarter of one.
template <int SP>
void launch_merge(const CacheAttnArgs& a, hipStream_t st)
{
    const int64_t bh = (int64_t)a.B * a.Hq;
    const int form = a.nsplit <= 8 ? 0 : a.nsplit <= 64 ? 1 : 2;
    const int64_t merge = a.nsplit <= 1 ? 0 : form == 0 ? (bh + 7) / 8 : form == 1 ? bh : 4 * bh;
    const int64_t add = a.s ? (int64_t)a.B * a.R * a.s_chunks : 0;
    if (merge + add == 0) return;
    const dim3 grid((unsigned)(merge + add));
    if (form == 0) hipLaunchKernelGGL((cache_merge_kernel<1, 32, SP>), grid, dim3(256), 0, st, a, merge);
    else if (form == 1) hipLaunchKernelGGL((cache_merge_kernel<8, 32, SP>), grid, dim3(256), 0, st, a, merge);
    else hipLaunchKernelGGL((cache_merge_kernel<32, 8, SP>), grid, dim3(256), 0, st, a, merge);
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnArgs& a, int dtype, hipStream_t st)
{
    if (a.kc) launch_rows<kRowsPacked>(a, st);
    else if (dtype == 1) launch_rows<kRowsBf16>(a, st);
    else launch_rows<kRowsF16>(a, st);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.s && a.s_per == 1) launch_merge<1>(a, st);
    else launch_merge<4>(a, st);
    return hipGetLastError();
}

}  // namespace hill
