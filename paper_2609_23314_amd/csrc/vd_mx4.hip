// Kernels of a KV cache held in 4 bits: append, read, attention, eviction.
//
// A row of D channels is D / 2 bytes of e2m1 codes (channel 2i in the low half
// of byte i) and D / 32 bytes of E8M0 scales, one power of two per 32 channels.
// gfx950 converts both ways (v_cvt_scalef32_pk_*_fp4); code times scale is exact
// in bf16, so that the matrix cores take a row's values without a rounding.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "vd.h"
#include "vd_mx4.h"

namespace vd {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T>
__device__ __forceinline__ uint32_t bits(T x) {
    return __builtin_bit_cast(uint32_t, x);
}
__device__ __forceinline__ float as_float(uint32_t x) { return __builtin_bit_cast(float, x); }

// The conversions' scale operand for an E8M0 byte: they read its exponent
// alone, 0 as 2^-127 and 255 as NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) { return as_float(byte << 23); }

template <int SEL>
__device__ __forceinline__ bf16x2 decode2(uint32_t codes, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL);
}
// Eight values of four bytes of codes.
__device__ __forceinline__ bf16x8 decode8(uint32_t codes, float scale) {
    const u32x4 r = {bits(decode2<0>(codes, scale)), bits(decode2<1>(codes, scale)), bits(decode2<2>(codes, scale)),
                     bits(decode2<3>(codes, scale))};
    return __builtin_bit_cast(bf16x8, r);
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E;   // quad_perm

// ---------------------------------------------------------------- append and read
//
// Eight channels a lane, the four lanes of a quad a group: the group's largest
// magnitude is two exchanges in the quad away.  Bandwidth bounds both (512 rows of 256
// units, bf16 in and out, K and V: append 18.5 us, 4.6 TB/s; read 16.6, 5.1 TB/s).

// E8M0 byte of a group: the least exponent e >= -127 with max < 7 * 2^e, so
// that the largest value rounds to at most 6 (code 7) and no value is cut by more
// than its rounding; at most 125, where 6 * 2^e is still finite.  Anything not
// finite makes the group NaN.
__device__ __forceinline__ uint32_t group_scale(uint32_t max_bits) {
    const int e = int(max_bits >> 23) - 2 + int((max_bits & 0x7FFFFFu) >= 0x600000u);
    return max_bits >= 0x7F800000u ? 255u : uint32_t(min(max(e, 0), 252));
}

template <int DTYPE, int D>
__global__ __launch_bounds__(kMxThreads) void append_kernel(const MxRowsParams p) {
    constexpr int LANES = D / 8;
    const uint32_t at = blockIdx.x * kMxThreads + threadIdx.x;
    const int lane = at % LANES;
    const uint32_t item = at / LANES;
    const int row = int(item % uint32_t(p.max_rows)), unit = int(item / uint32_t(p.max_rows));
    const bool is_v = blockIdx.y & 1;
    const int s = blockIdx.y >> 1;
    if (unit >= p.c.layers * p.c.heads || row >= p.rows[s]) return;   // (a row's lanes leave together)
    const int layer = unit / p.c.heads, head = unit % p.c.heads;
    const char *src = (is_v ? p.v + s * p.vs[0] + layer * p.vs[1] + head * p.vs[2] + row * p.vs[3]
                            : p.k + s * p.ks[0] + layer * p.ks[1] + head * p.ks[2] + row * p.ks[3]);
    uint32_t x[8];
    if (DTYPE == VD_DTYPE_F32) {
        const u32x4 u = reinterpret_cast<const u32x4 *>(src)[2 * lane], w = reinterpret_cast<const u32x4 *>(src)[2 * lane + 1];
        for (int i = 0; i < 4; ++i) x[i] = u[i], x[4 + i] = w[i];
    } else {
        const u32x4 u = reinterpret_cast<const u32x4 *>(src)[lane];
        for (int i = 0; i < 4; ++i) x[2 * i] = u[i] << 16, x[2 * i + 1] = u[i] & 0xFFFF0000u;
    }
    uint32_t top = 0;
    for (int i = 0; i < 8; ++i) top = max(top, x[i] & 0x7FFFFFFFu);
    top = max(top, dpp<kXor1>(top));
    top = max(top, dpp<kXor2>(top));
    const uint32_t byte = group_scale(top);
    const float scale = scale_of(byte);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, as_float(x[0]), as_float(x[1]), scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, as_float(x[2]), as_float(x[3]), scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, as_float(x[4]), as_float(x[5]), scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, as_float(x[6]), as_float(x[7]), scale, 3);
    if (byte == 255u) codes = 0;
    const int slot = p.first[s] + row;
    char *dst = (is_v ? p.c.v : p.c.k) + s * p.c.seq + layer * p.c.layer + head * p.c.head + uint32_t(slot) * p.c.slot;
    char *sdst = (is_v ? p.c.vs : p.c.ks) + s * p.c.sseq + layer * p.c.slayer + head * p.c.shead + uint32_t(slot) * p.c.sslot;
    reinterpret_cast<uint32_t *>(dst)[lane] = codes;
    if ((lane & 3) == 0) sdst[lane >> 2] = char(byte);
    if (p.pos && !is_v && lane == 0)
        p.pos[(int64_t(s) * p.c.layers * p.c.heads + unit) * p.capacity + slot] = p.pos0[s] + row;
}

template <int DTYPE, int D>
__global__ __launch_bounds__(kMxThreads) void read_kernel(const MxRowsParams p) {
    constexpr int LANES = D / 8;
    const uint32_t at = blockIdx.x * kMxThreads + threadIdx.x;
    const int lane = at % LANES;
    const uint32_t item = at / LANES;
    const int row = int(item % uint32_t(p.max_rows)), unit = int(item / uint32_t(p.max_rows));
    const bool is_v = blockIdx.y & 1;
    const int s = blockIdx.y >> 1;
    if (unit >= p.c.layers * p.c.heads || row >= p.rows[s]) return;
    const int layer = unit / p.c.heads, head = unit % p.c.heads;
    const uint32_t slot = uint32_t(p.first[s] + row);
    const char *src = (is_v ? p.c.v : p.c.k) + s * p.c.seq + layer * p.c.layer + head * p.c.head + slot * p.c.slot;
    const char *ssrc = (is_v ? p.c.vs : p.c.ks) + s * p.c.sseq + layer * p.c.slayer + head * p.c.shead + slot * p.c.sslot;
    const uint32_t codes = reinterpret_cast<const uint32_t *>(src)[lane];
    const float scale = scale_of(uint8_t(ssrc[lane >> 2]));
    char *dst = (is_v ? p.v + s * p.vs[0] + layer * p.vs[1] + head * p.vs[2] + row * p.vs[3]
                      : p.k + s * p.ks[0] + layer * p.ks[1] + head * p.ks[2] + row * p.ks[3]);
    if (DTYPE == VD_DTYPE_F32) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
        const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
        const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
        reinterpret_cast<f32x4 *>(dst)[2 * lane] = f32x4{a[0], a[1], b[0], b[1]};
        reinterpret_cast<f32x4 *>(dst)[2 * lane + 1] = f32x4{c[0], c[1], d[0], d[1]};
    } else {
        reinterpret_cast<bf16x8 *>(dst)[lane] = decode8(codes, scale);
    }
}

// ---------------------------------------------------------------- attention
//
// out_i = sum_j w_ij v_j, w_ij = exp(scale q_i.k_j - m_i) / sum, over the slots
// j < n - rows + 1 + i that query row i sees.  The G query heads of a KV head
// share its rows, so a tile's 16 query rows are m = i * G + g.
//
// A wave takes 32 cache rows at a time.  A lane reads a quarter of a row's codes
// (16 bytes at D = 128: one whole group, one scale) and converts them into the
// left operand of v_mfma_f32_16x16x32_bf16, whose sum over channels may take them
// in any order: here the quarter's eight by eight.  Its output has a lane hold one
// query's logits for 4 rows of 16, which is, for 32 rows, just the right operand of
// the product with V^T: weights never leave their lane.  V's rows are converted
// the same way, and turned in LDS: written by row, read by ds_read_b64_tr_b16.
//
// fp32 queries are three bf16 parts (exact), their weights two (2^-16 of a weight);
// bf16 queries take one part each (a weight's rounding is 2^-8 of it, as the
// output's; the sum of the weights is that of the rounded ones, so that a row with
// one weight is exact).  Sums, logits and the softmax are fp32.
//
// A row with a NaN group, in K or in V, makes NaN of the outputs that see it and
// only those: its K scale becomes NaN, and V's stays finite.
//
// Single tokens are bound by the conversions, the softmax and, for fp32 queries, the
// parts' products as much as by memory: 4096 units of 4097 rows, four fp32 queries
// each, 2.28 GB in 0.44 ms (5.2 TB/s); 8 units of 131072 rows, eight bf16 queries, 143
// MB in 24.9 us (5.7 TB/s) and 4.0 for the join.

template <int D>
struct Quarter {   // a lane's part of a row: D / 4 channels
    static constexpr int WORDS = D / 32;
    uint32_t w[WORDS];
};
template <int D>
__device__ __forceinline__ Quarter<D> load_quarter(const char *row, int kq) {
    Quarter<D> r;
    if (D == 64) {
        const u32x2 x = reinterpret_cast<const u32x2 *>(row)[kq];
        r.w[0] = x[0], r.w[1] = x[1];
    } else {
        for (int i = 0; i < D / 128; ++i) {
            const u32x4 x = reinterpret_cast<const u32x4 *>(row)[kq * (D / 128) + i];
            for (int e = 0; e < 4; ++e) r.w[(4 * i + e) % (D / 32)] = x[e];
        }
    }
    return r;
}
// All scales of a row.
template <int D>
struct Scales {
    static constexpr int WORDS = D == 256 ? 2 : 1;
    uint32_t w[WORDS];
    __device__ __forceinline__ uint32_t byte(int group) const {
        const uint32_t x = WORDS == 2 && group >= 4 ? w[WORDS - 1] : w[0];
        return (x >> (8 * (group & 3))) & 255u;
    }
    // 255 if any of the row's groups is NaN, else 0
    __device__ __forceinline__ uint32_t nan_bits() const {
        uint32_t nan = 0;
        for (int i = 0; i < WORDS; ++i) nan |= (~w[i] - 0x01010101u) & w[i] & 0x80808080u;   // a zero byte of ~w
        return nan ? 255u : 0u;
    }
};
template <int D>
__device__ __forceinline__ Scales<D> load_scales(const char *row) {
    Scales<D> r;
    if (D == 64) {
        r.w[0] = *reinterpret_cast<const uint16_t *>(row);
    } else if (D == 128) {
        r.w[0] = *reinterpret_cast<const uint32_t *>(row);
    } else {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(row);
        r.w[0] = x[0], r.w[Scales<D>::WORDS - 1] = x[1];
    }
    return r;
}

// Eight channels of a query row, in parts; `flip` turns their signs (a negative
// softmax scale, so that a larger product is always a larger logit).
template <int DTYPE, int QP, int FRAGS>
__device__ __forceinline__ void load_query(bf16x8 (&q)[QP][FRAGS], int f, const char *row, int ch, uint32_t flip) {
    if (DTYPE == VD_DTYPE_BF16) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(row + ch * 2);
        const uint32_t both = flip | flip >> 16;
        q[0][f] = __builtin_bit_cast(bf16x8, x ^ both);
        return;
    }
    const f32x4 a = *reinterpret_cast<const f32x4 *>(row + ch * 4), b = *reinterpret_cast<const f32x4 *>(row + ch * 4 + 16);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float x = as_float(bits(e < 4 ? a[e & 3] : b[e & 3]) ^ flip);
#pragma unroll
        for (int part = 0; part < QP; ++part) {
            q[part][f][e] = __bf16(x);
            x -= float(q[part][f][e]);
        }
    }
}

// Bytes of a row of one wave's V tile (32 rows of bf16): 32 bytes apart from a
// multiple of the banks, so that the turned reads do not collide.
template <int D>
constexpr int kVStride = D * 2 + 32;

template <int D>
constexpr int attn_lds() {
    const int tiles = 4 * 32 * kVStride<D>, merge = 4 * kMxTile * (D + 4) * 4 + 4 * kMxTile * 2 * 4;
    return tiles > merge ? tiles : merge;
}

template <int DTYPE, int D>
__global__ __launch_bounds__(kMxThreads) void attn_kernel(const MxAttnParams p) {
    constexpr int FRAGS = D / 32;                                // products over the channels of one logit tile
    constexpr int QP = DTYPE == VD_DTYPE_F32 ? 3 : 1;            // parts of a query
    constexpr int PP = DTYPE == VD_DTYPE_F32 ? 2 : 1;            // parts of a weight
    constexpr int CT = D / 16;                                   // channel tiles of the output
    __shared__ __attribute__((aligned(16))) char lds[attn_lds<D>()];
    const int split = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles;
    const int head = blockIdx.y, s = blockIdx.z / p.c.layers, layer = blockIdx.z % p.c.layers;
    const int n = p.n[s], rows = p.rows[s], G = p.group;
    const int queries = rows * G, m0 = tile * kMxTile;
    if (m0 >= queries) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, kq = lane >> 4;
    // the cache rows that any query of the tile sees, and this split's share of them
    const int seen = max(0, n - rows + 1 + min(m0 + kMxTile - 1, queries - 1) / G);
    const int share = ((seen + p.splits - 1) / p.splits + 127) & ~127;
    const int begin = min(split * share, seen), end = min(begin + share, seen);
    const int all_see = n - rows + 1 + m0 / G;                   // rows below this need no mask
    const int m = m0 + c, i = min(m, queries - 1) / G, g = min(m, queries - 1) - i * G;
    const int limit = n - rows + 1 + i;

    bf16x8 q[QP][FRAGS];   // the right operand: channels kq * D / 4 + 8 f + e of query c
    {
        const char *src = p.q + s * p.qs[0] + layer * p.qs[1] + (head * G + g) * p.qs[2] + i * p.qs[3];
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) load_query<DTYPE, QP>(q, f, src, kq * (D / 4) + 8 * f, p.flip);
    }

    const char *kb = p.c.k + s * p.c.seq + layer * p.c.layer + head * p.c.head;
    const char *vb = p.c.v + s * p.c.seq + layer * p.c.layer + head * p.c.head;
    const char *ksb = p.c.ks + s * p.c.sseq + layer * p.c.slayer + head * p.c.shead;
    const char *vsb = p.c.vs + s * p.c.sseq + layer * p.c.slayer + head * p.c.shead;
    char *tile_lds = lds + wave * 32 * kVStride<D>;

    f32x4 acc[CT + 1];   // the last: sum of the weights (a column of ones beside V)
#pragma unroll
    for (int t = 0; t <= CT; ++t) acc[t] = f32x4{0, 0, 0, 0};
    const uint32_t one2 = 0x3F803F80u;
    const bf16x8 ones = __builtin_bit_cast(bf16x8, (u32x4{one2, one2, one2, one2}));
    float top = -INFINITY, sub = 0.0f;   // the maximum that the weights are relative to

    Quarter<D> kc[2], vc[2];
    Scales<D> ks[2], vs[2];
    auto load = [&](int j0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {   // rows behind the end: the last row again, hidden below
            const uint32_t row = uint32_t(min(j0 + 16 * t + c, end - 1));
            kc[t] = load_quarter<D>(kb + row * p.c.slot, kq);
            ks[t] = load_scales<D>(ksb + row * p.c.sslot);
            vc[t] = load_quarter<D>(vb + row * p.c.slot, kq);
            vs[t] = load_scales<D>(vsb + row * p.c.sslot);
        }
    };
    if (begin + 32 * wave < end) load(begin + 32 * wave);
    for (int j0 = begin + 32 * wave; j0 < end; j0 += 128) {
        f32x4 z[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t nan = ks[t].nan_bits() | vs[t].nan_bits();
            z[t] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int f = 0; f < FRAGS; ++f) {
                const int group = (kq * (D / 4) + 8 * f) / kMxGroup;
                const float scale = scale_of(ks[t].byte(group) | nan);
                const bf16x8 a = decode8(kc[t].w[f], scale);
#pragma unroll
                for (int part = QP - 1; part >= 0; --part)
                    z[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[part][f], z[t], 0, 0, 0);
                const uint32_t vbyte = vs[t].byte(group);
                const float vscale = scale_of(vbyte == 255u ? 0u : vbyte);
                *reinterpret_cast<bf16x8 *>(tile_lds + (16 * t + c) * kVStride<D> + (kq * (D / 4) + 8 * f) * 2) = decode8(vc[t].w[f], vscale);
            }
        }
        load(j0 + 128);   // on its way while this one's weights are made (behind the end: not used)
        // lane: query c, rows j0 + 16 t + 4 kq + r
        if (j0 + 32 > min(all_see, end)) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) z[t][r] = j0 + 16 * t + 4 * kq + r < min(limit, end) ? z[t][r] : -INFINITY;
        }
        float best = z[0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) best = fmaxf(best, z[e >> 2][e & 3]);
        best *= p.qscale;
        // The weights are relative to a maximum that is raised only when a logit
        // passes it by 8 (log2 units): they stay below 2^8, and mostly no sum is rescaled.
        if (__builtin_amdgcn_ballot_w64(best > top + 8.0f)) {
            best = fmaxf(best, __shfl_xor(best, 16));
            best = fmaxf(best, __shfl_xor(best, 32));
            const float next = fmaxf(top, best);
            const float down = __builtin_amdgcn_exp2f(top - (next == -INFINITY ? 0.0f : next));
            top = next;
            sub = next == -INFINITY ? 0.0f : next;
#pragma unroll
            for (int t = 0; t <= CT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[t][r] *= down;
        }
        bf16x8 w[PP];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float x = __builtin_amdgcn_exp2f(fmaf(z[e >> 2][e & 3], p.qscale, -sub));
#pragma unroll
            for (int part = 0; part < PP; ++part) {
                w[part][e] = __bf16(x);
                x -= float(w[part][e]);
            }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            typedef __attribute__((address_space(3))) s16x4 *lds4;
            const char *at = tile_lds + (4 * kq + (c >> 2)) * kVStride<D> + ct * 32 + (c & 3) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 16 * kVStride<D>));
            const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int part = PP - 1; part >= 0; --part)
                acc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[part], acc[ct], 0, 0, 0);
        }
#pragma unroll
        for (int part = PP - 1; part >= 0; --part)
            acc[CT] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, w[part], acc[CT], 0, 0, 0);
    }

    // the four waves' sums
    __syncthreads();
    float *part = reinterpret_cast<float *>(lds);                         // [wave][query][D + 4]
    float *ml = part + 4 * kMxTile * (D + 4);                             // [wave][query][2]
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
        *reinterpret_cast<f32x4 *>(part + (wave * kMxTile + c) * (D + 4) + 16 * ct + 4 * kq) = acc[ct];
    if (kq == 0) {
        ml[(wave * kMxTile + c) * 2] = top;
        ml[(wave * kMxTile + c) * 2 + 1] = acc[CT][0];
    }
    __syncthreads();
    const int count = min(kMxTile, queries - m0);
    const int64_t unit = (int64_t(s) * p.c.layers + layer) * p.c.heads + head;
    const int64_t all = int64_t(p.max_rows) * G;
    for (int at = threadIdx.x; at < count * (D / 4); at += kMxThreads) {
        const int query = at / (D / 4), ch = at % (D / 4) * 4;
        float tops[4], high = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) high = fmaxf(high, tops[w] = ml[(w * kMxTile + query) * 2]);
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            // (a wave without a finite logit has no weights, or only NaN ones)
            const float f = tops[w] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(tops[w] - high);
            const f32x4 x = *reinterpret_cast<const f32x4 *>(part + (w * kMxTile + query) * (D + 4) + ch);
            sum = fmaf(ml[(w * kMxTile + query) * 2 + 1], f, sum);
            for (int e = 0; e < 4; ++e) o[e] = fmaf(x[e], f, o[e]);
        }
        if (p.splits > 1) {
            const int64_t to = (unit * p.splits + split) * all + m0 + query;
            *reinterpret_cast<f32x4 *>(p.ws_acc + to * D + ch) = o;
            if (ch == 0) p.ws_ml[to * 2] = high, p.ws_ml[to * 2 + 1] = sum;
            continue;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;     // no row seen: 0
        const int qi = (m0 + query) / G, qg = (m0 + query) - qi * G;
        char *dst = p.out + s * p.os[0] + layer * p.os[1] + (head * G + qg) * p.os[2] + qi * p.os[3];
        if (DTYPE == VD_DTYPE_F32) {
            *reinterpret_cast<f32x4 *>(dst + ch * 4) = o * inv;
        } else {
            bf16x4 b;
            for (int e = 0; e < 4; ++e) b[e] = __bf16(o[e] * inv);
            *reinterpret_cast<bf16x4 *>(dst + ch * 2) = b;
        }
    }
}

// Blocks of query rows.  A workgroup takes 128 query rows of a KV head, a wave 32
// of them, and passes over the cache 64 rows at a time: the four waves bring a tile of
// K and V into LDS, while they work on the tile before.  As above, transposed: a lane
// holds one query's logits of 16 rows of 32, which are the right operand of the
// product with V^T (v_mfma_f32_32x32x16_bf16).
//
// K of bf16 queries stays in 4 bits: v_mfma_scale_f32_32x32x64_f8f6f4 takes its codes
// and scales as they are.  A query is two e4m3 parts with a power of two for each 32
// channels: eight significant bits, exact but for what is below 2^-21 of the largest
// of its 32.  That takes the matrix cores the time of the bf16 product, but neither a
// conversion nor more than a quarter of the LDS reads.  (V's scales belong to rows,
// along which its product sums: it is converted.)  fp32 queries meet K in bf16.
//
// Arithmetic and products bound it together, since a SIMD hardly runs the one beside the
// other (a loop of 32x32x16 products alone takes 37 cycles each, with 7 fused multiplies
// beside each 60, the multiplies alone 34): 32 layers x 8 KV heads, 512 rows of 4 heads
// over 2560, D = 128, 0.62 TFLOP in 0.60 ms, 1030 TFLOP/s; 777 rows of 2 heads over up
// to 4873, D = 256, 0.19 ms, 700.  With K in bf16 as well 0.65 and 0.27 ms; with V's
// tile padded rather than swizzled, and K's by 32 bytes, 5 % more.

constexpr int kBlockRows = 64;
template <int DTYPE, int D>
struct KTile {   // K in LDS; sixteen rows' 16-byte reads fall into different banks
    static constexpr bool CODES = DTYPE == VD_DTYPE_BF16;
    static constexpr int STRIDE = (CODES ? D / 2 : D * 2) + 16;
    static constexpr int SCALE = D == 256 ? 8 : 4;                                  // bytes of a row's scales
    static constexpr int BYTES = kBlockRows * (STRIDE + (CODES ? SCALE : 0));       // (behind all rows)
};

// V's tile has no padding: where four rows are read together 64 bytes wide, and
// sixteen lanes write 16 bytes each, both meet every bank once if a row's 64-byte
// units and their 16-byte pieces change places with the row.
template <int D>
__device__ __forceinline__ int v_place(int row, int unit, int piece) {
    const int u = D == 64 ? (row >> 1) & 1 : row & 3, c = D == 64 ? (row >> 1) & 3 : row & 3;
    return row * (D * 2) + ((unit ^ u) * 64) + ((piece ^ c) * 16);
}

// A thread's part of a tile on its way from memory: groups of K, then groups of V
// (of D = 64 one group of either).
template <int DTYPE, int D>
struct BlockStage {
    static constexpr int GROUPS = D / 32, ROWS = kBlockRows, ITEMS = 2 * ROWS * GROUPS / kMxThreads, K_ITEMS = (ITEMS + 1) / 2;
    u32x4 x[ITEMS];
    Scales<D> ks[K_ITEMS], vs[K_ITEMS];   // of the whole row, whose NaN groups K's items look for
    uint32_t vbyte[ITEMS];                // of V's items
    __device__ __forceinline__ static bool is_v(int i) { return ITEMS == 1 ? int(threadIdx.x) >= ROWS * GROUPS : i >= K_ITEMS; }
    __device__ __forceinline__ static int at(int i) { return (int(threadIdx.x) + i * kMxThreads) % (ROWS * GROUPS); }
    // K's items of the tile at jk, V's of the one at jv
    __device__ __forceinline__ void load(const char *kb, const char *vb, const char *ksb, const char *vsb, uint32_t slot,
                                         uint32_t sslot, int jk, int jv, int end) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t row = uint32_t(min((is_v(i) ? jv : jk) + at(i) / GROUPS, end - 1));   // behind the end: the last row, hidden later
            x[i] = reinterpret_cast<const u32x4 *>((is_v(i) ? vb : kb) + row * slot)[at(i) % GROUPS];
            if (i < K_ITEMS) {
                ks[i % K_ITEMS] = load_scales<D>(ksb + row * sslot);
                vs[i % K_ITEMS] = load_scales<D>(vsb + row * sslot);
            } else {
                vbyte[i] = uint8_t(vsb[row * sslot + at(i) % GROUPS]);
            }
        }
    }
    __device__ __forceinline__ void store(int i, char *kt, char *vt) const {
        using Tile = KTile<DTYPE, D>;
        const int row = at(i) / GROUPS, group = at(i) % GROUPS;
        if (is_v(i)) {
            const uint32_t own = i < K_ITEMS ? vs[i % K_ITEMS].byte(group) : vbyte[i], byte = own == 255u ? 0u : own;
#pragma unroll
            for (int w = 0; w < 4; ++w) *reinterpret_cast<bf16x8 *>(vt + v_place<D>(row, group, w)) = decode8(x[i][w], scale_of(byte));
            return;
        }
        const uint32_t nan = ks[i % K_ITEMS].nan_bits() | vs[i % K_ITEMS].nan_bits();
        if (Tile::CODES) {
            *reinterpret_cast<u32x4 *>(kt + row * Tile::STRIDE + group * 16) = x[i];
            kt[kBlockRows * Tile::STRIDE + row * Tile::SCALE + group] = char(ks[i % K_ITEMS].byte(group) | nan);
            return;
        }
        const uint32_t byte = ks[i % K_ITEMS].byte(group) | nan;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            *reinterpret_cast<bf16x8 *>(kt + row * Tile::STRIDE + group * 64 + 16 * w) = decode8(x[i][w], scale_of(byte));
    }
};

__device__ __forceinline__ float dot2(bf16x2 a, bf16x2 b, float c) { return __builtin_amdgcn_fdot2_f32_bf16(a, b, c, false); }
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// A wave's 32 queries as right operands, and their logits with a tile of K: a lane
// has query c = lane & 31, rows 32 t + 8 (r / 4) + 4 half + r % 4.
template <int DTYPE, int D>
struct BlockQueries {   // fp32: three bf16 parts, channels 16 f + 8 half + e
    static constexpr int FRAGS = D / 16, QP = 3, PRODUCTS = FRAGS * QP;
    bf16x8 q[QP][FRAGS];
    __device__ __forceinline__ void load(const char *src, int half, uint32_t flip) {
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) load_query<DTYPE, QP>(q, f, src, 16 * f + 8 * half, flip);
    }
    __device__ __forceinline__ f32x16 logits(const char *kt, int t, int c, int half) const {
        f32x16 z = {};
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) {
            const bf16x8 a = *reinterpret_cast<const bf16x8 *>(kt + (32 * t + c) * KTile<DTYPE, D>::STRIDE + (16 * f + 8 * half) * 2);
#pragma unroll
            for (int part = QP - 1; part >= 0; --part) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[part][f], z, 0, 0, 0);
        }
        return z;
    }
};

// The product of 64 channels: codes and their scale (byte BYTE of ka), e4m3 values and theirs.
template <int BYTE, int PART>
__device__ __forceinline__ f32x16 mx_product(const u32x4 &k, uint32_t ks, const i32x8 &q, uint32_t qs, const f32x16 &z) {
    const i32x8 a = {int(k[0]), int(k[1]), int(k[2]), int(k[3]), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q, z, 4, 0, BYTE, int(ks), BYTE + PART, int(qs));
}

template <int D>
struct BlockQueries<VD_DTYPE_BF16, D> {
    // For 64 channels the left operand has a half's lanes hold 32 neighbouring ones (a
    // group), the right one 16 of the first 32 and 16 of the second; scales are a half's own.
    static constexpr int FRAGS = D / 64, PRODUCTS = FRAGS * 2;
    i32x8 high[FRAGS], low[FRAGS];
    uint32_t scale[(FRAGS + 1) / 2];   // bytes: of high and low of an even f, then of an odd one
    __device__ __forceinline__ void load(const char *src, int half, uint32_t flip) {
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) {
            uint32_t byte[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                u32x4 x[2];
#pragma unroll
                for (int w = 0; w < 2; ++w)
                    x[w] = *reinterpret_cast<const u32x4 *>(src + (64 * f + 32 * b + 16 * half + 8 * w) * 2) ^ (flip | flip >> 16);
                uint32_t most = 0;
#pragma unroll
                for (int w = 0; w < 8; ++w) most = max(most, max(x[w >> 2][w & 3] & 0x7FFF0000u, x[w >> 2][w & 3] << 16 & 0x7FFF0000u));
                most = max(most, uint32_t(__shfl_xor(int(most), 32)));
                // 2^(byte - 127): the largest becomes 128 .. 256, e4m3 ends at 448
                byte[b] = uint32_t(max(int(most >> 23) - 7, 4));
                const float to = as_float((254u - byte[b]) << 23);
#pragma unroll
                for (int w = 0; w < 4; ++w) {   // four channels
                    const uint32_t u = x[w >> 1][2 * (w & 1)], v = x[w >> 1][2 * (w & 1) + 1];
                    const float y[4] = {as_float(u << 16) * to, as_float(u & 0xFFFF0000u) * to, as_float(v << 16) * to,
                                        as_float(v & 0xFFFF0000u) * to};
                    int h = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
                    h = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], h, true);
                    const float r0 = y[0] - __builtin_amdgcn_cvt_f32_fp8(h, 0), r1 = y[1] - __builtin_amdgcn_cvt_f32_fp8(h, 1);
                    const float r2 = y[2] - __builtin_amdgcn_cvt_f32_fp8(h, 2), r3 = y[3] - __builtin_amdgcn_cvt_f32_fp8(h, 3);
                    int l = __builtin_amdgcn_cvt_pk_fp8_f32(r0 * 16.0f, r1 * 16.0f, 0, false);
                    l = __builtin_amdgcn_cvt_pk_fp8_f32(r2 * 16.0f, r3 * 16.0f, l, true);
                    high[f][4 * b + w] = h;
                    low[f][4 * b + w] = l;
                }
            }
            const uint32_t own = half ? byte[1] : byte[0], both = own | (own - 4) << 8;
            scale[f / 2] = f % 2 ? scale[f / 2] | both << 16 : both;
        }
    }
    __device__ __forceinline__ f32x16 logits(const char *kt, int t, int c, int half) const {
        using Tile = KTile<VD_DTYPE_BF16, D>;
        const char *row = kt + (32 * t + c) * Tile::STRIDE + 16 * half;
        const uint32_t *scales = reinterpret_cast<const uint32_t *>(kt + kBlockRows * Tile::STRIDE + (32 * t + c) * Tile::SCALE);
        f32x16 z = {};
#pragma unroll
        for (int f = 0; f < FRAGS; f += 2) {
            const uint32_t ks = scales[f / 2] >> (8 * half);
            const u32x4 k = *reinterpret_cast<const u32x4 *>(row + 32 * f);
            z = mx_product<0, 1>(k, ks, low[f], scale[f / 2], z);
            z = mx_product<0, 0>(k, ks, high[f], scale[f / 2], z);
            if (FRAGS > 1) {
                const u32x4 next = *reinterpret_cast<const u32x4 *>(row + 32 * (f + 1));
                z = mx_product<2, 1>(next, ks, low[(f + 1) % FRAGS], scale[f / 2], z);
                z = mx_product<2, 0>(next, ks, high[(f + 1) % FRAGS], scale[f / 2], z);
            }
        }
        return z;
    }
};

template <int DTYPE, int D>
__global__ __launch_bounds__(kMxThreads, block_groups(DTYPE, D)) void attn_block_kernel(const MxAttnParams p) {
    constexpr int CT = D / 32, SUBS = kBlockRows / 32, PP = DTYPE == VD_DTYPE_F32 ? 2 : 1;
    constexpr int T = kBlockRows, KT = KTile<DTYPE, D>::BYTES, VT = T * D * 2, STEPS = SUBS * 2;
    __shared__ __attribute__((aligned(16))) char lds[2 * (KT + VT)];
    const int split = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles;
    const int head = blockIdx.y, s = blockIdx.z / p.c.layers, layer = blockIdx.z % p.c.layers;
    const int n = p.n[s], rows = p.rows[s], G = p.group;
    const int queries = rows * G, m0 = tile * kMxBlockTile;
    if (m0 >= queries) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
    const int seen = max(0, n - rows + 1 + min(m0 + kMxBlockTile - 1, queries - 1) / G);
    const int share = ((seen + p.splits - 1) / p.splits + T - 1) / T * T;
    const int begin = min(split * share, seen), end = min(begin + share, seen);
    const int wm0 = m0 + 32 * wave, m = wm0 + c;
    const int i = min(m, queries - 1) / G, g = min(m, queries - 1) - i * G;
    const int limit = min(n - rows + 1 + i, end);
    const int all_see = min(n - rows + 1 + min(wm0, queries - 1) / G, end);   // rows that every query of the wave sees

    BlockQueries<DTYPE, D> query;
    query.load(p.q + s * p.qs[0] + layer * p.qs[1] + (head * G + g) * p.qs[2] + i * p.qs[3], half, p.flip);
    const char *kb = p.c.k + s * p.c.seq + layer * p.c.layer + head * p.c.head;
    const char *vb = p.c.v + s * p.c.seq + layer * p.c.layer + head * p.c.head;
    const char *ksb = p.c.ks + s * p.c.sseq + layer * p.c.slayer + head * p.c.shead;
    const char *vsb = p.c.vs + s * p.c.sseq + layer * p.c.slayer + head * p.c.shead;

    f32x16 acc[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] = 0.0f;
    float top = -INFINITY, sub = 0.0f, sum = 0.0f;   // (the sum of the lane's rows)
    const bf16x2 ones = {__bf16(1.0f), __bf16(1.0f)};

    // where the lane's turned reads of V start (the rows of a tile that differ by 8 have their places alike)
    int v_at[CT < 4 ? CT : 4];
#pragma unroll
    for (int ct = 0; ct < (CT < 4 ? CT : 4); ++ct)
        v_at[ct] = v_place<D>(4 * half + ((lane & 15) >> 2), ct, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + (lane & 1) * 8;

    // weights of sixteen rows: the right operand of the product with V
    auto weights = [&](bf16x8 (&w)[PP], const f32x16 &z, int k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float x = __builtin_amdgcn_exp2f(fmaf(z[8 * k + e], p.qscale, -sub));
#pragma unroll
            for (int part = 0; part < PP; ++part) {
                w[part][e] = __bf16(x);
                x -= float(w[part][e]);
            }
        }
#pragma unroll
        for (int part = 0; part < PP; ++part) {
            sum = dot2(__builtin_shufflevector(w[part], w[part], 0, 1), ones, sum);
            sum = dot2(__builtin_shufflevector(w[part], w[part], 2, 3), ones, sum);
            sum = dot2(__builtin_shufflevector(w[part], w[part], 4, 5), ones, sum);
            sum = dot2(__builtin_shufflevector(w[part], w[part], 6, 7), ones, sum);
        }
    };
    auto read_values = [&](bf16x8 (&a)[CT], const char *vt, int step) {   // sixteen rows of V, turned
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            typedef __attribute__((address_space(3))) s16x4 *lds4;
            const char *at = vt + v_at[ct & 3] + (ct >> 2) * 256 + step * 16 * (D * 2);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 8 * (D * 2)));
            a[ct] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };
    constexpr int ITEMS = BlockStage<DTYPE, D>::ITEMS;
    char *k_lds = lds, *v_lds = lds + 2 * KT;
    BlockStage<DTYPE, D> stage;
    if (begin < end) {
        stage.load(kb, vb, ksb, vsb, p.c.slot, p.c.sslot, begin, begin, end);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) stage.store(i, k_lds, v_lds);
    }
    __syncthreads();
    int buffer = 0;
    for (int j0 = begin; j0 < end; j0 += T, buffer ^= 1) {
        stage.load(kb, vb, ksb, vsb, p.c.slot, p.c.sslot, j0 + T, j0 + T, end);   // (behind the last tile: not used)
        const char *vt = v_lds + buffer * VT;
        f32x16 now[SUBS];
#pragma unroll
        for (int t = 0; t < SUBS; ++t) now[t] = query.logits(k_lds + buffer * KT, t, c, half);
        if (D == 256) __builtin_amdgcn_sched_barrier(0);   // (the wide case 205 -> 192 us; of 128 channels 602 -> 610)
        bf16x8 va[2][CT], w[2][PP];
        read_values(va[0], vt, 0);
        // the next tile's loads first, and the matrix cores' operands read well ahead of the products
        __builtin_amdgcn_sched_group_barrier(0x020, 16, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
        for (int i = 0; i < SUBS * BlockQueries<DTYPE, D>::FRAGS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, BlockQueries<DTYPE, D>::PRODUCTS / BlockQueries<DTYPE, D>::FRAGS, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        if (j0 + T > all_see) {
#pragma unroll
            for (int t = 0; t < SUBS; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    now[t][r] = j0 + 32 * t + 8 * (r >> 2) + 4 * half + (r & 3) < limit ? now[t][r] : -INFINITY;
        }
        float best = now[0][0];
#pragma unroll
        for (int e = 1; e < 16 * SUBS; ++e) best = fmaxf(best, now[e >> 4][e & 15]);
        best *= p.qscale;
        if (__builtin_amdgcn_ballot_w64(best > top + 8.0f)) {   // (as above)
            best = fmaxf(best, __shfl_xor(best, 32));
            const float next = fmaxf(top, best);
            const float to = next == -INFINITY ? 0.0f : next;
            const float down = __builtin_amdgcn_exp2f(top - to);
            top = next;
            sub = to;
            sum *= down;
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[t][r] *= down;
        }
        // Sixteen rows at a time: the products with V stand between the arithmetic of the
        // next sixteen rows' weights, or, at the end, of the next tile's conversion.
        weights(w[0], now[0], 0);
        __builtin_amdgcn_s_setprio(1);   // before the other workgroup's logits (613 -> 602 us)
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
            __builtin_amdgcn_sched_barrier(0);
            if (step + 1 < STEPS) {
                read_values(va[(step + 1) & 1], vt, step + 1);
                weights(w[(step + 1) & 1], now[(step + 1) >> 1], (step + 1) & 1);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int part = PP - 1; part >= 0; --part)
                    acc[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[step & 1][ct], w[step & 1][part], acc[ct], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (step == max(STEPS - ITEMS, 0) + i || (step == STEPS - 1 && i >= STEPS))
                    stage.store(i, k_lds + (buffer ^ 1) * KT, v_lds + (buffer ^ 1) * VT);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                __builtin_amdgcn_sched_group_barrier(0x008, PP, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        __syncthreads();
    }
    if (m >= queries) return;
    sum += __shfl_xor(sum, 32);
    const int64_t unit = (int64_t(s) * p.c.layers + layer) * p.c.heads + head;
    const int64_t to = (unit * p.splits + split) * (int64_t(p.max_rows) * G) + m;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;     // no row seen: 0
    char *dst = p.out + s * p.os[0] + layer * p.os[1] + (head * G + g) * p.os[2] + i * p.os[3];
    if (p.splits > 1 && half == 0) p.ws_ml[to * 2] = top, p.ws_ml[to * 2 + 1] = sum;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int ch = 32 * ct + 2 * r + 4 * half;
            const f32x4 x = {acc[ct][r], acc[ct][r + 1], acc[ct][r + 2], acc[ct][r + 3]};
            if (p.splits > 1)
                *reinterpret_cast<f32x4 *>(p.ws_acc + to * D + ch) = x;
            else if (DTYPE == VD_DTYPE_F32)
                *reinterpret_cast<f32x4 *>(dst + ch * 4) = x * inv;
            else
                *reinterpret_cast<bf16x4 *>(dst + ch * 2) = bf16x4{__bf16(x[0] * inv), __bf16(x[1] * inv), __bf16(x[2] * inv), __bf16(x[3] * inv)};
        }
}

// Joins the splits of a query row.  WAVES waves of a workgroup take a row, of many
// splits all four; D / 4 lanes add up a split's sums.
template <int DTYPE, int D, int WAVES>
__global__ __launch_bounds__(kMxThreads) void attn_join_kernel(const MxAttnParams p) {
    constexpr int LANES = D / 4, AT_ONCE = WAVES * 64 / LANES;   // splits at a time
    __shared__ __attribute__((aligned(16))) f32x4 sums[kMxThreads];
    const int G = p.group, lane = threadIdx.x & 63;
    const int head = blockIdx.y, s = blockIdx.z / p.c.layers, layer = blockIdx.z % p.c.layers;
    const int row = threadIdx.x / (WAVES * 64), at = threadIdx.x % (WAVES * 64);
    const int query = min(int(blockIdx.x) * (4 / WAVES) + row, p.rows[s] * G - 1);   // (behind the last: the last again, not written)
    if (query < 0) return;                                                         // (a sequence without query rows)
    const int64_t unit = (int64_t(s) * p.c.layers + layer) * p.c.heads + head;
    const int64_t all = int64_t(p.max_rows) * G, first = unit * p.splits * all + query;
    const int mine = at / LANES, ch = at % LANES * 4;
    f32x4 x[4], o = {0, 0, 0, 0};
    auto load = [&](int base) {   // (behind the last split: the last again, not added)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = *reinterpret_cast<const f32x4 *>(p.ws_acc + (first + min(base + i * AT_ONCE + mine, p.splits - 1) * all) * D + ch);
    };
    load(0);
    float top[2], sum[2], high = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool has = lane + 64 * i < p.splits;
        const float *ml = p.ws_ml + (first + (has ? lane + 64 * i : 0) * all) * 2;
        top[i] = has ? ml[0] : -INFINITY;
        sum[i] = has ? ml[1] : 0.0f;
        high = fmaxf(high, top[i]);
    }
    for (int d = 1; d < 64; d *= 2) high = fmaxf(high, __shfl_xor(high, d));
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        top[i] = top[i] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top[i] - high);   // the split's factor
        total = fmaf(sum[i], top[i], total);
    }
    for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d);
    for (int base = 0; base < p.splits; base += 4 * AT_ONCE) {
        if (base > 0) load(base);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int split = base + i * AT_ONCE + mine;
            const float f0 = __shfl(top[0], split & 63), f1 = __shfl(top[1], split & 63), f = split < 64 ? f0 : f1;
            if (split < p.splits)
                for (int e = 0; e < 4; ++e) o[e] = fmaf(x[i][e], f, o[e]);
        }
    }
    if (AT_ONCE > 1) {
        sums[threadIdx.x] = o;
        __syncthreads();
        if (mine > 0) return;
        for (int i = 1; i < AT_ONCE; ++i) o += sums[threadIdx.x + i * LANES];
    }
    if (int(blockIdx.x) * (4 / WAVES) + row != query) return;
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const int qi = query / G, qg = query - qi * G;
    char *dst = p.out + s * p.os[0] + layer * p.os[1] + (head * G + qg) * p.os[2] + qi * p.os[3];
    if (DTYPE == VD_DTYPE_F32)
        *reinterpret_cast<f32x4 *>(dst + ch * 4) = o * inv;
    else
        *reinterpret_cast<bf16x4 *>(dst + ch * 2) = bf16x4{__bf16(o[0] * inv), __bf16(o[1] * inv), __bf16(o[2] * inv), __bf16(o[3] * inv)};
}

// ---------------------------------------------------------------- eviction
//
// One workgroup a unit: the column sums of its scored rows, their distances from
// the mean, the N highest, the gather.  Values are exact, sums and distances fp64:
// the fp32 scores, which the selection ranks, are correctly rounded but for a
// last-bit tie, whatever the order of the sums.
//
// A lane takes one group of a row (16 bytes and a scale), and always the same
// channels, whose sums and then means stay in its registers.  What bounds it is the
// arithmetic, not the reads: four rows are added in fp32 where that is exact (1.75
// instructions a value), a distance takes 3.5 (two values' conversion to fp32, one's to
// fp64, a subtraction and a fused multiply there).  256 units of 2560 rows of 128
// channels, 512 evicted, 38 us, of which the sums take 10, the mean 5, the scores 12,
// the selection 6, the gather 2; 1024 units of 1025 to 4097 rows, one evicted, 84 us.

constexpr int kEvictBatch = 4;    // rows of a lane in flight
constexpr int kEvictBins = 2048;
constexpr int kEvictMaxWaves = kMxEvictThreads / 64;

struct EvictHead {
    uint32_t hist[kEvictBins];
    uint32_t low[kEvictMaxWaves], high[kEvictMaxWaves];   // smallest and largest key
    uint32_t count[2][kEvictMaxWaves];
    uint32_t word[4];
    uint32_t cand_key[64], cand_slot[64];
    double mean[256];
    double len[1];
};

template <int CTRL>
__device__ __forceinline__ double dpp_double(double x) {
    const unsigned long long b = __builtin_bit_cast(unsigned long long, x);
    const uint32_t lo = dpp<CTRL>(uint32_t(b)), hi = dpp<CTRL>(uint32_t(b >> 32));
    return __builtin_bit_cast(double, (unsigned long long)(hi) << 32 | lo);
}
__device__ __forceinline__ double shfl_xor_double(double x, int d) {
    const unsigned long long b = __builtin_bit_cast(unsigned long long, x);
    const uint32_t lo = __shfl_xor(uint32_t(b), d), hi = __shfl_xor(uint32_t(b >> 32), d);
    return __builtin_bit_cast(double, (unsigned long long)(hi) << 32 | lo);
}
// Sum over the LANES neighbouring lanes (2, 4 or 8) of a row, in each of them.
template <int LANES>
__device__ __forceinline__ double row_sum(double x) {
    x += dpp_double<kXor1>(x);
    if (LANES >= 4) x += dpp_double<kXor2>(x);
    if (LANES >= 8) x += dpp_double<0x141>(x);   // the other four of eight
    return x;
}
// In lanes [0, 32) the sum of a over both halves of the wave, in [32, 64) that of b
// (Upper false: over both sixteens of each half).
template <bool UPPER>
__device__ __forceinline__ double halves_sum(double a, double b) {
    const unsigned long long x = __builtin_bit_cast(unsigned long long, a), y = __builtin_bit_cast(unsigned long long, b);
    u32x2 lo, hi;
    if (UPPER) {
        lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(uint32_t(x), uint32_t(y), false, false));
        hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(uint32_t(x >> 32), uint32_t(y >> 32), false, false));
    } else {
        lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(uint32_t(x), uint32_t(y), false, false));
        hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(uint32_t(x >> 32), uint32_t(y >> 32), false, false));
    }
    return __builtin_bit_cast(double, (unsigned long long)(hi[0]) << 32 | lo[0]) +
           __builtin_bit_cast(double, (unsigned long long)(hi[1]) << 32 | lo[1]);
}

// A larger key ranks higher; KeyNorm keeps the smallest norms.
__device__ __forceinline__ uint32_t rank_key(float score, bool smallest) {
    uint32_t b = bits(score == 0.0f ? 0.0f : score);
    b = b & 0x80000000u ? ~b : b | 0x80000000u;
    return smallest ? ~b : b;
}

struct GroupRow {
    u32x4 x;
    uint32_t scale;
};
// A lane's groups of the rows j, j + step, ...; rows behind the last read as 0.
__device__ __forceinline__ void load_groups(GroupRow (&r)[kEvictBatch], const char *xb, const char *sb, uint32_t slot,
                                            uint32_t sslot, int g, int j, int step, int n) {
#pragma unroll
    for (int u = 0; u < kEvictBatch; ++u) {
        const int row = j + u * step;
        const uint32_t at = uint32_t(min(row, n - 1));
        r[u].x = reinterpret_cast<const u32x4 *>(xb + at * slot)[g];
        r[u].scale = uint8_t(sb[at * sslot + g]);
        if (row >= n) r[u].x = u32x4{0, 0, 0, 0}, r[u].scale = 0;
    }
}
// Calls f(channel, value) for the 32 values of a group.
template <class F>
__device__ __forceinline__ void each_value(const GroupRow &r, F f) {
    const float scale = scale_of(r.scale);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x[w], scale, 0);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x[w], scale, 1);
        const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x[w], scale, 2);
        const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x[w], scale, 3);
        f(8 * w + 0, double(a[0])), f(8 * w + 1, double(a[1])), f(8 * w + 2, double(b[0])), f(8 * w + 3, double(b[1]));
        f(8 * w + 4, double(c[0])), f(8 * w + 5, double(c[1])), f(8 * w + 6, double(d[0])), f(8 * w + 7, double(d[1]));
    }
}

// Whether the sum of a batch's values, channel by channel, is exact in fp32: multiples
// of half the smallest scale, up to 24 times the largest, are for scales up to 2^16
// apart (and none so large that the sum is infinite).  Rows of zeros do not count.
__device__ __forceinline__ bool sum_is_exact(const GroupRow (&r)[kEvictBatch]) {
    uint32_t low = 255, high = 0;
#pragma unroll
    for (int u = 0; u < kEvictBatch; ++u) {
        const bool zero = (r[u].x[0] | r[u].x[1] | r[u].x[2] | r[u].x[3]) == 0;
        low = min(low, zero ? 255u : r[u].scale);
        high = max(high, zero ? 0u : r[u].scale);
    }
    return high <= 250 && int(high - low) <= 16;
}
__device__ __forceinline__ void add_batch(const GroupRow (&r)[kEvictBatch], double (&sum)[32]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        auto two = [&](auto sel) {
            f32x2 v[kEvictBatch];
#pragma unroll
            for (int u = 0; u < kEvictBatch; ++u)
                v[u] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r[u].x[w], scale_of(r[u].scale), decltype(sel)::value);
            constexpr int at = decltype(sel)::value;
            sum[8 * w + 2 * at] += double((v[0][0] + v[1][0]) + (v[2][0] + v[3][0]));
            sum[8 * w + 2 * at + 1] += double((v[0][1] + v[1][1]) + (v[2][1] + v[3][1]));
        };
        two(std::integral_constant<int, 0>()), two(std::integral_constant<int, 1>());
        two(std::integral_constant<int, 2>()), two(std::integral_constant<int, 3>());
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The boundary of the N highest of n > N keys (equal ones by the lower slot): a
// row stays if its key is above `key`, or equal to it in a slot up to `slot`.
// Keys are counted in bins of equal width between the smallest and the largest; the
// bin that the boundary falls into is narrowed until it holds at most 64 keys,
// which one wave ranks, or one value.
struct Boundary {
    uint32_t key;
    int slot;
};
template <int THREADS>
__device__ __forceinline__ Boundary boundary(EvictHead &sh, const uint32_t *keys, int n, int N, uint32_t low, uint32_t high) {
    constexpr int WAVES = THREADS / 64, EACH = kEvictBins / THREADS;   // bins of a thread
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int want = N;   // keys to keep among those in [low, high]
    for (;;) {
        const uint32_t range = high - low;
        const int shift = range < uint32_t(kEvictBins) ? 0 : 32 - __builtin_clz(range) - 11;   // (2^11 bins)
        for (int i = tid; i < kEvictBins; i += THREADS) sh.hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += THREADS) {
            const uint32_t at = keys[j] - low;
            if (at <= range) atomicAdd(&sh.hist[at >> shift], 1u);
        }
        __syncthreads();
        // from the highest bin down, a few bins a thread
        uint32_t c[EACH], mine = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) mine += c[i] = sh.hist[kEvictBins - 1 - EACH * tid - i];
        uint32_t upto = mine;
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 63) sh.count[0][wave] = upto;
        __syncthreads();
        for (int w = 0; w < WAVES; ++w) upto += w < wave ? sh.count[0][w] : 0u;
        uint32_t above = upto - mine;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (above < uint32_t(want) && above + c[i] >= uint32_t(want))
                sh.word[0] = uint32_t(kEvictBins - 1 - EACH * tid - i), sh.word[1] = above, sh.word[2] = c[i];
            above += c[i];
        }
        if (tid == 0) sh.word[3] = 0;
        __syncthreads();
        const uint32_t bin = sh.word[0], count = sh.word[2];
        want -= int(sh.word[1]);
        low += bin << shift;
        high = min(high, low + ((1u << shift) - 1));
        if (count <= 64) {
            for (int j = tid; j < n; j += THREADS) {
                const uint32_t key = keys[j];
                if (key - low <= high - low) {
                    const uint32_t i = atomicAdd(&sh.word[3], 1u);
                    if (i < 64) sh.cand_key[i] = key, sh.cand_slot[i] = uint32_t(j);
                }
            }
            __syncthreads();
            if (wave == 0) {
                const bool mine = lane < int(count);
                const uint32_t key = mine ? sh.cand_key[lane] : 0u, slot = mine ? sh.cand_slot[lane] : 0u;
                int rank = 0;
                for (int i = 0; i < int(count); ++i) {
                    const uint32_t k = __shfl(key, i), s = __shfl(slot, i);
                    rank += k > key || (k == key && s < slot);
                }
                if (mine && rank == want - 1) sh.word[0] = key, sh.word[1] = slot;
            }
            __syncthreads();
            return {sh.word[0], int(sh.word[1])};
        }
        if (shift == 0) break;
    }
    // more than 64 equal keys: the slot of the want-th of them; a wave takes a run of slots
    const int span = (n + THREADS - 1) / THREADS * 64;
    const int first = wave * span, last = min(first + span, n);
    int ties = 0;
    for (int base = first; base < last; base += 64)
        ties += __popcll(__builtin_amdgcn_ballot_w64(base + lane < last && keys[min(base + lane, n - 1)] == low));
    if (lane == 0) sh.count[0][wave] = uint32_t(ties);
    __syncthreads();
    int before = 0;
    for (int w = 0; w < WAVES; ++w) before += w < wave ? int(sh.count[0][w]) : 0;
    for (int base = first; base < last; base += 64) {
        const bool tie = base + lane < last && keys[min(base + lane, n - 1)] == low;
        const unsigned long long b = __builtin_amdgcn_ballot_w64(tie);
        if (tie && before + __popcll(b & ((1ull << lane) - 1)) == want - 1) sh.word[1] = uint32_t(base + lane);
        before += __popcll(b);
    }
    __syncthreads();
    return {low, int(sh.word[1])};
}

template <int D, int FORM, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void evict_kernel(const MxEvictParams p) {
    constexpr int LANES = D / 32, WAVES = THREADS / 64;   // lanes of a row: a group each
    constexpr int ROWS = THREADS / LANES;         // rows that the workgroup takes at a time
    extern __shared__ __attribute__((aligned(16))) char dyn[];
    __shared__ EvictHead sh;
    uint32_t *keys = reinterpret_cast<uint32_t *>(dyn);
    uint16_t *holes = reinterpret_cast<uint16_t *>(dyn + p.off_lists), *movers = holes + p.list_cap;
    double *partial = reinterpret_cast<double *>(dyn);    // [wave][D], before the keys
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int head = blockIdx.x, layer = blockIdx.y, s = blockIdx.z;
    const int n = p.n[s], N = p.budget[s];
    if (n == 0) return;
    const int64_t unit = (int64_t(s) * p.c.layers + layer) * p.c.heads + head;
    const int64_t code_at = s * p.c.seq + layer * p.c.layer + head * p.c.head;
    const int64_t scale_at = s * p.c.sseq + layer * p.c.slayer + head * p.c.shead;
    const bool key_side = p.variant >= VD_SCORE_KEY_L2;
    const bool smallest = p.variant == VD_SCORE_KEY_NORM;
    float *scores = p.scores ? p.scores + unit * p.capacity : nullptr;
    uint8_t *keep = p.keep ? p.keep + unit * p.capacity : nullptr;
    if (n <= N && keep)
        for (int j = tid; j < n; j += THREADS) keep[j] = 1;
    if (n <= N && !scores) return;
    const char *xb = (key_side ? p.c.k : p.c.v) + code_at, *sb = (key_side ? p.c.ks : p.c.vs) + scale_at;
    const int g = tid % LANES, r0 = tid / LANES;          // the lane's group, its row of the workgroup's
    const int w0 = __builtin_amdgcn_readfirstlane(r0);     // the wave's first

    GroupRow row[kEvictBatch];
    load_groups(row, xb, sb, p.c.slot, p.c.sslot, g, r0, ROWS, n);
    double mean[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) mean[i] = 0.0;
    double length = 0.0;
    if (FORM != VD_SCORE_NORM) {
        bool exact = true;
        int from = 0;
        for (; from + w0 + (kEvictBatch - 1) * ROWS < n; from += kEvictBatch * ROWS) {
            if (from > 0) load_groups(row, xb, sb, p.c.slot, p.c.sslot, g, from + r0, ROWS, n);
            exact = exact && sum_is_exact(row);
            add_batch(row, mean);
        }
        if (from + w0 < n) {   // the rest, a row at a time
            if (from > 0) load_groups(row, xb, sb, p.c.slot, p.c.sslot, g, from + r0, ROWS, n);
#pragma unroll
            for (int u = 0; u + 1 < kEvictBatch; ++u)
                if (from + w0 + u * ROWS < n) each_value(row[u], [&](int i, double v) { mean[i] += v; });
        }
        if (__builtin_amdgcn_ballot_w64(!exact)) {   // (rare: the wave's rows again, value by value in fp64)
#pragma unroll
            for (int i = 0; i < 32; ++i) mean[i] = 0.0;
            for (int j = r0; j < n; j += kEvictBatch * ROWS) {
                load_groups(row, xb, sb, p.c.slot, p.c.sslot, g, j, ROWS, n);
#pragma unroll
                for (int u = 0; u < kEvictBatch; ++u) {
                    each_value(row[u], [&](int i, double v) { mean[i] += v; });
                    __builtin_amdgcn_sched_barrier(0);   // one row's conversions at a time: registers
                }
            }
        }
        load_groups(row, xb, sb, p.c.slot, p.c.sslot, g, r0, ROWS, n);   // the second reading's first, on their way meanwhile
        // over the lanes with the same group: halves of the wave and of those keep half
        // of the channels each, then the lanes of sixteen are added up
#pragma unroll
        for (int i = 0; i < 16; ++i) mean[i] = halves_sum<true>(mean[i], mean[i + 16]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            double t = halves_sum<false>(mean[i], mean[i + 8]);
            if (LANES <= 8) t += dpp_double<0x128>(t);   // row_ror:8
            if (LANES <= 4) t += dpp_double<0x124>(t);   // row_ror:4
            if (LANES <= 2) t += dpp_double<0x122>(t);   // row_ror:2
            if ((lane & 15) < LANES) partial[wave * D + g * 32 + i + 8 * ((lane >> 4) & 1) + 16 * (lane >> 5)] = t;
        }
        __syncthreads();
        if (tid < D) {
            double t = 0.0;
            for (int w = 0; w < WAVES; ++w) t += partial[w * D + tid];
            sh.mean[tid] = t / double(n);
        }
        __syncthreads();
        if (FORM == VD_SCORE_DIR) {
            if (wave == 0) {
                double t = 0.0;
                for (int c = lane; c < D; c += 64) t = fma(sh.mean[c], sh.mean[c], t);
                for (int d = 1; d < 64; d *= 2) t += shfl_xor_double(t, d);
                if (lane == 0) sh.len[0] = sqrt(t);
            }
            __syncthreads();
            length = sh.len[0];
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) mean[i] = sh.mean[g * 32 + i];
    }

    uint32_t low = ~0u, high = 0u;
    for (int j = r0; j < n; j += kEvictBatch * ROWS) {
        if (j != r0) load_groups(row, xb, sb, p.c.slot, p.c.sslot, g, j, ROWS, n);
        double sq[kEvictBatch], dot[kEvictBatch];
#pragma unroll
        for (int u = 0; u < kEvictBatch; ++u) {
            double a = 0.0, b = 0.0;
            if (j - r0 + w0 + u * ROWS < n)   // (else none of the wave's rows)
                each_value(row[u], [&](int i, double v) {
                    if (FORM == VD_SCORE_L2) v -= mean[i];
                    a = fma(v, v, a);
                    if (FORM == VD_SCORE_DIR) b = fma(v, mean[i], b);
                });
            sq[u] = row_sum<LANES>(a);
            if (FORM == VD_SCORE_DIR) dot[u] = row_sum<LANES>(b);
            __builtin_amdgcn_sched_barrier(0);
        }
        // every lane of a row has its sums: the row's lanes finish one row of the batch each
#pragma unroll
        for (int u0 = 0; u0 < kEvictBatch; u0 += LANES) {
            const int u = u0 + g;
            double a = sq[u0], b = FORM == VD_SCORE_DIR ? dot[u0] : 0.0;
#pragma unroll
            for (int e = 1; e < (LANES < kEvictBatch ? LANES : kEvictBatch); ++e) {
                a = g == e ? sq[(u0 + e) % kEvictBatch] : a;
                if (FORM == VD_SCORE_DIR) b = g == e ? dot[(u0 + e) % kEvictBatch] : b;
            }
            double score = sqrt(a);
            if (FORM == VD_SCORE_DIR) {
                const double both = score * length;
                score = both > 0.0 ? 1.0 - b / both : both == 0.0 ? 1.0 : both;
            }
            const int slot = j + u * ROWS;
            if (u < kEvictBatch && slot < n) {
                const float out = float(score);
                const uint32_t key = rank_key(out, smallest);
                low = min(low, key);
                high = max(high, key);
                if (scores) scores[slot] = out;
                if (n > N) keys[slot] = key;
            }
        }
    }
    if (n <= N) return;
    for (int d = 1; d < 64; d *= 2) low = min(low, __shfl_xor(low, d)), high = max(high, __shfl_xor(high, d));
    if (lane == 0) sh.low[wave] = low, sh.high[wave] = high;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) low = min(low, sh.low[w]), high = max(high, sh.high[w]);

    int moved;   // rows to move: movers[k] onto holes[k]
    if (n == N + 1) {
        // the lowest key goes, the highest slot among equal ones
        int gone = -1;
        for (int j = tid; j < n; j += THREADS)
            if (keys[j] == low) gone = j;
        for (int d = 1; d < 64; d *= 2) gone = max(gone, __shfl_xor(gone, d));
        if (lane == 0) sh.count[0][wave] = uint32_t(gone + 1);
        __syncthreads();
        for (int w = 0; w < WAVES; ++w) gone = max(gone, int(sh.count[0][w]) - 1);
        if (keep)
            for (int j = tid; j < n; j += THREADS) keep[j] = j != gone;
        if (tid == 0) holes[0] = uint16_t(gone), movers[0] = uint16_t(N);
        moved = gone < N;
        __syncthreads();
    } else {
        const Boundary edge = boundary<THREADS>(sh, keys, n, N, low, high);
        // the lists in the order of the slots: a wave takes a run of them, counts, then writes
        const int span = (n + THREADS - 1) / THREADS * 64;
        const int first = wave * span, last = min(first + span, n);
        const unsigned long long below = (1ull << lane) - 1;
        auto stays = [&](int j) { return keys[j] > edge.key || (keys[j] == edge.key && j <= edge.slot); };
        int nh = 0, nm = 0;
        for (int base = first; base < last; base += 64) {
            const int j = base + lane;
            const bool kept = j < last && stays(j);
            if (keep && j < last) keep[j] = kept;
            nh += __popcll(__builtin_amdgcn_ballot_w64(j < min(N, last) && !kept));
            nm += __popcll(__builtin_amdgcn_ballot_w64(j >= N && kept));
        }
        if (lane == 0) sh.count[0][wave] = uint32_t(nh), sh.count[1][wave] = uint32_t(nm);
        __syncthreads();
        int hr = 0, mr = 0;
        nh = nm = 0;
        for (int w = 0; w < WAVES; ++w) {
            hr += w < wave ? int(sh.count[0][w]) : 0;
            mr += w < wave ? int(sh.count[1][w]) : 0;
            nh += int(sh.count[0][w]);
            nm += int(sh.count[1][w]);
        }
        for (int base = first; base < last; base += 64) {
            const int j = base + lane;
            const bool kept = j < last && stays(j), hole = j < min(N, last) && !kept, mover = j >= N && kept;
            const unsigned long long hb = __builtin_amdgcn_ballot_w64(hole), mb = __builtin_amdgcn_ballot_w64(mover);
            const int hi = hr + __popcll(hb & below), mi = mr + __popcll(mb & below);
            if (hole && hi < p.list_cap) holes[hi] = uint16_t(j);
            if (mover && mi < p.list_cap) movers[mi] = uint16_t(j);
            hr += __popcll(hb);
            mr += __popcll(mb);
        }
        moved = min(min(nh, nm), p.list_cap);
        __syncthreads();
    }

    // The gather: codes in 16-byte words (K's, then V's), a few loads in flight; rows'
    // scales in one word each, and the tokens' indices.
    constexpr int WORDS = D / 32;
    char *kb = p.c.k + code_at, *vb = p.c.v + code_at, *ksb = p.c.ks + scale_at, *vsb = p.c.vs + scale_at;
    int32_t *pos = p.pos ? p.pos + unit * p.capacity : nullptr;
    using Word = std::conditional_t<D == 64, uint16_t, std::conditional_t<D == 128, uint32_t, u32x2>>;
    for (int first = 0; first < moved; first += THREADS) {
        const int rows = min(THREADS, moved - first), mine = first + min(tid, rows - 1);
        const uint32_t to = holes[mine], from = movers[mine];
        const Word a = *reinterpret_cast<const Word *>(ksb + from * p.c.sslot), b = *reinterpret_cast<const Word *>(vsb + from * p.c.sslot);
        const int32_t t = pos ? pos[from] : 0;
        for (int base = tid; base < rows * 2 * WORDS; base += 4 * THREADS) {
            u32x4 x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int at = min(base + u * THREADS, rows * 2 * WORDS - 1), w = at % (2 * WORDS);
                x[u] = reinterpret_cast<const u32x4 *>((w < WORDS ? kb : vb) + movers[first + at / (2 * WORDS)] * p.c.slot)[w % WORDS];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int at = base + u * THREADS, w = at % (2 * WORDS);
                if (at < rows * 2 * WORDS)
                    reinterpret_cast<u32x4 *>((w < WORDS ? kb : vb) + holes[first + at / (2 * WORDS)] * p.c.slot)[w % WORDS] = x[u];
            }
        }
        if (tid < rows) {
            *reinterpret_cast<Word *>(ksb + to * p.c.sslot) = a;
            *reinterpret_cast<Word *>(vsb + to * p.c.sslot) = b;
            if (pos) pos[to] = t;
        }
    }
}

}  // namespace

// ---------------------------------------------------------------- launches

namespace {

template <class P, class F>
hipError_t launch_rows(const P &p, int seqs, int head_dim, F kernel, hipStream_t stream) {
    const int64_t threads = int64_t(p.c.layers) * p.c.heads * p.max_rows * (head_dim / 8);
    const dim3 grid(uint32_t((threads + kMxThreads - 1) / kMxThreads), uint32_t(2 * seqs));
    return launch_with<P>(kernel, grid, kMxThreads, 0, stream, p);
}

template <int DTYPE, int D>
hipError_t launch_attn(const MxAttnParams &p, int seqs, hipStream_t stream) {
    const dim3 grid(uint32_t(p.splits) * p.tiles, p.c.heads, seqs * p.c.layers);
    constexpr bool BLOCK = !(DTYPE == VD_DTYPE_F32 && D == 256);   // (whose registers do not hold it)
    const hipError_t e = launch_with(p.block ? attn_block_kernel<DTYPE, BLOCK ? D : 128> : attn_kernel<DTYPE, D>, grid, kMxThreads, 0, stream, p);
    if (e != hipSuccess || p.splits == 1) return e;
    const bool many = p.splits > 8;
    const uint32_t per = many ? 1 : 4, queries = uint32_t(p.max_rows) * p.group;
    return launch_with(many ? attn_join_kernel<DTYPE, D, 4> : attn_join_kernel<DTYPE, D, 1>,
                       dim3((queries + per - 1) / per, p.c.heads, seqs * p.c.layers), kMxThreads, 0, stream, p);
}

template <int D, int THREADS>
hipError_t launch_evict(const MxEvictParams &p, int seqs, size_t lds, hipStream_t stream) {
    const int form = p.variant - (p.variant >= VD_SCORE_KEY_L2 ? VD_SCORE_KEY_L2 : 0);
    return launch_with(form == VD_SCORE_L2    ? evict_kernel<D, VD_SCORE_L2, THREADS>
                       : form == VD_SCORE_DIR ? evict_kernel<D, VD_SCORE_DIR, THREADS>
                                              : evict_kernel<D, VD_SCORE_NORM, THREADS>,
                       dim3(p.c.heads, p.c.layers, seqs), THREADS, lds, stream, p);
}

}  // namespace

hipError_t launch_mx_append(const MxRowsParams &p, int seqs, int dtype, int D, hipStream_t stream) {
    const bool b = dtype == VD_DTYPE_BF16;
    return D == 64    ? launch_rows(p, seqs, D, b ? append_kernel<VD_DTYPE_BF16, 64> : append_kernel<VD_DTYPE_F32, 64>, stream)
           : D == 128 ? launch_rows(p, seqs, D, b ? append_kernel<VD_DTYPE_BF16, 128> : append_kernel<VD_DTYPE_F32, 128>, stream)
                      : launch_rows(p, seqs, D, b ? append_kernel<VD_DTYPE_BF16, 256> : append_kernel<VD_DTYPE_F32, 256>, stream);
}
hipError_t launch_mx_read(const MxRowsParams &p, int seqs, int dtype, int D, hipStream_t stream) {
    const bool b = dtype == VD_DTYPE_BF16;
    return D == 64    ? launch_rows(p, seqs, D, b ? read_kernel<VD_DTYPE_BF16, 64> : read_kernel<VD_DTYPE_F32, 64>, stream)
           : D == 128 ? launch_rows(p, seqs, D, b ? read_kernel<VD_DTYPE_BF16, 128> : read_kernel<VD_DTYPE_F32, 128>, stream)
                      : launch_rows(p, seqs, D, b ? read_kernel<VD_DTYPE_BF16, 256> : read_kernel<VD_DTYPE_F32, 256>, stream);
}
hipError_t launch_mx_attention(const MxAttnParams &p, int seqs, int dtype, int D, hipStream_t stream) {
    if (dtype == VD_DTYPE_BF16)
        return D == 64    ? launch_attn<VD_DTYPE_BF16, 64>(p, seqs, stream)
               : D == 128 ? launch_attn<VD_DTYPE_BF16, 128>(p, seqs, stream)
                          : launch_attn<VD_DTYPE_BF16, 256>(p, seqs, stream);
    return D == 64    ? launch_attn<VD_DTYPE_F32, 64>(p, seqs, stream)
           : D == 128 ? launch_attn<VD_DTYPE_F32, 128>(p, seqs, stream)
                      : launch_attn<VD_DTYPE_F32, 256>(p, seqs, stream);
}
hipError_t launch_mx_evict(const MxEvictParams &p, int seqs, int D, size_t lds, hipStream_t stream) {
    if (p.threads == kMxEvictThreads)
        return D == 64    ? launch_evict<64, kMxEvictThreads>(p, seqs, lds, stream)
               : D == 128 ? launch_evict<128, kMxEvictThreads>(p, seqs, lds, stream)
                          : launch_evict<256, kMxEvictThreads>(p, seqs, lds, stream);
    return D == 64    ? launch_evict<64, kMxEvictThreads / 2>(p, seqs, lds, stream)
           : D == 128 ? launch_evict<128, kMxEvictThreads / 2>(p, seqs, lds, stream)
                      : launch_evict<256, kMxEvictThreads / 2>(p, seqs, lds, stream);
}

}  // namespace vd
