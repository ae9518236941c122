// Norms of query and key rows and their rotation, in one read and one write.
//
// y = x / sqrt(mean(x^2) + eps) * w over the D channels of a row (one head of
// one token), then for each rotated pair (a, b) of channels
//   (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = pos * inv_freq[i].
//
// Bandwidth bounds it: about ten operations for each value that is read and
// written.  A row is taken by D / 8 lanes, each with four pairs, so that a pair
// never leaves its lane: the partner channel, D / 2 away or the next one, is a
// second load and not a shuffle.  A lane keeps its pairs' cos and sin for all
// (layer, head) rows that it takes of a token.  512 tokens of 1280 rows of 128 bf16
// channels, 336 MB read and written, 69 us (4.8 TB/s, a large copy's rate); 999 tokens of
// 156 rows of 256 fp32 channels, 319 MB, 59 us.
#include <hip/hip_runtime.h>

#include "vd.h"
#include "vd_mx4.h"

namespace vd {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float low_bf16(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float high_bf16(uint32_t x) { return __builtin_bit_cast(float, x & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, (bf16x2{__bf16(a), __bf16(b)})); }

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

// Sum over the LANES lanes (8, 16 or 32) that share a row, in each of them.
template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
    x = dpp_add<0xB1>(x);    // lane ^ 1
    x = dpp_add<0x4E>(x);    // lane ^ 2
    x = dpp_add<0x141>(x);   // the other four of eight
    if (LANES >= 16) x = dpp_add<0x140>(x);   // the other eight of sixteen
    if (LANES >= 32)
        x += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, x), 0x401F));  // lane ^ 16
    return x;
}

// A lane's eight channels: a[i], b[i] are its pairs.  Neighbours: eight
// channels from `ca` on.  Halves: four from `ca` and four from `cb`.
struct Pairs {
    f32x4 a, b;
};

template <bool NEXT>
__device__ __forceinline__ Pairs load_pairs(const char *row, int ca, int cb, bool f32) {
    Pairs r;
    if (f32) {
        const f32x4 u = *reinterpret_cast<const f32x4 *>(row + ca * 4);
        const f32x4 w = *reinterpret_cast<const f32x4 *>(row + (NEXT ? ca + 4 : cb) * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.a[i] = NEXT ? (i < 2 ? u[2 * (i & 1)] : w[2 * (i & 1)]) : u[i];
            r.b[i] = NEXT ? (i < 2 ? u[2 * (i & 1) + 1] : w[2 * (i & 1) + 1]) : w[i];
        }
    } else if (NEXT) {
        const u32x4 u = *reinterpret_cast<const u32x4 *>(row + ca * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.a[i] = low_bf16(u[i]), r.b[i] = high_bf16(u[i]);
    } else {
        const u32x2 u = *reinterpret_cast<const u32x2 *>(row + ca * 2), w = *reinterpret_cast<const u32x2 *>(row + cb * 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            r.a[2 * i] = low_bf16(u[i]), r.a[2 * i + 1] = high_bf16(u[i]);
            r.b[2 * i] = low_bf16(w[i]), r.b[2 * i + 1] = high_bf16(w[i]);
        }
    }
    return r;
}

template <bool NEXT>
__device__ __forceinline__ void store_pairs(char *row, int ca, int cb, bool f32, const Pairs &r) {
    if (f32) {
        const f32x4 u = NEXT ? f32x4{r.a[0], r.b[0], r.a[1], r.b[1]} : f32x4{r.a[0], r.a[1], r.a[2], r.a[3]};
        const f32x4 w = NEXT ? f32x4{r.a[2], r.b[2], r.a[3], r.b[3]} : f32x4{r.b[0], r.b[1], r.b[2], r.b[3]};
        *reinterpret_cast<f32x4 *>(row + ca * 4) = u;
        *reinterpret_cast<f32x4 *>(row + (NEXT ? ca + 4 : cb) * 4) = w;
    } else if (NEXT) {
        *reinterpret_cast<u32x4 *>(row + ca * 2) =
            u32x4{pack(r.a[0], r.b[0]), pack(r.a[1], r.b[1]), pack(r.a[2], r.b[2]), pack(r.a[3], r.b[3])};
    } else {
        *reinterpret_cast<u32x2 *>(row + ca * 2) = u32x2{pack(r.a[0], r.a[1]), pack(r.a[2], r.a[3])};
        *reinterpret_cast<u32x2 *>(row + cb * 2) = u32x2{pack(r.b[0], r.b[1]), pack(r.b[2], r.b[3])};
    }
}

template <int DTYPE, int D, bool NEXT>
__global__ __launch_bounds__(256) void rope_kernel(const RopeParams p) {
    constexpr int LANES = D / 8;
    const uint32_t group = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int lane = threadIdx.x % LANES;
    const uint32_t token = group % uint32_t(p.tokens), item = group / uint32_t(p.tokens);
    if (item >= uint32_t(p.items)) return;
    const int s = int(token / uint32_t(p.rows)), row = int(token % uint32_t(p.rows));
    const int half = p.rotary / 2, first = 4 * lane;   // the lane's pairs: first .. first + 3 of D / 2
    const bool turned = first < half;
    int ca, cb;
    if (NEXT) {
        ca = 2 * first;
        cb = ca;
    } else if (turned) {
        ca = first;
        cb = half + first;
    } else {  // channels that only the norm touches
        ca = p.rotary + first - half;
        cb = ca + (D - p.rotary) / 2;
    }
    // The angle in turns, in fp64 (a far position times a frequency keeps an
    // absolute error of 2^-53 of its size), less its whole turns.
    f32x4 cos = {1, 1, 1, 1}, sin = {0, 0, 0, 0};
    if (turned) {
        const double at = double(p.pos[token]) * 0.15915494309189533577;
        const f32x4 f = *reinterpret_cast<const f32x4 *>(p.inv_freq + first);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double turns = at * double(f[i]);
            const float half_turns = 2.0f * float(turns - rint(turns));
            cos[i] = cospif(half_turns);
            sin[i] = sinpif(half_turns);
        }
    }
    const int heads = p.q.heads + p.k.heads;
    int r = int(item) * p.per_item;
    const int end = min(r + p.per_item, p.layers * heads);
    int layer = r / heads, head = r % heads;
    for (; r < end; ++r) {
        const bool is_q = head < p.q.heads;
        const int h = is_q ? head : head - p.q.heads;
        const char *x;
        char *y;
        const char *w;
        int y_dtype;
        if (is_q) {
            x = p.q.x + s * p.q.xs[0] + layer * p.q.xs[1] + h * p.q.xs[2] + row * p.q.xs[3];
            y = p.q.y + s * p.q.ys[0] + layer * p.q.ys[1] + h * p.q.ys[2] + row * p.q.ys[3];
            w = p.q.w;
            y_dtype = p.q.y_dtype;
        } else {
            x = p.k.x + s * p.k.xs[0] + layer * p.k.xs[1] + h * p.k.xs[2] + row * p.k.xs[3];
            y = p.k.y + s * p.k.ys[0] + layer * p.k.ys[1] + h * p.k.ys[2] + row * p.k.ys[3];
            w = p.k.w;
            y_dtype = p.k.y_dtype;
        }
        Pairs v = load_pairs<NEXT>(x, ca, cb, DTYPE == VD_DTYPE_F32);
        if (w) {
            const bool wide = p.w_dtype == VD_DTYPE_F32;
            const Pairs g = load_pairs<NEXT>(w + int64_t(layer) * D * (wide ? 4 : 2), ca, cb, wide);
            float sq = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sq = fmaf(v.a[i], v.a[i], fmaf(v.b[i], v.b[i], sq));
            const float scale = 1.0f / sqrtf(row_sum<LANES>(sq) * (1.0f / D) + p.eps);
#pragma unroll
            for (int i = 0; i < 4; ++i) v.a[i] *= scale * g.a[i], v.b[i] *= scale * g.b[i];
        }
        Pairs o = v;   // (where not turned: a product with cos = 1, sin = 0 would make NaN of an infinity)
#pragma unroll
        for (int i = 0; i < 4 && turned; ++i) {
            o.a[i] = fmaf(v.a[i], cos[i], -v.b[i] * sin[i]);
            o.b[i] = fmaf(v.b[i], cos[i], v.a[i] * sin[i]);
        }
        store_pairs<NEXT>(y, ca, cb, y_dtype == VD_DTYPE_F32, o);
        if (++head == heads) head = 0, ++layer;
    }
}

template <int DTYPE, int D>
hipError_t launch(const RopeParams &p, bool interleaved, hipStream_t stream) {
    const int64_t groups = int64_t(p.tokens) * p.items, per_block = 256 / (D / 8);
    const dim3 grid(uint32_t((groups + per_block - 1) / per_block));
    return launch_with(interleaved ? rope_kernel<DTYPE, D, true> : rope_kernel<DTYPE, D, false>, grid, 256, 0, stream, p);
}

}  // namespace

hipError_t launch_rope(const RopeParams &p, int dtype, int head_dim, bool interleaved, hipStream_t stream) {
    if (dtype == VD_DTYPE_BF16)
        return head_dim == 64    ? launch<VD_DTYPE_BF16, 64>(p, interleaved, stream)
               : head_dim == 128 ? launch<VD_DTYPE_BF16, 128>(p, interleaved, stream)
                                 : launch<VD_DTYPE_BF16, 256>(p, interleaved, stream);
    return head_dim == 64    ? launch<VD_DTYPE_F32, 64>(p, interleaved, stream)
           : head_dim == 128 ? launch<VD_DTYPE_F32, 128>(p, interleaved, stream)
                             : launch<VD_DTYPE_F32, 256>(p, interleaved, stream);
}

}  // namespace vd
