// Internal contract between the host entry points of the 4-bit cache
// (vd_mx4.cpp), of the rotated rows (vd_rope.cpp) and their kernels.
// Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vd {

constexpr int kMxSeqs = 256;      // sequences per launch: their counts travel as kernel arguments
constexpr int kMxGroup = 32;      // channels that share a scale
constexpr int kMxThreads = 256;   // threads of an append, read or attention workgroup
constexpr int kMxEvictThreads = 1024;
constexpr int kMxTile = 16;       // query rows of the attention kernel's tile
constexpr int kMxBlockTile = 128; // and of the one for blocks of them
// its workgroups on a CU: with one wave a SIMD the sums and queries of 256 channels, or
// the three parts of 128, stay in registers (those of 256 do not)
constexpr int block_groups(int dtype, int head_dim) { return head_dim == 256 || (dtype == 1 && head_dim == 128) ? 1 : 2; }
constexpr int kMxMaxSplits = 128; // two for each lane of a joining wave

// A 4-bit cache as the kernels see it: bases of the launch's first sequence,
// strides in bytes.  A unit's slab spans < 4 GiB.
struct MxCache {
    char *k, *v, *ks, *vs;
    int64_t seq, layer, head;      // of the codes
    int64_t sseq, slayer, shead;   // of the scales
    uint32_t slot, sslot;
    int32_t layers, heads;
};

struct MxRowsParams {  // append and read
    MxCache c;
    char *k, *v;               // rows of the launch's first sequence
    int64_t ks[4], vs[4];      // their strides (sequence, layer, head, row) in bytes
    int32_t *pos;              // [U][capacity] of the launch's first sequence, or null
    int32_t capacity, max_rows;
    int32_t first[kMxSeqs], rows[kMxSeqs], pos0[kMxSeqs];
};
hipError_t launch_mx_append(const MxRowsParams &p, int seqs, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_mx_read(const MxRowsParams &p, int seqs, int dtype, int head_dim, hipStream_t stream);

struct MxAttnParams {
    MxCache c;
    const char *q;
    char *out;
    int64_t qs[4], os[4];      // strides (sequence, layer, query head, row) in bytes
    float *ws_acc;             // [unit][split][query row][D] unnormalised sums of the values
    float *ws_ml;              // [unit][split][query row][2] largest logit (log2 units), sum of the weights
    float qscale;              // size of the softmax scale times log2(e), > 0
    uint32_t flip;             // sign bit of the softmax scale
    int32_t group;             // query heads per KV head
    int32_t max_rows, splits, tiles;
    int32_t block;             // the kernel for blocks of query rows, its tiles of kMxBlockTile
    int32_t n[kMxSeqs], rows[kMxSeqs];
};
hipError_t launch_mx_attention(const MxAttnParams &p, int seqs, int dtype, int head_dim, hipStream_t stream);

struct MxEvictParams {
    MxCache c;
    int32_t *pos;              // [U][capacity] of the launch's first sequence, or null
    float *scores;             // the same, or null
    uint8_t *keep;             // the same, or null
    int32_t capacity, variant;
    int32_t threads;           // of a workgroup: kMxEvictThreads or half of them
    int32_t off_lists;         // dynamic LDS: keys, then the lists from this byte on
    int32_t list_cap;          // entries of each list
    int32_t n[kMxSeqs], budget[kMxSeqs];
};
hipError_t launch_mx_evict(const MxEvictParams &p, int seqs, int head_dim, size_t lds, hipStream_t stream);

// One launch; the kernel's only argument is its parameters.
template <class P>
inline hipError_t launch_with(void (*kernel)(P), dim3 grid, uint32_t threads, size_t lds, hipStream_t stream, const P &p) {
    void *args[] = {const_cast<P *>(&p)};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(threads), args, lds, stream);
}

struct RopeSide {
    const char *x;
    char *y;
    const char *w;             // [layers][D] or null
    int64_t xs[4], ys[4];      // strides (sequence, layer, head, row) in bytes
    int32_t heads, y_dtype;
};
struct RopeParams {
    RopeSide q, k;
    const int32_t *pos;        // [sequences][rows]
    const float *inv_freq;     // [rotary / 2]
    int32_t tokens, rows, layers, rotary, w_dtype;
    int32_t per_item, items;   // (layer, head) rows that one group of lanes takes; such items per token
    float eps;
};
hipError_t launch_rope(const RopeParams &p, int dtype, int head_dim, bool interleaved, hipStream_t stream);

}  // namespace vd
