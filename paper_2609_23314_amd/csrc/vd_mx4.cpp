// Host side of the 4-bit cache and of the rotated rows (include/vd.h):
// validation before any HIP call, then the launches, at most kMxSeqs sequences
// each.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "vd.h"
#include "vd_check.h"
#include "vd_mx4.h"

using namespace vd::host;

namespace {

constexpr int64_t kFar = int64_t(1) << 46;   // byte offsets stay far from 64 bits

struct Extent {
    uintptr_t at;
    uint64_t bytes;
    bool meets(const Extent &o) const { return at < o.at + o.bytes && o.at < at + bytes; }
};

// The bytes from the first element to the last of an array [count...] of
// `strides` (bytes) whose last axis holds `row` bytes; false if it is absurd.  (An axis
// of one element is never stepped along: its stride may be anything.)
bool extent_of(const void *base, const int64_t *count, const int64_t *strides, int axes, int64_t row, Extent &e) {
    e.at = reinterpret_cast<uintptr_t>(base);
    e.bytes = uint64_t(row);
    for (int i = 0; i < axes; ++i) {
        if (count[i] == 1) continue;
        if (strides[i] < 0 || strides[i] > kFar / count[i]) return false;
        e.bytes += uint64_t(strides[i]) * uint64_t(count[i] - 1);
    }
    return e.at <= UINTPTR_MAX - e.bytes;
}

bool shares(const int64_t *count, const int64_t *strides, int axes) {
    for (int i = 0; i < axes; ++i)
        if (count[i] > 1 && strides[i] == 0) return true;
    return false;
}

int64_t code_bytes(const vd_mx4_cache *c) { return c->head_dim / 2; }
int64_t scale_bytes(const vd_mx4_cache *c) { return c->head_dim / vd::kMxGroup; }

vd_status check_cache(const vd_mx4_cache *c, bool written, Extent *extents = nullptr) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return VD_ERR_INVALID_ARG;
    if (c->num_seqs < 1 || c->num_layers < 1 || c->num_kv_heads < 1 || c->num_q_heads < 1) return VD_ERR_INVALID_ARG;
    if (c->num_q_heads % c->num_kv_heads != 0) return VD_ERR_INVALID_ARG;
    if (c->head_dim < 1 || c->capacity < 1) return VD_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return VD_ERR_UNSUPPORTED;
    if (c->capacity > VD_MX4_MAX_CAPACITY) return VD_ERR_UNSUPPORTED;
    if (c->num_layers > 65535 || c->num_kv_heads > 65535) return VD_ERR_UNSUPPORTED;   // grid dimensions
    if (int64_t(c->num_seqs) * c->num_layers * c->num_kv_heads > INT32_MAX) return VD_ERR_UNSUPPORTED;
    const int64_t code[4] = {c->stride_seq, c->stride_layer, c->stride_head, c->stride_slot};
    const int64_t scale[4] = {c->scale_seq, c->scale_layer, c->scale_head, c->scale_slot};
    const int64_t count[4] = {c->num_seqs, c->num_layers, c->num_kv_heads, c->capacity};
    const int64_t cb = code_bytes(c), sb = scale_bytes(c);
    for (int i = 0; i < 4; ++i)
        if (count[i] > 1 || i == 3)
            if (code[i] < 0 || scale[i] < 0 || code[i] % 16 != 0 || scale[i] % sb != 0) return VD_ERR_INVALID_ARG;
    if (code[3] < cb || scale[3] < sb) return VD_ERR_INVALID_ARG;   // rows would overlap
    // a unit's slab is addressed with 32-bit byte offsets
    if (code[3] > int64_t(UINT32_MAX) / c->capacity || scale[3] > int64_t(UINT32_MAX) / c->capacity) return VD_ERR_UNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, sb) || !aligned(c->v_scale, sb)) return VD_ERR_INVALID_ARG;
    if (written && (shares(count, code, 3) || shares(count, scale, 3))) return VD_ERR_INVALID_ARG;
    Extent e[4];
    if (!extent_of(c->k, count, code, 4, cb, e[0]) || !extent_of(c->v, count, code, 4, cb, e[1]) ||
        !extent_of(c->k_scale, count, scale, 4, sb, e[2]) || !extent_of(c->v_scale, count, scale, 4, sb, e[3]))
        return VD_ERR_UNSUPPORTED;
    if (c->k == c->v || c->k_scale == c->v_scale) return VD_ERR_INVALID_ARG;
    if (extents) std::copy(e, e + 4, extents);
    return VD_OK;
}

vd::MxCache first_unit(const vd_mx4_cache *c, int s0) {
    vd::MxCache m;
    m.k = static_cast<char *>(c->k) + s0 * c->stride_seq;
    m.v = static_cast<char *>(c->v) + s0 * c->stride_seq;
    m.ks = static_cast<char *>(c->k_scale) + s0 * c->scale_seq;
    m.vs = static_cast<char *>(c->v_scale) + s0 * c->scale_seq;
    m.seq = c->stride_seq, m.layer = c->stride_layer, m.head = c->stride_head;
    m.sseq = c->scale_seq, m.slayer = c->scale_layer, m.shead = c->scale_head;
    m.slot = uint32_t(c->stride_slot), m.sslot = uint32_t(c->scale_slot);
    m.layers = c->num_layers, m.heads = c->num_kv_heads;
    return m;
}

// Rows of activations: strides in elements on entry, in bytes on return.
vd_status check_rows(const void *base, const int64_t *strides, const int64_t *count, int32_t dtype, int64_t head_dim,
                     int64_t *bytes, Extent &e) {
    if (!base || !strides || !aligned(base, 16)) return VD_ERR_INVALID_ARG;
    const int64_t es = elem_bytes(dtype);
    for (int i = 0; i < 4; ++i) {
        bytes[i] = 0;
        if (count[i] == 1) continue;
        if (strides[i] < 0 || strides[i] > kFar / es / count[i]) return VD_ERR_INVALID_ARG;
        bytes[i] = strides[i] * es;
        if (bytes[i] % 16 != 0) return VD_ERR_INVALID_ARG;
    }
    return extent_of(base, count, bytes, 4, head_dim * es, e) ? VD_OK : VD_ERR_INVALID_ARG;
}

bool known_dtype(int32_t d) { return d == VD_DTYPE_BF16 || d == VD_DTYPE_F32; }

// Shared by append and read.
vd_status rows_call(const vd_mx4_cache *cache, const int32_t *first, const int32_t *rows, int32_t max_rows,
                    int32_t dtype, const void *k_rows, const int64_t *k_strides, const void *v_rows,
                    const int64_t *v_strides, int32_t *pos, const int32_t *pos0, bool append, vd_stream stream) {
    Extent cached[4], mine[2];
    vd_status st = check_cache(cache, append, cached);
    if (st != VD_OK) return st;
    if (!known_dtype(dtype) || !first || max_rows < 1) return VD_ERR_INVALID_ARG;
    if (pos && !aligned(pos, 4)) return VD_ERR_INVALID_ARG;
    for (int s = 0; s < cache->num_seqs; ++s) {
        const int r = rows ? rows[s] : max_rows;
        if (first[s] < 0 || r < 0 || r > max_rows || first[s] > cache->capacity - r) return VD_ERR_INVALID_ARG;
        const int32_t p0 = pos0 ? pos0[s] : first[s];
        if (pos && (p0 < 0 || p0 > INT32_MAX - r)) return VD_ERR_INVALID_ARG;
    }
    vd::MxRowsParams p;
    std::memset(&p, 0, sizeof p);
    const int64_t count[4] = {cache->num_seqs, cache->num_layers, cache->num_kv_heads, max_rows};
    if ((st = check_rows(k_rows, k_strides, count, dtype, cache->head_dim, p.ks, mine[0])) != VD_OK) return st;
    if ((st = check_rows(v_rows, v_strides, count, dtype, cache->head_dim, p.vs, mine[1])) != VD_OK) return st;
    for (const Extent &a : mine)
        for (const Extent &b : cached)
            if (a.meets(b)) return VD_ERR_INVALID_ARG;
    if (!append && (mine[0].at == mine[1].at || shares(count, p.ks, 4) || shares(count, p.vs, 4))) return VD_ERR_INVALID_ARG;
    // threads of a launch, in 32 bits
    if (int64_t(cache->num_layers) * cache->num_kv_heads > INT32_MAX / (cache->head_dim / 8) / max_rows) return VD_ERR_UNSUPPORTED;
    const int64_t units = int64_t(cache->num_layers) * cache->num_kv_heads;
    p.capacity = cache->capacity;
    p.max_rows = max_rows;
    for (int s0 = 0; s0 < cache->num_seqs; s0 += vd::kMxSeqs) {
        const int ns = std::min(vd::kMxSeqs, cache->num_seqs - s0);
        p.c = first_unit(cache, s0);
        p.k = static_cast<char *>(const_cast<void *>(k_rows)) + s0 * p.ks[0];
        p.v = static_cast<char *>(const_cast<void *>(v_rows)) + s0 * p.vs[0];
        p.pos = pos ? pos + s0 * units * cache->capacity : nullptr;
        bool any = false;
        for (int i = 0; i < ns; ++i) {
            p.first[i] = first[s0 + i];
            p.rows[i] = rows ? rows[s0 + i] : max_rows;
            p.pos0[i] = pos0 ? pos0[s0 + i] : first[s0 + i];
            any = any || p.rows[i] > 0;
        }
        if (!any) continue;
        st = launched((append ? vd::launch_mx_append : vd::launch_mx_read)(p, ns, dtype, cache->head_dim,
                                                                            reinterpret_cast<hipStream_t>(stream)));
        if (st != VD_OK) return st;
    }
    return VD_OK;
}

// Tiles of query rows and splits of the cache rows.
struct AttnPlan {
    int block, tiles, splits;
};
AttnPlan attn_plan(const vd_mx4_cache *c, int32_t dtype, int64_t max_rows, int64_t n) {
    const int64_t queries = max_rows * (c->num_q_heads / c->num_kv_heads);
    const int64_t units = int64_t(c->num_seqs) * c->num_layers * c->num_kv_heads;
    AttnPlan a;
    // Up to four tiles of single query rows the wide kernel's idle waves cost more than its
    // tiles of cache rows, converted once for all, save (64 sequences' layers x 8 heads, 4000
    // rows, us, tiles of 16 and blocks: bf16, D = 128, 24 queries 82 and 137, 48 122 and 148, 64
    // 156 and 145, 96 231 and 148; D = 256, 64 315 and 367, 96 466 and 372; fp32, D = 128, 64 200
    // and 283, 96 - and 297).  Three parts of 256 channels do not fit its registers.
    a.block = queries > 4 * vd::kMxTile && !(dtype == VD_DTYPE_F32 && c->head_dim == 256);
    const int64_t tile = a.block ? vd::kMxBlockTile : vd::kMxTile;
    a.tiles = int((queries + tile - 1) / tile);
    // Splits where the launch has fewer workgroups than the CUs hold: as many as make two on
    // each (of blocks, as many as are resident).  More cost the join what they save (one
    // sequence of 131072 rows, 8 units, two and four workgroups a CU 33.9 and 36.2 us; sixteen
    // of up to 4097, 128 units, 17.6 and 17.8, eight 19.0).
    const int64_t groups = units * a.tiles, resident = (a.block ? vd::block_groups(dtype, c->head_dim) : 2) * 256;
    a.splits = int(std::max<int64_t>(1, std::min<int64_t>({vd::kMxMaxSplits, resident / groups, n / 256})));
    return a;
}
// [unit][split][query row]: D sums, then two floats each.
size_t attn_ws(const vd_mx4_cache *c, int64_t max_rows, const AttnPlan &a) {
    if (a.splits == 1) return 0;
    const int64_t parts = int64_t(c->num_seqs) * c->num_layers * c->num_q_heads * max_rows * a.splits;
    return size_t(parts * (c->head_dim + 2) * 4);
}
vd_status check_queries(const vd_mx4_cache *c, int32_t dtype, int32_t max_rows) {
    if (!known_dtype(dtype) || max_rows < 1) return VD_ERR_INVALID_ARG;
    // query rows of a unit, and threads of a launch along a grid's first axis, in 32 bits
    if (int64_t(max_rows) * (c->num_q_heads / c->num_kv_heads) > (1 << 26)) return VD_ERR_UNSUPPORTED;
    return VD_OK;
}

}  // namespace

extern "C" vd_status vd_append_mx4(const vd_mx4_cache *cache, const int32_t *n_old, const int32_t *rows, int32_t max_rows,
                                   int32_t dtype, const void *k_rows, const int64_t *k_strides, const void *v_rows,
                                   const int64_t *v_strides, int32_t *pos, const int32_t *pos0, vd_stream stream) {
    return rows_call(cache, n_old, rows, max_rows, dtype, k_rows, k_strides, v_rows, v_strides, pos, pos0, true, stream);
}

extern "C" vd_status vd_read_mx4(const vd_mx4_cache *cache, const int32_t *first, const int32_t *rows, int32_t max_rows,
                                 int32_t dtype, void *k_rows, const int64_t *k_strides, void *v_rows,
                                 const int64_t *v_strides, vd_stream stream) {
    return rows_call(cache, first, rows, max_rows, dtype, k_rows, k_strides, v_rows, v_strides, nullptr, nullptr, false, stream);
}

extern "C" size_t vd_attention_mx4_workspace_size(const vd_mx4_cache *cache, int32_t dtype, int32_t max_rows, int32_t n) {
    if (check_cache(cache, false) != VD_OK || check_queries(cache, dtype, max_rows) != VD_OK || n < 0 || n > cache->capacity) return 0;
    return attn_ws(cache, max_rows, attn_plan(cache, dtype, max_rows, n));
}

extern "C" vd_status vd_attention_mx4(const vd_mx4_cache *cache, int32_t dtype, const void *q, const int64_t *q_strides,
                                      int32_t max_rows, const int32_t *rows, float scale, const int32_t *n_valid, void *out,
                                      const int64_t *out_strides, void *workspace, size_t workspace_bytes,
                                      vd_stream stream) {
    Extent cached[4], qe, oe;
    vd_status st = check_cache(cache, false, cached);
    if (st != VD_OK) return st;
    if ((st = check_queries(cache, dtype, max_rows)) != VD_OK) return st;
    if (!n_valid || !std::isfinite(scale)) return VD_ERR_INVALID_ARG;
    int n = 0;
    for (int s = 0; s < cache->num_seqs; ++s) {
        if (n_valid[s] < 0 || n_valid[s] > cache->capacity) return VD_ERR_INVALID_ARG;
        if (rows && (rows[s] < 0 || rows[s] > max_rows)) return VD_ERR_INVALID_ARG;
        n = std::max(n, n_valid[s]);
    }
    vd::MxAttnParams p;
    std::memset(&p, 0, sizeof p);
    const int64_t count[4] = {cache->num_seqs, cache->num_layers, cache->num_q_heads, max_rows};
    if ((st = check_rows(q, q_strides, count, dtype, cache->head_dim, p.qs, qe)) != VD_OK) return st;
    if ((st = check_rows(out, out_strides, count, dtype, cache->head_dim, p.os, oe)) != VD_OK) return st;
    if (shares(count, p.os, 4) || oe.meets(qe)) return VD_ERR_INVALID_ARG;
    for (const Extent &c : cached)
        if (oe.meets(c)) return VD_ERR_INVALID_ARG;
    const AttnPlan a = attn_plan(cache, dtype, max_rows, n);
    const size_t need = attn_ws(cache, max_rows, a);
    if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return VD_ERR_WORKSPACE;
    const int64_t L = cache->num_layers, per_seq = L * cache->num_q_heads * max_rows * a.splits;   // partial rows
    const int64_t parts = per_seq * cache->num_seqs;
    // (a positive number: a hidden row's logit of -infinity times it stays that)
    p.qscale = float(std::clamp(std::fabs(double(scale)) * 1.4426950408889634, double(FLT_MIN), double(FLT_MAX)));  // log2(e)
    p.flip = scale < 0 ? 0x80000000u : 0u;
    p.group = cache->num_q_heads / cache->num_kv_heads;
    p.max_rows = max_rows;
    p.splits = a.splits;
    p.tiles = a.tiles;
    p.block = a.block;
    const int chunk = std::max(1, std::min(vd::kMxSeqs, int(65535 / L)));
    for (int s0 = 0; s0 < cache->num_seqs; s0 += chunk) {
        const int ns = std::min(chunk, cache->num_seqs - s0);
        p.c = first_unit(cache, s0);
        p.q = static_cast<const char *>(q) + s0 * p.qs[0];
        p.out = static_cast<char *>(out) + s0 * p.os[0];
        if (need) {
            p.ws_acc = static_cast<float *>(workspace) + s0 * per_seq * cache->head_dim;
            p.ws_ml = static_cast<float *>(workspace) + parts * cache->head_dim + s0 * per_seq * 2;
        }
        for (int i = 0; i < ns; ++i) {
            p.n[i] = n_valid[s0 + i];
            p.rows[i] = rows ? rows[s0 + i] : max_rows;
        }
        st = launched(vd::launch_mx_attention(p, ns, dtype, cache->head_dim, reinterpret_cast<hipStream_t>(stream)));
        if (st != VD_OK) return st;
    }
    return VD_OK;
}

extern "C" vd_status vd_evict_step_mx4(const vd_mx4_cache *cache, const int32_t *n_valid, const int32_t *budget,
                                       vd_variant variant, int32_t *pos, float *scores_out, uint8_t *keep_out,
                                       vd_stream stream) {
    vd_status st = check_cache(cache, true);
    if (st != VD_OK) return st;
    if (cache->capacity > VD_MAX_CAPACITY) return VD_ERR_UNSUPPORTED;
    if (!n_valid || !budget || variant < VD_SCORE_L2 || variant > VD_SCORE_KEY_NORM) return VD_ERR_INVALID_ARG;
    for (int s = 0; s < cache->num_seqs; ++s)
        if (n_valid[s] < 0 || n_valid[s] > cache->capacity || budget[s] < 1) return VD_ERR_INVALID_ARG;
    if ((pos && !aligned(pos, 4)) || (scores_out && !aligned(scores_out, 4))) return VD_ERR_INVALID_ARG;
    const int64_t units = int64_t(cache->num_layers) * cache->num_kv_heads;
    vd::MxEvictParams p;
    std::memset(&p, 0, sizeof p);
    p.capacity = cache->capacity;
    p.variant = variant;
    for (int s0 = 0; s0 < cache->num_seqs; s0 += vd::kMxSeqs) {
        const int ns = std::min(vd::kMxSeqs, cache->num_seqs - s0);
        const int64_t at = s0 * units * cache->capacity;
        p.c = first_unit(cache, s0);
        p.pos = pos ? pos + at : nullptr;
        p.scores = scores_out ? scores_out + at : nullptr;
        p.keep = keep_out ? keep_out + at : nullptr;
        int keys = 0, moves = 0;
        bool any = false;
        for (int i = 0; i < ns; ++i) {
            const int n = p.n[i] = n_valid[s0 + i], N = p.budget[i] = budget[s0 + i];
            any = any || (n > 0 && (n > N || scores_out || keep_out));
            if (n > N) {
                keys = std::max(keys, n);
                moves = std::max(moves, std::min(N, n - N));
            }
        }
        if (!any) continue;
        // Keys (the sums' partials lie there before them), then two lists of 16-bit slots.
        // More units than CUs: two workgroups of half the threads on a CU, if its LDS holds
        // both (12 KB each beside this), so that one's selection and gather run beside
        // another's rows (1024 units of 4097 rows, one evicted, 154 and 124 us).
        size_t lds = 0;
        for (int threads : {vd::kMxEvictThreads / 2, vd::kMxEvictThreads}) {
            const int64_t partial = int64_t(threads / 64) * cache->head_dim * 8;
            p.threads = threads;
            p.off_lists = int32_t(std::max(align16(int64_t(keys) * 4), partial));
            p.list_cap = moves;
            lds = size_t(p.off_lists + align16(int64_t(moves) * 4));
            if (units * ns > 256 && lds + 12 * 1024 <= 80 * 1024) break;
        }
        st = launched(vd::launch_mx_evict(p, ns, cache->head_dim, lds, reinterpret_cast<hipStream_t>(stream)));
        if (st != VD_OK) return st;
    }
    return VD_OK;
}

extern "C" vd_status vd_qk_norm_rope(const vd_rope_args *a, vd_stream stream) {
    if (!a || (!a->q.x && !a->k.x) || !a->pos || !aligned(a->pos, 4)) return VD_ERR_INVALID_ARG;
    if (!known_dtype(a->dtype) || !known_dtype(a->weight_dtype)) return VD_ERR_INVALID_ARG;
    if (a->num_seqs < 1 || a->num_layers < 1 || a->rows < 1 || a->head_dim < 1) return VD_ERR_INVALID_ARG;
    if (a->head_dim != 64 && a->head_dim != 128 && a->head_dim != 256) return VD_ERR_UNSUPPORTED;
    if (a->rotary < 8 || a->rotary > a->head_dim || a->rotary % 8 != 0) return VD_ERR_INVALID_ARG;
    if (a->interleaved != 0 && a->interleaved != 1) return VD_ERR_INVALID_ARG;
    if (!a->inv_freq || !aligned(a->inv_freq, 16)) return VD_ERR_INVALID_ARG;
    if (!std::isfinite(a->eps) || a->eps < 0) return VD_ERR_INVALID_ARG;
    vd::RopeParams p;
    std::memset(&p, 0, sizeof p);
    const vd_rope_side *from[2] = {&a->q, &a->k};
    vd::RopeSide *to[2] = {&p.q, &p.k};
    Extent written[2];
    int sides = 0;
    for (int i = 0; i < 2; ++i) {
        const vd_rope_side &f = *from[i];
        if (!f.x) {
            if (f.out) return VD_ERR_INVALID_ARG;
            continue;
        }
        if (f.heads < 1 || !known_dtype(f.out_dtype) || (f.weight && !aligned(f.weight, 16))) return VD_ERR_INVALID_ARG;
        const int64_t count[4] = {a->num_seqs, a->num_layers, f.heads, a->rows};
        Extent x;
        vd_status st = check_rows(f.x, f.strides, count, a->dtype, a->head_dim, to[i]->xs, x);
        if (st != VD_OK) return st;
        if ((st = check_rows(f.out, f.out_strides, count, f.out_dtype, a->head_dim, to[i]->ys, written[sides])) != VD_OK) return st;
        if (shares(count, to[i]->ys, 4)) return VD_ERR_INVALID_ARG;
        const bool in_place = f.out == f.x && f.out_dtype == a->dtype && std::equal(to[i]->xs, to[i]->xs + 4, to[i]->ys);
        if (!in_place && x.meets(written[sides])) return VD_ERR_INVALID_ARG;
        to[i]->x = static_cast<const char *>(f.x);
        to[i]->y = static_cast<char *>(f.out);
        to[i]->w = static_cast<const char *>(f.weight);
        to[i]->heads = f.heads;
        to[i]->y_dtype = f.out_dtype;
        ++sides;
    }
    if (a->q.x && a->k.x && a->q.out == a->k.out) return VD_ERR_INVALID_ARG;
    p.pos = a->pos;
    p.inv_freq = a->inv_freq;
    p.rows = a->rows;
    p.layers = a->num_layers;
    p.rotary = a->rotary;
    p.w_dtype = a->weight_dtype;
    p.eps = a->eps;
    const int64_t tokens = int64_t(a->num_seqs) * a->rows, heads = int64_t(p.q.heads) + p.k.heads;
    if (heads > INT32_MAX / a->num_layers || tokens > INT32_MAX / 2) return VD_ERR_UNSUPPORTED;
    const int64_t all = heads * a->num_layers, lanes = a->head_dim / 8;
    // Rows of a token that one group of lanes takes, whose cos and sin it makes once:
    // about 4 KB of them, read and written, but only as many as leave about sixteen waves
    // for each CU.  More make the groups' paths through memory long and scattered (us, rows
    // 1, 2, 4, 8, 16: 512 tokens x 1280 rows of 128 bf16 channels 111, 84, 73, 71, 78; 999
    // tokens x 156 of 256 fp32 channels 60, 62, 67, 69, 68).
    const int64_t groups = int64_t(256) * 16 * 64 / lanes;
    const int64_t bytes = a->head_dim * (elem_bytes(a->dtype) + elem_bytes(a->q.x ? a->q.out_dtype : a->k.out_dtype));
    const int64_t most = std::max<int64_t>(1, 4096 / bytes);
    p.tokens = int32_t(tokens);
    p.per_item = int32_t(std::max<int64_t>(1, std::min<int64_t>(most, tokens * all / groups)));
    p.items = int32_t((all + p.per_item - 1) / p.per_item);
    if (tokens * p.items > INT32_MAX) return VD_ERR_UNSUPPORTED;
    return launched(vd::launch_rope(p, a->dtype, a->head_dim, a->interleaved != 0, reinterpret_cast<hipStream_t>(stream)));
}
