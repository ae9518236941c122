// Runs the host side of the 4-bit cache and of the rotated rows under the
// sanitizers, the device launches replaced by stubs that check their parameters
// and report no device.  Built and run by tests/test_mx4_cpu.py.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstring>
#include <vector>

#include "vd.h"
#include "vd_mx4.h"

static int failures = 0, launches = 0;
#define EXPECT(x)                                                                \
    do {                                                                         \
        if (!(x)) {                                                              \
            std::fprintf(stderr, "expectation failed at line %d: %s\n", __LINE__, #x); \
            ++failures;                                                          \
        }                                                                        \
    } while (0)

namespace vd {
hipError_t launch_mx_append(const MxRowsParams &p, int seqs, int, int, hipStream_t) {
    ++launches;
    EXPECT(seqs >= 1 && seqs <= kMxSeqs);
    for (int s = 0; s < seqs; ++s) EXPECT(p.first[s] >= 0 && p.rows[s] >= 0 && p.rows[s] <= p.max_rows && p.first[s] + p.rows[s] <= p.capacity);
    return hipSuccess;
}
hipError_t launch_mx_read(const MxRowsParams &p, int seqs, int dtype, int D, hipStream_t s) { return launch_mx_append(p, seqs, dtype, D, s); }
hipError_t launch_mx_attention(const MxAttnParams &p, int seqs, int, int, hipStream_t) {
    ++launches;
    EXPECT(seqs >= 1 && seqs <= kMxSeqs && int64_t(seqs) * p.c.layers <= 65535);
    EXPECT(p.splits >= 1 && p.splits <= kMxMaxSplits && p.tiles >= 1);
    EXPECT(p.tiles * (p.block ? kMxBlockTile : kMxTile) >= p.max_rows * p.group);
    EXPECT((p.splits > 1) == (p.ws_acc != nullptr) && p.qscale > 0);
    return hipSuccess;
}
hipError_t launch_mx_evict(const MxEvictParams &p, int seqs, int D, size_t lds, hipStream_t) {
    ++launches;
    EXPECT(seqs >= 1 && seqs <= kMxSeqs && lds + 12 * 1024 <= 160 * 1024);
    EXPECT(p.threads == kMxEvictThreads || p.threads == kMxEvictThreads / 2);
    EXPECT(p.off_lists >= p.threads / 64 * D * 8 && p.off_lists % 16 == 0);
    for (int s = 0; s < seqs; ++s)
        if (p.n[s] > p.budget[s]) {
            const int moves = p.n[s] - p.budget[s] < p.budget[s] ? p.n[s] - p.budget[s] : p.budget[s];
            EXPECT(p.off_lists >= p.n[s] * 4 && p.list_cap >= moves && lds >= size_t(p.off_lists) + size_t(p.list_cap) * 4);
        }
    return hipSuccess;
}
hipError_t launch_rope(const RopeParams &p, int, int, bool, hipStream_t) {
    ++launches;
    EXPECT(p.per_item >= 1 && int64_t(p.items) * p.per_item >= int64_t(p.layers) * (p.q.heads + p.k.heads));
    EXPECT(int64_t(p.tokens) * p.items <= INT32_MAX);
    return hipErrorNoDevice;
}
}  // namespace vd

static char *at(unsigned long long x) { return reinterpret_cast<char *>(0x700000000000ull + x); }

static vd_mx4_cache cache(int S, int L, int H, int Hq, int D, int C) {
    vd_mx4_cache c;
    std::memset(&c, 0, sizeof c);
    c.k = at(0), c.v = at(1ull << 38), c.k_scale = at(2ull << 38), c.v_scale = at(3ull << 38);
    c.num_seqs = S, c.num_layers = L, c.num_kv_heads = H, c.num_q_heads = Hq, c.head_dim = D, c.capacity = C;
    c.stride_slot = D / 2, c.stride_head = c.stride_slot * C, c.stride_layer = c.stride_head * H, c.stride_seq = c.stride_layer * L;
    c.scale_slot = D / 32, c.scale_head = c.scale_slot * C, c.scale_layer = c.scale_head * H, c.scale_seq = c.scale_layer * L;
    return c;
}

int main() {
    for (int D : {64, 128, 256})
        for (int S : {1, 3, 300})
            for (int C : {1, 700, 16384}) {
                const int L = S == 300 ? 400 : 2, H = 2, G = 3;
                const vd_mx4_cache c = cache(S, L, H, H * G, D, C);
                std::vector<int32_t> n(S), N(S), rows(S), zero(S, 0);
                for (int s = 0; s < S; ++s) n[s] = C - s % 3 > 0 ? C - s % 3 : 0, N[s] = 1 + (s * 37) % C, rows[s] = s % 2;
                for (int t : {1, 7, 200})
                    for (int dtype : {0, 1}) {
                        const int64_t q[4] = {int64_t(L) * H * G * t * D, int64_t(H) * G * t * D, int64_t(t) * D, D};
                        const size_t size = vd_attention_mx4_workspace_size(&c, dtype, t, C);
                        const vd_status st = vd_attention_mx4(&c, dtype, at(5ull << 38), q, t, rows.data(), -0.1f, n.data(), at(6ull << 38), q,
                                                              at(7ull << 38), size, nullptr);
                        EXPECT(st == VD_OK);
                        const int64_t r[4] = {int64_t(L) * H * t * D, int64_t(H) * t * D, int64_t(t) * D, D};
                        if (t <= C) {
                            EXPECT(vd_append_mx4(&c, zero.data(), nullptr, t, dtype, at(5ull << 38), r, at(6ull << 38), r,
                                                 reinterpret_cast<int32_t *>(at(7ull << 38)), n.data(), nullptr) == VD_OK);
                            EXPECT(vd_read_mx4(&c, zero.data(), rows.data(), t, dtype, at(5ull << 38), r, at(6ull << 38), r, nullptr) == VD_OK);
                        }
                    }
                for (int variant = VD_SCORE_L2; variant <= VD_SCORE_KEY_NORM; ++variant)
                    EXPECT(vd_evict_step_mx4(&c, n.data(), N.data(), vd_variant(variant), nullptr, nullptr, nullptr, nullptr) == VD_OK);
                // nothing to do: nothing is queued
                const int before = launches;
                EXPECT(vd_evict_step_mx4(&c, zero.data(), N.data(), VD_SCORE_L2, nullptr, nullptr, nullptr, nullptr) == VD_OK);
                const int64_t r[4] = {0, 0, 0, D};
                EXPECT(vd_append_mx4(&c, zero.data(), zero.data(), 1, 0, at(5ull << 38), r, at(6ull << 38), r, nullptr, nullptr, nullptr) == VD_OK);
                EXPECT(launches == before);
            }
    vd_rope_args a;
    std::memset(&a, 0, sizeof a);
    a.pos = reinterpret_cast<int32_t *>(at(0)), a.inv_freq = reinterpret_cast<float *>(at(0));
    a.num_seqs = 64, a.num_layers = 36, a.rows = 1024, a.head_dim = 128, a.rotary = 128;
    a.q.x = at(1ull << 38), a.q.out = at(2ull << 38), a.q.heads = 32;
    const int64_t q[4] = {36ll * 32 * 1024 * 128, 32ll * 1024 * 128, 1024 * 128, 128};
    std::memcpy(a.q.strides, q, sizeof q);
    std::memcpy(a.q.out_strides, q, sizeof q);
    EXPECT(vd_qk_norm_rope(&a, nullptr) == VD_ERR_HIP);   // (the stub's answer)
    a.num_seqs = 1, a.num_layers = 1, a.rows = 1;
    EXPECT(vd_qk_norm_rope(&a, nullptr) == VD_ERR_HIP);
    EXPECT(vd_qk_norm_rope(nullptr, nullptr) == VD_ERR_INVALID_ARG);
    if (failures) return 1;
    std::printf("mx4 sanitizer run ok (%d launches)\n", launches);
    return 0;
}
