// Every launch that kvr_continue_shared, kvr_cache_weigh and kvr_cache_evict plan, up to the
// sizes that kvr.h says are served, has fewer than 2^32 threads, which a launch must not
// exceed.  Host code alone: the launchers are stubs that work the grids out as the kernels'
// own do, and fail (KVR_ERR_DEVICE: the call was accepted).
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "kvr.h"
#include "kvr_internal.hpp"
#include "readers/readers_internal.hpp"

static int g_bad = 0, g_launches = 0;
static const char *g_call = "";

static void threads(const char *kernel, int64_t blocks, int64_t per_block) {
    if (blocks > 0 && blocks <= 0x7fffffff && blocks * per_block < ((int64_t)1 << 32)) return;
    ++g_bad;
    fprintf(stderr, "%s: %s with %lld blocks of %lld threads\n", g_call, kernel, (long long)blocks, (long long)per_block);
}
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

namespace kvr {
hipError_t launch_attn_bf16(const AttnParams &, int, int, bool, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_merge_bf16(const MergeParams &, int, bool, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_attn_pp(const AttnParams &, int, bool, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_attn_pk(const AttnParams &, int, bool, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_attn_rows(const AttnParams &, bool, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_attn_cont(const AttnParams &, int, bool, bool, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_quantize(const QuantParams &, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_attn_f32(const AttnParams &, int, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_append(const AppendParams &, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_rope(const RopeParams &, int, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_rope_table(float *, int, double, int64_t, hipStream_t) { return hipErrorUnknown; }

hipError_t launch_shared(const SharedParams &p, int head_dim, int, int pw, int, hipStream_t) {
    ++g_launches;
    if (pw == kAlone) {
        threads("a workgroup a reader and kv head", (int64_t)p.n * p.n_kv_heads, 512);
        return hipErrorUnknown;
    }
    threads("items", (int64_t)p.oct_all * 8, 256);
    threads("merge", ceil_div(p.rows, 256 / head_dim), 256);
    return hipErrorUnknown;
}
hipError_t launch_weigh(const WeighParams &p, int, int dtype, int way, int held, hipStream_t) {
    ++g_launches;
    const int64_t rows = (int64_t)p.S * p.group, keys = dtype == KVR_F32 ? 16 : 32;
    threads("stats", ceil_div(rows, way > kByRows ? 64 * (way - kByRows) : 16 * way) * p.nsplit * p.n_kv_heads, 256);
    if (p.norm) threads("norms", ceil_div(rows * p.n_kv_heads, 32), 256);
    threads("sums", ceil_div(ceil_div(p.L, keys) + ceil_div(p.S, keys), 4 * held) * p.n_kv_heads, 256);
    return hipErrorUnknown;
}
hipError_t launch_evict(const EvictParams &p, hipStream_t) {
    ++g_launches;
    threads("search and copy", (int64_t)p.n_kv_heads * (p.L <= kHeldRows ? p.parts : 1), 1024);
    return hipErrorUnknown;
}
}  // namespace kvr

int main() {
    void *const A = (void *)(uintptr_t)0x10000;
    static const int heads[][2] = {{1, 1}, {2, 1}, {8, 8}, {32, 8}, {64, 1}, {12, 3}, {4096, 4096}, {4096, 1}};
    const size_t all = (size_t)1 << 62;
    char name[200];
    g_call = name;
    for (const auto &h : heads)
        for (int dtype = 0; dtype < 3; ++dtype)
            for (int d = 64; d <= 128; d += 64) {
                kvr_desc desc;
                memset(&desc, 0, sizeof desc);
                desc.n_q_heads = h[0];
                desc.n_kv_heads = h[1];
                desc.head_dim = d;
                desc.dtype = dtype;
                desc.capacity = (int64_t)1 << 31;
                // readers: all sizes that are served, and those where the call may be refused but not mistaken
                for (int64_t rows : {(int64_t)4096, (int64_t)1 << 20, ((int64_t)1 << 23) - 1, ((int64_t)1 << 24) - 1})
                    for (int64_t S : {1, 4, 100})
                        for (int64_t L : {0, 1, 600, 100000, 0x7fffffff})
                            for (int64_t tcap : {0, 1, 40, 100000, 0x7fffffff}) {
                                const int64_t n = rows / h[0] / S;
                                if (n < 1) continue;
                                snprintf(name, sizeof name, "shared: %d / %d heads of %d, type %d, %lld readers x %lld, L %lld, room %lld", h[0], h[1],
                                         d, dtype, (long long)n, (long long)S, (long long)L, (long long)tcap);
                                const int before = g_launches;
                                const int st = kvr_continue_shared(&desc, nullptr, A, A, A, (int32_t)n, (int32_t)S, A, A, L, 0, A, A, tcap,
                                                                   (const int32_t *)A, 0, A, A, all, nullptr);
                                if (st != (g_launches > before ? KVR_ERR_DEVICE : KVR_ERR_SHAPE) || (st == KVR_ERR_SHAPE && rows < (1 << 23))) {
                                    ++g_bad;
                                    fprintf(stderr, "%s: status %d\n", name, st);
                                }
                            }
                for (int64_t total : {(int64_t)4096, (int64_t)1 << 20, ((int64_t)1 << 28) - 1, ((int64_t)1 << 29) + 4096, (int64_t)1 << 31})
                    for (int64_t L : {(int64_t)0, (int64_t)1, (int64_t)100000, ((int64_t)1 << 28) / h[1] - 1}) {
                        int64_t S = total / h[0];
                        if (S < 1) continue;
                        const bool served = total < (1 << 28) && (L + S) * h[1] < (1 << 28);
                        snprintf(name, sizeof name, "weigh: %d / %d heads of %d, type %d, %lld tokens, L %lld", h[0], h[1], d, dtype, (long long)S,
                                 (long long)L);
                        const int before = g_launches;
                        const int st = kvr_cache_weigh(&desc, A, A, A, L, S, (float *)A, A, all, nullptr);
                        const int want = g_launches > before ? KVR_ERR_DEVICE : KVR_ERR_SHAPE;
                        if (st != want && !(st == KVR_ERR_CAPACITY && L + S > desc.capacity) || (st == KVR_ERR_SHAPE && served)) {
                            ++g_bad;
                            fprintf(stderr, "%s: status %d\n", name, st);
                        }
                    }
            }
    printf("%d launches\n", g_launches);
    if (g_bad || g_launches < 1000) return 1;
    printf("all checks passed\n");
    return 0;
}
