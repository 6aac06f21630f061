// Drives the host side of kvr_continue_shared, kvr_cache_weigh and kvr_cache_evict
// (readers_api.hip) under AddressSanitizer and UndefinedBehaviorSanitizer, without a
// GPU.  The kernel launchers are stubs that check the plan they are given and fail: a
// call with valid arguments ends in KVR_ERR_DEVICE, a rejected one reaches no launcher.
// Device pointers are fake aligned integers and are never dereferenced.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <vector>

#include "kvr.h"
#include "kvr_internal.hpp"
#include "readers/readers_internal.hpp"

static int g_launches = 0, g_bad = 0;
static size_t g_ws_given = 0;

#define BAD(...) (++g_bad, fprintf(stderr, __VA_ARGS__), fputc('\n', stderr))

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

// The grid's blocks, decoded as the kernel decodes them, name every prefix item and
// every own item exactly once; splits cover the prefix; records fit the workspace.
hipError_t launch_shared(const SharedParams &p, int head_dim, int dtype, int pw, int ow, hipStream_t) {
    ++g_launches;
    const int64_t G = p.group, rows_p = (int64_t)p.n * p.S * G, rows_o = (int64_t)p.S * G;
    const bool f32 = dtype == KVR_F32;
    if (pw == kAlone) {      // a workgroup for each reader and kv head
        const int64_t keys = f32 ? 16 : 32;
        if (rows_o > 16 || (p.L + keys - 1) / keys + (p.tcap + keys - 1) / keys > 20) BAD("alone");
        if ((int64_t)p.n * p.n_kv_heads > 0xffffff) BAD("alone: grid");
        return hipErrorUnknown;
    }
    const int64_t tp = pw > kByRows ? 64 * (pw - kByRows) : 16 * pw, to = ow > kByRows ? 64 * (ow - kByRows) : 16 * ow;
    if (ow > pw || (f32 ? pw > 2 : pw == 2 || ow == 2 || pw > kByRows + 2 || ow > kByRows + 1)) BAD("ways %d %d", pw, ow);
    if (p.p_tiles != (rows_p + tp - 1) / tp || p.t_tiles != (rows_o + to - 1) / to) BAD("tiles");
    if (p.rows != (int64_t)p.n * p.S * p.n_q_heads || p.rows > 0x7fffffff) BAD("rows");
    if (p.nrec != p.np + p.nt + 1 || p.nt < 0 || (p.tcap > 0 && p.nt < 1)) BAD("records");
    if ((p.L == 0) != (p.np == 0)) BAD("no split of a prefix");
    if (p.np && ((int64_t)p.np * p.chunk < p.L || (int64_t)(p.np - 1) * p.chunk >= p.L)) BAD("prefix splits");
    if ((size_t)p.nrec * p.rows * (head_dim + 2) * 4 > g_ws_given) BAD("workspace");
    const int64_t own = (int64_t)p.n * p.t_tiles * p.n_kv_heads * p.nt;
    const int64_t pre = (int64_t)p.np * p.n_kv_heads * p.p_tiles;
    const int64_t fresh = (int64_t)p.n * p.n_kv_heads * ((rows_o + 15) / 16);
    if (p.oct_all * (int64_t)8 > 0x7fffffff) BAD("grid");
    if (p.oct_all < 100000) {
        std::vector<uint8_t> seen_o((size_t)own), seen_p((size_t)pre), seen_n((size_t)fresh);
        for (uint32_t oct = 0; oct < p.oct_all; ++oct)
            for (uint32_t in8 = 0; in8 < 8; ++in8)
                for (uint32_t wave = 0; wave < 4; ++wave) {
                    if (oct < p.oct_own) {
                        const uint32_t pair = oct / p.p_tiles * 8 + in8;
                        const int64_t split = pair / p.n_kv_heads;
                        if (wave == 0 && split < p.np) ++seen_p[(size_t)pair * p.p_tiles + oct % p.p_tiles];
                    } else if (oct < p.oct_new) {
                        const int64_t b = (int64_t)(oct - p.oct_own) * 8 + in8;
                        if (wave == 0 && b < own) ++seen_o[(size_t)b];            // past the last: split >= nt
                    } else {
                        const int64_t b = (int64_t)((oct - p.oct_new) * 8 + in8) * 4 + wave;
                        if (b < fresh) ++seen_n[(size_t)b];                       // past the last: reader >= n
                    }
                }
        for (uint8_t x : seen_o) if (x != 1) { BAD("own item seen %d times", x); break; }
        for (uint8_t x : seen_p) if (x != 1) { BAD("prefix item seen %d times", x); break; }
        for (uint8_t x : seen_n) if (x != 1) { BAD("new item seen %d times", x); break; }
    }
    return hipErrorUnknown;
}
hipError_t launch_weigh(const WeighParams &p, int, int dtype, int way, int held, hipStream_t) {
    ++g_launches;
    const int64_t keys = dtype == KVR_F32 ? 16 : 32;
    const int64_t stages = (p.L + keys - 1) / keys + (p.S + keys - 1) / keys, rows = (int64_t)p.S * p.group;
    if ((int64_t)p.nsplit * p.chunk < stages || (int64_t)(p.nsplit - 1) * p.chunk >= stages) BAD("weigh splits");
    if ((size_t)p.nsplit * p.n_kv_heads * rows * 8 > g_ws_given) BAD("weigh workspace");
    const int64_t per = way > kByRows ? 64 * (way - kByRows) : 16 * way;
    if ((rows + per - 1) / per * p.nsplit * p.n_kv_heads > 0x7fffffff) BAD("weigh grid");
    const bool f32 = dtype == KVR_F32;
    const bool direct = way == 1 || (f32 && way == 2), ring = !f32 && (way == kByRows + 2 || way == kByRows + 4);
    if ((!direct && !ring) || (held != 1 && (held != 2 || !f32))) BAD("weigh way %d %d", way, held);
    return hipErrorUnknown;
}
hipError_t launch_evict(const EvictParams &p, hipStream_t) {
    ++g_launches;
    if (p.n_first + p.n_last > p.n_keep || p.n_keep > p.L || p.L > p.cap || p.n_keep > p.cap_out) BAD("evict rows");
    if (p.L > kHeldRows && (size_t)p.n_kv_heads * p.n_keep * 4 > g_ws_given) BAD("evict workspace");
    if (p.L <= kHeldRows && (p.parts < 1 || (int64_t)p.parts * p.n_kv_heads > 0x7fffffff)) BAD("evict grid");
    if (p.row_chunks != 1 << p.chunk_bits) BAD("evict chunks");
    return hipErrorUnknown;
}
}  // namespace kvr

static uint64_t g_rng = 88172645463325252ull;
static uint64_t rnd(uint64_t n) {
    g_rng ^= g_rng << 13;
    g_rng ^= g_rng >> 7;
    g_rng ^= g_rng << 17;
    return g_rng % n;
}
static int64_t odd_size() {
    static const int64_t v[] = {-1, 0, 1, 2, 15, 16, 17, 31, 32, 33, 100, 255, 3774, 32768, 1 << 20,
                                0x7fffffff, (int64_t)1 << 31, (int64_t)1 << 40, INT64_MAX, INT64_MIN};
    return v[rnd(sizeof v / sizeof v[0])];
}

int main() {
    void *const A = (void *)(uintptr_t)0x10000;
    int n_ok = 0, n_rej = 0;
    size_t last_shared = 0, last_weigh = 0;
    for (int it = 0; it < 60000; ++it) {
        kvr_desc d;
        memset(&d, 0, sizeof d);
        static const int heads[][2] = {{32, 8}, {8, 8}, {12, 3}, {64, 8}, {16, 2}, {1, 1}, {4096, 1}, {4096, 4096}, {30, 8}, {0, 1}};
        const int h = (int)rnd(10);
        d.n_q_heads = heads[h][0];
        d.n_kv_heads = heads[h][1];
        d.head_dim = rnd(8) ? (rnd(2) ? 64 : 128) : (int)rnd(300);
        d.dtype = rnd(8) ? (int)rnd(3) : (int)rnd(10) - 3;
        d.capacity = rnd(4) ? 40000 : odd_size();
        const bool wild = rnd(2);
        const int64_t L = wild ? odd_size() : (int64_t)rnd(40000), tcap = wild ? odd_size() : (int64_t)rnd(3000);
        const int32_t n = wild ? (int32_t)odd_size() : (int32_t)rnd(80), S = wild ? (int32_t)odd_size() : (int32_t)rnd(70);
        const kvr_rope rope = {(const float *)A, wild ? odd_size() : 100000};
        const int before = g_launches;
        const size_t nb = kvr_workspace_bytes_shared(&d, L, n, S, tcap);
        g_ws_given = nb == (size_t)-1 ? (size_t)1 << 40 : nb;
        const int st = kvr_continue_shared(&d, rnd(2) ? &rope : nullptr, A, A, A, n, S, A, A, L, wild ? odd_size() : L, A, A,
                                           tcap, (const int32_t *)A, (int)rnd(2), A, A, g_ws_given, nullptr);
        if ((st == KVR_ERR_DEVICE) != (g_launches > before)) BAD("shared: status %d, launches %d", st, g_launches - before);
        if (nb == (size_t)-1 && st != KVR_ERR_SHAPE && st != KVR_ERR_DTYPE) BAD("shared: no workspace size, status %d", st);
        if (st == KVR_ERR_DEVICE) {
            ++n_ok;
            const int b2 = g_launches;
            if (kvr_continue_shared(&d, nullptr, A, A, A, n, S, A, A, L, 0, A, A, tcap, (const int32_t *)A, 0, A, A, nb - 1,
                                    nullptr) != KVR_ERR_WORKSPACE || g_launches != b2) BAD("shared: short workspace");
            // never less for a longer prefix or longer own rows
            last_shared = kvr_workspace_bytes_shared(&d, L + (int64_t)rnd(500), n, S, tcap + (int64_t)rnd(500));
            if (last_shared < nb) BAD("shared: workspace shrinks");
        } else ++n_rej;

        const int before_w = g_launches;
        const size_t wb = kvr_workspace_bytes_weigh(&d, L, S);
        g_ws_given = wb == (size_t)-1 ? (size_t)1 << 40 : wb;
        const int sw = kvr_cache_weigh(&d, A, A, A, L, S, (float *)A, A, g_ws_given, nullptr);
        if ((sw == KVR_ERR_DEVICE) != (g_launches > before_w)) BAD("weigh: status %d", sw);
        if (sw == KVR_ERR_DEVICE) {
            ++n_ok;
            if (kvr_cache_weigh(&d, A, A, A, L, S, (float *)A, A, wb - 1, nullptr) != KVR_ERR_WORKSPACE) BAD("weigh: short workspace");
            last_weigh = kvr_workspace_bytes_weigh(&d, L + (int64_t)rnd(500), S);
            if (last_weigh < wb) BAD("weigh: workspace shrinks");
        } else ++n_rej;

        const int before_e = g_launches;
        const size_t eb = kvr_workspace_bytes_evict(&d, L);
        g_ws_given = eb == (size_t)-1 ? (size_t)1 << 40 : eb;
        // buffers far apart: no overlap for the capacities drawn most
        auto at = [](int k) { return (void *)(((uintptr_t)1 << 44) * (uintptr_t)(k + 1)); };
        const int64_t keep = wild ? odd_size() : L / 3;
        const int se = kvr_cache_evict(&d, at(0), at(1), L, (const float *)at(2), wild ? odd_size() : (int64_t)rnd(9),
                                       wild ? odd_size() : (int64_t)rnd(9), keep, at(3), at(4), wild ? odd_size() : keep,
                                       rnd(2) ? (float *)at(5) : nullptr, rnd(2) ? (int32_t *)at(6) : nullptr, at(7), g_ws_given,
                                       nullptr);
        if ((se == KVR_ERR_DEVICE) != (g_launches > before_e)) BAD("evict: status %d", se);
        if (se == KVR_ERR_DEVICE) ++n_ok; else ++n_rej;
    }
    printf("%d accepted, %d rejected, %d launches\n", n_ok, n_rej, g_launches);
    if (n_ok < 20000 || n_rej < 20000) BAD("one side of the fuzz is thin");
    if (g_bad) return 1;
    printf("all checks passed\n");
    return 0;
}
