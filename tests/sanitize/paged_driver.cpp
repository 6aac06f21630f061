// Drives the host side of kvr_qk_norm_rope, kvr_paged_append and kvr_paged_decode (paged_api.hip)
// under AddressSanitizer and UndefinedBehaviorSanitizer, without a GPU.  The kernel launchers
// are stubs that check the plan they are given and fail: a call with valid arguments ends in
// KVR_ERR_DEVICE, a rejected one reaches no launcher.  Device pointers are fake aligned integers
// and are never dereferenced.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "kvr.h"
#include "kvr_internal.hpp"
#include "paged/paged_internal.hpp"

static int g_launches = 0, g_bad = 0;
static size_t g_ws_given = 0;

#define BAD(...) (++g_bad, fprintf(stderr, __VA_ARGS__), fputc('\n', stderr))

static void threads(const char *kernel, int64_t blocks, int64_t per_block) {
    if (blocks <= 0 || blocks > 0x7fffffff || blocks * per_block >= ((int64_t)1 << 32)) BAD("%s: %lld blocks", kernel, (long long)blocks);
}

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

// The grid's waves cover every row of every token once, none takes more than 64 tokens
hipError_t launch_rows(const RowsParams &p, int, int, int64_t grid, hipStream_t) {
    ++g_launches;
    const int64_t per = (int64_t)p.n_q + p.n_k + p.n_v;
    threads("rows", grid, 64 * kRowWaves);
    if (p.tokens < 1 || p.tokens > 64 || p.parts < 1 || p.part_rows < 1) BAD("rows: tokens %d parts %d", p.tokens, p.parts);
    if ((int64_t)p.parts * p.part_rows < per || (int64_t)(p.parts - 1) * p.part_rows >= per) BAD("rows: parts");
    const int64_t groups = grid * kRowWaves / p.parts;
    if (groups * p.tokens < p.n_tok) BAD("rows: tokens are left out");
    if ((grid - 1) * kRowWaves / p.parts * p.tokens >= p.n_tok) BAD("rows: workgroups without a token");
    return hipErrorUnknown;
}

// Units, cut as the kernel cuts them, are covered once and found again; records fit the workspace;
// pages of parts are those of their rows.
hipError_t launch_decode(const DecodeParams &p, int head_dim, int dtype, hipStream_t) {
    ++g_launches;
    const int64_t heads = (int64_t)p.n_kv_heads * p.tiles, segs = p.n * heads;
    const int64_t unit = (dtype == KVR_F32 ? kStageKeysF32 : kStageKeys) * (int64_t)p.waves;
    threads("decode", p.grid, 64 * p.waves);
    if (p.waves != 1 && p.waves != 4) BAD("waves %d", p.waves);
    if ((int64_t)p.tiles * p.rows < p.group || p.rows > 32 || (p.tiles > 1 && p.rows != 32)) BAD("tiles");
    if (!p.table) BAD("no table");
    const uint64_t pp = p.page_size / 16;
    for (uint64_t part : {(uint64_t)0, (uint64_t)1, pp - 1, pp, 2 * pp - 1, (uint64_t)p.max_len / 16, ((uint64_t)1 << 27) - 1})
        if (part < ((uint64_t)1 << 27) && (part * p.part_mul) >> p.part_shift != part / pp) BAD("page of part %llu", (unsigned long long)part);
    if (p.alone) {
        if (p.grid != segs) BAD("a workgroup for each");
        return hipErrorUnknown;
    }
    threads("join", segs * (p.merge_rows == 1 ? p.rows : (p.rows + 3) / 4), 256);
    if ((size_t)(2 * (int64_t)p.grid * p.rows * (head_dim + 2)) * 4 + (size_t)segs * 8 > g_ws_given) BAD("workspace");
    const int64_t most = (std::max<int64_t>(p.max_len, 1) + unit - 1) / unit * segs;
    if (most > 0x7fffffff) BAD("units");
    for (int64_t total : {most, std::max<int64_t>(most / 3, 1), (int64_t)1, std::min<int64_t>(most, p.grid + 1)}) {
        const int64_t n = std::min<int64_t>(p.grid, total), each = total / n, more = total - each * n;
        auto start = [&](int64_t w) { return w * each + std::min(w, more); };
        if (start(0) != 0 || start(n) != total) BAD("cut");
        for (int64_t w : {(int64_t)0, more - 1, more, n - 1})
            if (w >= 0 && w < n)
                for (int64_t u : {start(w), start(w + 1) - 1}) {
                    const int64_t longer = more * (each + 1);
                    if ((u < longer ? u / (each + 1) : more + (u - longer) / each) != w) BAD("range of a unit");
                }
    }
    return hipErrorUnknown;
}
}  // namespace kvr

static uint64_t g_state = 88172645463325252ull;
static uint64_t rnd() {
    g_state ^= g_state << 13; g_state ^= g_state >> 7; g_state ^= g_state << 17;
    return g_state;
}
static int64_t pick(std::initializer_list<int64_t> v) { return v.begin()[rnd() % v.size()]; }

int main() {
    void *const A = (void *)(uintptr_t)0x10000;
    int ok = 0;
    for (int it = 0; it < 200000; ++it) {
        kvr_desc d;
        memset(&d, 0, sizeof d);
        d.n_kv_heads = (int32_t)pick({1, 2, 3, 8, 8, 17, 64, 0, -1, 40000});
        d.n_q_heads = d.n_kv_heads * (int32_t)pick({1, 2, 4, 4, 8, 17, 32, 33, 64});
        d.head_dim = (int32_t)pick({64, 128, 128, 128, 96});
        d.dtype = (int32_t)pick({KVR_BF16, KVR_F16, KVR_F32, KVR_BF16, 9});
        const int64_t by = d.dtype == KVR_F32 ? 4 : 8;
        kvr_pages g;
        memset(&g, 0, sizeof g);
        g.k = A; g.v = A;
        g.page_size = (int32_t)pick({16, 16, 32, 48, 64, 256, 1024, 8, 0, -16, 1 << 20, 0x7ffffff0});
        g.n_pages = (int32_t)pick({0, 1, 9, 1000, 0x7fffffff, -1});
        g.max_pages = (int32_t)pick({0, 1, 2, 63, 1000, 70000, 0x7fffffff, -1});
        g.page_stride = (int64_t)d.n_kv_heads * g.page_size * d.head_dim * pick({1, 1, 2}) + pick({0, 0, by, 3, -by});
        g.table = (const int32_t *)A;
        const int32_t n = (int32_t)pick({0, 1, 2, 7, 64, 200, 4500, 1 << 20, 0x7fffffff, -1});
        const int64_t reach = (int64_t)g.max_pages * (g.page_size > 0 ? g.page_size : 0);
        const int64_t most = pick({0, 1, 100, 512, 1000, 4096, reach, reach, reach + 1, 0x7fffffff, ((int64_t)1 << 40), -1});
        g_ws_given = kvr_workspace_bytes_paged(&d, n, most);
        const int before = g_launches;
        kvr_rows q = {A, (int64_t)d.n_q_heads * d.head_dim, d.head_dim};
        kvr_rows k = {A, pick({(int64_t)d.n_kv_heads * d.head_dim, (int64_t)(d.n_q_heads + 2 * (int64_t)d.n_kv_heads) * d.head_dim,
                               d.head_dim, 4, -8, (int64_t)1 << 62}), pick({d.head_dim, d.head_dim, 100 * d.head_dim, 3, (int64_t)1 << 61})};
        const int st = kvr_paged_decode(&d, &g, &q, n, (const int32_t *)A, (int32_t)pick({0, 1, 0x7fffffff, -1}), most, A, A,
                                        g_ws_given == (size_t)-1 ? 0 : g_ws_given, nullptr);
        if ((st == KVR_ERR_DEVICE) != (g_launches > before)) BAD("decode: status %d", st);
        ok += st == KVR_ERR_DEVICE;
        if (g_ws_given != (size_t)-1 && most > 0) {
            const size_t less = kvr_workspace_bytes_paged(&d, n, (int64_t)(rnd() % (uint64_t)most));
            if (less == (size_t)-1 || less > g_ws_given) BAD("workspace of a shorter max_len");
        }
        kvr_rope rope = {(const float *)A, pick({0, 1, reach, reach + 10, -1})};
        const int64_t T = pick({0, 1, 5, n, n, 700, 40000, (int64_t)1 << 28, (int64_t)1 << 40, -1});
        const bool with_q = rnd() & 1;
        const int b2 = g_launches;
        const int s2 = kvr_paged_append(&d, &g, rnd() & 1 ? &rope : nullptr, &k, &k, with_q ? &q : nullptr, with_q ? A : nullptr, A, 1e-6f, n, T,
                                        rnd() & 1 ? (const int32_t *)A : nullptr, (const int32_t *)A, rnd() & 1 ? (const int32_t *)A : nullptr,
                                        with_q ? &q : nullptr, nullptr);
        if ((s2 == KVR_ERR_DEVICE) != (g_launches > b2)) BAD("append: status %d", s2);
        ok += s2 == KVR_ERR_DEVICE;
        const int b3 = g_launches;
        const int s3 = kvr_qk_norm_rope(&d, rnd() & 1 ? &rope : nullptr, &q, &k, A, nullptr, 0.f, T, rnd() & 1 ? (const int32_t *)A : nullptr,
                                        pick({0, 5, (int64_t)1 << 50, -1}), &q, &k, nullptr);
        if ((s3 == KVR_ERR_DEVICE) != (g_launches > b3)) BAD("norm_rope: status %d", s3);
        ok += s3 == KVR_ERR_DEVICE;
    }
    if (ok < 5000) BAD("only %d calls were valid", ok);
    if (g_bad) return 1;
    printf("%d launches, all checks passed\n", g_launches);
    return 0;
}
