// paged_api.hip -- host side of kvr_paged_append, kvr_qk_norm_rope and kvr_paged_decode:
// argument validation (before any HIP call), work planning and workspaces, as kvr_api.hip
// does for the other entry points.
#include <math.h>
#include <string.h>

#include "kvr.h"
#include "paged/paged_internal.hpp"

namespace kvr {
namespace {

constexpr int64_t kCus = 256;
constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int64_t kMaxStride = (int64_t)1 << 40;      // elements
constexpr int64_t kMaxExtent = (int64_t)1 << 60;      // elements of an array: bytes in 64 bits
constexpr int64_t kMaxLen = (int64_t)1 << 30;           // rows of a sequence in decode: 32-bit on the device, with room for a unit
constexpr int64_t kMaxHeads = 65535;                  // rows of a token
constexpr int64_t kMaxGrid = ((int64_t)1 << 24) - 1;  // workgroups of a launch: 2^32 threads are too many

// The library's check of a descriptor: an update of no rows ends after it
int check_desc(const kvr_desc *d) { return kvr_cache_append(d, nullptr, nullptr, 0, nullptr, nullptr, 0, nullptr); }

float eff_scale(const kvr_desc *d) { return d->scale > 0.f ? d->scale : 1.f / sqrtf((float)d->head_dim); }
int elt_bytes(const kvr_desc *d) { return d->dtype == KVR_F32 ? 4 : 2; }

bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int to_status(hipError_t e) { return e == hipSuccess ? KVR_OK : KVR_ERR_DEVICE; }

// ---- rows
// Rows of `heads` heads of n_tok tokens.  Those that are written must not share memory: one token's after
// the other's, or one head's.
int check_rows(const kvr_desc *d, const kvr_rows *r, int64_t n_tok, int64_t heads, bool out) {
    const int64_t D = d->head_dim, by = 16 / elt_bytes(d);
    const struct { int64_t stride, n; } dims[] = {{r->token_stride, n_tok}, {r->head_stride, heads}};
    for (const auto &x : dims) {
        if (x.n <= 1) continue;      // the stride of a single one is not used
        if (x.stride < 0 || x.stride > kMaxStride || x.stride > kMaxExtent / x.n) return KVR_ERR_SHAPE;
        if (x.stride % by) return KVR_ERR_ALIGN;
    }
    if (!r->data) return KVR_ERR_NULL;
    if (!aligned(r->data, 16)) return KVR_ERR_ALIGN;
    if (!out) return KVR_OK;
    if (heads > 1 && r->head_stride < D) return KVR_ERR_SHAPE;
    if (n_tok > 1 && r->token_stride < D) return KVR_ERR_SHAPE;
    if (heads > 1 && n_tok > 1 && r->token_stride < (heads - 1) * r->head_stride + D &&
        (r->head_stride - D) / r->token_stride < n_tok - 1)
        return KVR_ERR_SHAPE;
    return KVR_OK;
}

RowsAt rows_at(const kvr_rows *r) {
    RowsAt a = {nullptr, 0, 0};
    if (r) { a.p = r->data; a.token = r->token_stride; a.head = r->head_stride; }
    return a;
}

int check_table(const kvr_rope *rope, int64_t n_pos) {
    if (!rope) return KVR_OK;
    if (!rope->cos_sin) return KVR_ERR_NULL;
    if (rope->n_pos < n_pos) return KVR_ERR_POSITION;
    return aligned(rope->cos_sin, 16) ? KVR_OK : KVR_ERR_ALIGN;
}

// Few tokens: several waves to one, down to a row for each lane (up to 1024, 2048 and 4096 waves:
// 3774 tokens' keys and values 14.0, 10.9 and 11.0 us, 600 tokens' norms 8.4, 6.5 and 6.2, 945 in
// fp32 5.5, 5.1 and 5.1).  Many: so many tokens to a wave that its lanes have this many rows to load
// (8 and 12: 32768 tokens' norms 136 and 143 us, keys and values 66 and 77; one token each: 81).
constexpr int64_t kFewWaves = 8 * kCus, kLoads = 8;

int run_rows(const kvr_desc *d, RowsParams &p, void *stream) {
    const int64_t per = (int64_t)p.n_q + p.n_k + p.n_v;
    const int64_t step = 64 / (d->head_dim * elt_bytes(d) / 32);      // rows that a wave's lanes hold
    if (per > kMaxHeads) return KVR_ERR_SHAPE;
    int64_t parts = ceil_div(per, step);
    if (parts > kFewWaves / p.n_tok) parts = kFewWaves / p.n_tok > 1 ? kFewWaves / p.n_tok : 1;
    const int64_t part_rows = ceil_div(ceil_div(per, parts), step) * step;
    parts = ceil_div(per, part_rows);
    int64_t tokens = parts > 1 ? 1 : kLoads / ceil_div(per, step);
    if (tokens < 1) tokens = 1;
    while (tokens > 1 && p.n_tok / tokens < kFewWaves) --tokens;
    const int64_t grid = ceil_div(ceil_div(p.n_tok, tokens) * parts, kRowWaves);
    if (grid > kMaxGrid) return KVR_ERR_SHAPE;
    p.tokens = (int32_t)tokens;
    p.parts = (int32_t)parts;
    p.part_rows = (int32_t)part_rows;
    return to_status(launch_rows(p, d->head_dim, d->dtype, grid, (hipStream_t)stream));
}

// ---- pages
int check_pages(const kvr_desc *d, const kvr_pages *g) {
    if (!g) return KVR_ERR_NULL;
    if (g->reserved != 0 || g->n_pages < 0 || g->max_pages < 0) return KVR_ERR_SHAPE;
    if (g->page_size <= 0 || g->page_size % 16) return KVR_ERR_SHAPE;
    if (g->max_pages > kMaxRows / g->page_size) return KVR_ERR_SHAPE;
    const int64_t page = (int64_t)d->n_kv_heads * d->head_dim;
    if (page > kMaxStride / g->page_size) return KVR_ERR_SHAPE;
    if (g->page_stride < page * g->page_size || g->page_stride > kMaxStride) return KVR_ERR_SHAPE;
    if (g->n_pages > 0 && g->page_stride > kMaxExtent / g->n_pages) return KVR_ERR_SHAPE;
    if (g->page_stride % (16 / elt_bytes(d))) return KVR_ERR_ALIGN;
    return KVR_OK;
}
int check_page_pointers(const kvr_pages *g) {
    if (g->n_pages > 0 && (!g->k || !g->v)) return KVR_ERR_NULL;
    if (g->max_pages > 0 && !g->table) return KVR_ERR_NULL;
    return aligned(g->k, 16) && aligned(g->v, 16) && aligned(g->table, 4) ? KVR_OK : KVR_ERR_ALIGN;
}

// ---- decode
// All in a captured graph, us a call, 16-bit, 32 / 8 heads of 128 where nothing else is said ("16 / 2":
// heads of 64); a stage is a wave's 16 KB of keys and values (8 KB at 64).
//
// Waves that share the units out: as many as ask for this much at once on a compute unit.  32, 64 and
// 128 KB: one sequence of 32768 rows 38.0, 27.4 and 29.0, 64 of 100 to 4096 143, 99 and 98, in fp16 153, 95 and 106, of
// 300 to 32768 1116, 682 and 683; 16 / 2, 64 of 100 to 3900 19.1, 19.7 and 21.2.
constexpr int64_t kAskedBytes = 64 << 10;
// A sequence and head of at most this many bytes is one workgroup's of four waves, and nothing is joined:
// 256 KB, more where there are many of them, as far as one long sequence among short ones does not hold the
// others up for long.  In one launch and shared out, in a graph and (in brackets) issued one by one, where two launches
// take the host 10: 1 sequence of 310 rows 6.6 and 7.0 (7.5 and 10.5), 480 (240 KB) 7.7 and 7.0 (8.1 and 10.3), 600
// 8.7 and 7.3 (9.0 and 10.3); 8 of 20 to 480 8.6 and 8.7 (8.3 and 10.1), to 600 9.7 and 9.0 (9.6 and 9.9); 16 / 2, 1 of 900
// (232 KB) 9.2 and 6.9 (9.5 and 9.8); fp32, 8 of 10 to 250 (256 KB) 10.2 and 8.9 (10.1 and 9.9).  In a graph: 32 of 10 to 980
// (496 KB) 18.4 and 20.1, 64 of 100 to 1500 (752 KB) 47.7 and 45.7; 16 / 2, 64 of 10 to 900 10.1 and 10.9; fp32, 64 of
// 10 to 480 (480 KB) 33.7 and 37.2.
constexpr int64_t kAloneBytes = 256 << 10, kAloneMost = 512 << 10, kAloneByHeads = 2 << 10;
// One wave instead of four, where many of them are short: 128 sequences of 10 to 200 rows 16.6 instead of 18.4, 256
// 27.3 instead of 29.8, 256 of 10 to 480 (240 KB) 56.9 and 55.6; 64 of 10 to 250 12.0 and 11.2.
constexpr int64_t kOneWaveHeads = 1024, kOneWaveBytes = 128 << 10;
// Shared out, ranges of one wave up to this many stages of a sequence, of four beyond (records of which
// there are fewer): 1 sequence of 480 rows 7.0 and 8.1, 980 (31 stages) 7.9 and 8.6, 1500 8.9 and 9.0, 3774
// 11.6 and 9.9; 8 of 100 to 980 11.2 and 11.6.
constexpr int64_t kOneWaveStages = 32;
// Records are joined a query row a workgroup, or four where there are many: 1 and 4, one sequence of 3774
// rows 9.8 and 11.6, of 32768 27.1 and 29.0, 16 of 100 to 3980 31.3 and 31.2, 32 53.4 and 52.5, 64 of up to 4096 in fp16 95.5 and 93.8.
constexpr int64_t kMergeHeads = 128;
// Keys and values of a whole call from which they are loaded with the non-temporal hint, in ranges of four
// waves and up to 16 query rows of a kv head.  Without and with it: 64 sequences of 300 to 32768 rows 767 and
// 678, 64 of 100 to 4096 (538 MB) 105 and 94, one of 32768 (134 MB) 29.6 and 26.9, 8 of 100 to 3980 (67 MB) 20.3
// and 19.4; one of 16000 (66 MB) 19.2 and 18.1, that the caches still hold 16.9 and 16.8, 4 of 100 to 3980 (34 MB) 14.4 and
// 14.7, held 11.1 and 12.6; fp32, 64 of 100 to 16000 756 and 747.  What is read is counted, not what is
// distinct: pages that sequences share come from the caches more slowly with the hint, 64 sequences with 256 rows each
// behind one prefix of 4096 rows 93 and 107, of 32768 573 and 752.
constexpr int64_t kStreamBytes = 48 << 20;

struct DecodePlan {
    int64_t tiles, rows, grid, stage_bytes, units;
    int waves, merge_rows;
    bool alone;
    size_t ws_bytes;
};

bool plan_decode(const kvr_desc *d, int64_t n, int64_t max_len, DecodePlan *out) {
    DecodePlan s;
    memset(&s, 0, sizeof s);
    const int64_t G = d->n_q_heads / d->n_kv_heads, stage = d->dtype == KVR_F32 ? kStageKeysF32 : kStageKeys;
    s.rows = G < 32 ? G : 32;
    s.tiles = ceil_div(G, 32);
    if (n > kMaxGrid / d->n_kv_heads / s.tiles || n > kMaxGrid / d->n_q_heads) return false;
    const int64_t heads = n * d->n_kv_heads * s.tiles;
    const int64_t stages = max_len > 0 ? ceil_div(max_len, stage) : 1;
    if (heads > 0 && stages > kMaxRows / heads) return false;
    s.stage_bytes = stage * d->head_dim * elt_bytes(d) * 2;
    const int64_t bytes = stages * s.stage_bytes;      // of a sequence and head, at most
    const int64_t waves = kAskedBytes / s.stage_bytes * kCus;
    const int64_t by_heads = heads * kAloneByHeads < kAloneMost ? heads * kAloneByHeads : kAloneMost;
    const int64_t alone_bytes = by_heads > kAloneBytes ? by_heads : kAloneBytes;
    s.alone = bytes <= alone_bytes;
    if (s.alone) s.waves = heads >= kOneWaveHeads && bytes <= kOneWaveBytes ? 1 : 4;
    else s.waves = stages <= kOneWaveStages ? 1 : 4;
    s.merge_rows = heads >= kMergeHeads ? 4 : 1;
    s.units = ceil_div(stages, s.waves) * heads;      // at most
    s.grid = s.alone ? heads : s.units < waves / s.waves ? s.units : waves / s.waves;
    // (single waves have more records than workgroups of four: room for what a shorter max_len needs, too, where one
    // that is not one launch has single waves)
    const int64_t one = kOneWaveStages * s.stage_bytes > alone_bytes ? (stages < kOneWaveStages ? stages : kOneWaveStages) * heads : 0;
    const int64_t most = one < waves ? one : waves;
    const int64_t sharers = s.grid > most ? s.grid : most;
    if (!s.alone) s.ws_bytes = (size_t)(2 * sharers * s.rows * (d->head_dim + 2)) * sizeof(float) + (size_t)heads * 8;
    *out = s;
    return true;
}

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" {

int kvr_qk_norm_rope(const kvr_desc *desc, const kvr_rope *rope, const kvr_rows *q, const kvr_rows *k, const void *q_norm,
                     const void *k_norm, float eps, int64_t n_tok, const int32_t *pos, int64_t pos0, const kvr_rows *q_out,
                     const kvr_rows *k_out, void *stream) {
    int st = check_desc(desc);
    if (st) return st;
    if (n_tok < 0 || n_tok > kMaxRows || !(eps >= 0.f) || isinf(eps)) return KVR_ERR_SHAPE;
    if (rope && !pos && (pos0 < 0 || pos0 > kMaxStride)) return KVR_ERR_POSITION;
    if (n_tok == 0) return KVR_OK;
    if ((!q && !k) || !q != !q_out || !k != !k_out) return KVR_ERR_NULL;
    if ((q_norm && !q) || (k_norm && !k)) return KVR_ERR_NULL;
    if (q && ((st = check_rows(desc, q, n_tok, desc->n_q_heads, false)) || (st = check_rows(desc, q_out, n_tok, desc->n_q_heads, true)))) return st;
    if (k && ((st = check_rows(desc, k, n_tok, desc->n_kv_heads, false)) || (st = check_rows(desc, k_out, n_tok, desc->n_kv_heads, true)))) return st;
    if ((st = check_table(rope, pos ? 1 : pos0 + n_tok))) return st;
    if (!aligned(q_norm, 16) || !aligned(k_norm, 16) || !aligned(pos, 4)) return KVR_ERR_ALIGN;

    RowsParams p;
    memset(&p, 0, sizeof p);
    p.q = rows_at(q); p.k = rows_at(k); p.qo = rows_at(q_out); p.ko = rows_at(k_out);
    p.qn = q_norm; p.kn = k_norm;
    p.eps = eps;
    if (rope) { p.cs = rope->cos_sin; p.n_pos = rope->n_pos; }
    p.pos = pos;
    p.pos0 = pos0;
    p.n_tok = n_tok;
    p.n_q = q ? desc->n_q_heads : 0;
    p.n_k = k ? desc->n_kv_heads : 0;
    return run_rows(desc, p, stream);
}

int kvr_paged_append(const kvr_desc *desc, const kvr_pages *pages, const kvr_rope *rope, const kvr_rows *k, const kvr_rows *v,
                     const kvr_rows *q, const void *q_norm, const void *k_norm, float eps, int32_t n, int64_t n_tok,
                     const int32_t *cu_seqlens, const int32_t *len, const int32_t *pos, const kvr_rows *q_out, void *stream) {
    int st = check_desc(desc);
    if (st) return st;
    if ((st = check_pages(desc, pages))) return st;
    if (n < 0 || n > kMaxGrid || n_tok < 0 || n_tok > kMaxRows || (!cu_seqlens && n_tok != n) || !(eps >= 0.f) || isinf(eps)) return KVR_ERR_SHAPE;
    if (n == 0 || n_tok == 0) return KVR_OK;
    if (!k || !v || !len || !q != !q_out || (q_norm && !q)) return KVR_ERR_NULL;
    if ((st = check_page_pointers(pages))) return st;
    if ((st = check_rows(desc, k, n_tok, desc->n_kv_heads, false)) || (st = check_rows(desc, v, n_tok, desc->n_kv_heads, false))) return st;
    if (q && ((st = check_rows(desc, q, n_tok, desc->n_q_heads, false)) || (st = check_rows(desc, q_out, n_tok, desc->n_q_heads, true)))) return st;
    if ((st = check_table(rope, pos ? 1 : (int64_t)pages->max_pages * pages->page_size))) return st;
    if (!aligned(q_norm, 16) || !aligned(k_norm, 16)) return KVR_ERR_ALIGN;
    if (!aligned(cu_seqlens, 4) || !aligned(len, 4) || !aligned(pos, 4)) return KVR_ERR_ALIGN;
    if (pages->n_pages == 0 || pages->max_pages == 0) return KVR_OK;      // no token has a place

    RowsParams p;
    memset(&p, 0, sizeof p);
    p.q = rows_at(q); p.k = rows_at(k); p.v = rows_at(v); p.qo = rows_at(q_out);
    p.qn = q_norm; p.kn = k_norm;
    p.eps = eps;
    if (rope) { p.cs = rope->cos_sin; p.n_pos = rope->n_pos; }
    p.pos = pos;
    p.kp = (unsigned char *)pages->k; p.vp = (unsigned char *)pages->v;
    p.page_bytes = pages->page_stride * elt_bytes(desc);
    p.table = pages->table; p.cu = cu_seqlens; p.len = len;
    p.n_pages = pages->n_pages;
    p.page_size = pages->page_size;
    p.max_pages = pages->max_pages;
    p.n_seq = n;
    p.n_tok = n_tok;
    p.n_q = q ? desc->n_q_heads : 0;
    p.n_k = p.n_v = desc->n_kv_heads;
    return run_rows(desc, p, stream);
}

size_t kvr_workspace_bytes_paged(const kvr_desc *desc, int32_t n, int64_t max_len) {
    DecodePlan s;
    if (check_desc(desc) != KVR_OK || n < 0 || max_len < 0 || max_len > kMaxLen) return (size_t)-1;
    return plan_decode(desc, n, max_len, &s) ? s.ws_bytes : (size_t)-1;
}

int kvr_paged_decode(const kvr_desc *desc, const kvr_pages *pages, const kvr_rows *q, int32_t n, const int32_t *len, int32_t n_new,
                     int64_t max_len, void *out, void *ws, size_t ws_bytes, void *stream) {
    int st = check_desc(desc);
    if (st) return st;
    if ((st = check_pages(desc, pages))) return st;
    if (n < 0 || n_new < 0 || max_len < 0 || max_len > kMaxLen) return KVR_ERR_SHAPE;
    if (max_len > (int64_t)pages->max_pages * pages->page_size) return KVR_ERR_CAPACITY;
    DecodePlan plan;
    if (!plan_decode(desc, n, max_len, &plan)) return KVR_ERR_SHAPE;
    if (n == 0) return KVR_OK;
    if (!q || !out || !len) return KVR_ERR_NULL;
    if ((st = check_rows(desc, q, n, desc->n_q_heads, false))) return st;
    if ((st = check_page_pointers(pages))) return st;
    if (!aligned(out, 16) || !aligned(ws, 16) || !aligned(len, 4)) return KVR_ERR_ALIGN;
    if (plan.ws_bytes && (!ws || ws_bytes < plan.ws_bytes)) return KVR_ERR_WORKSPACE;

    DecodeParams p;
    memset(&p, 0, sizeof p);
    p.q = rows_at(q);
    p.out = out;
    p.kp = (const unsigned char *)pages->k; p.vp = (const unsigned char *)pages->v;
    p.page_bytes = pages->page_stride * elt_bytes(desc);
    p.table = pages->max_pages ? pages->table : len;      // (no rows then: what is read is not used)
    p.len = len;
    p.ws = (float *)ws;
    p.n = n;
    p.n_new = n_new;
    p.max_len = (int32_t)max_len;
    p.n_pages = pages->n_pages;
    p.page_size = pages->page_size;
    p.max_pages = pages->max_pages;
    p.n_q_heads = desc->n_q_heads;
    p.n_kv_heads = desc->n_kv_heads;
    p.group = desc->n_q_heads / desc->n_kv_heads;
    p.tiles = (int32_t)plan.tiles;
    p.rows = (int32_t)plan.rows;
    p.grid = (int32_t)plan.grid;
    p.waves = plan.waves;
    const int64_t stream_units = kStreamBytes / (plan.waves * plan.stage_bytes);
    p.stream_units = !plan.alone && plan.waves == 4 && plan.units >= stream_units ? (int32_t)stream_units : 0;
    p.merge_rows = plan.merge_rows;
    p.alone = plan.alone ? 1 : 0;
    // part / (parts of a page), exact for the parts of 2^31 rows: with 2^b parts or more, ceil(2^(32 + b) / parts)
    // is less than 2^b too large in 2^(32 + b), and a part is below 2^28
    const uint64_t parts = pages->page_size / 16;
    int bits = 0;
    while (((uint64_t)1 << bits) < parts) ++bits;
    p.part_shift = 32 + bits;
    p.part_mul = (((uint64_t)1 << p.part_shift) + parts - 1) / parts;
    // Weights enter the second product times this, the largest one 1.  fp16 numbers end at 2^-24 and below 2^16: 2^15;
    // bf16 and fp32 numbers reach down to 2^-126, and a sum over max_len rows of the largest values is finite, as their
    // mean is, with 1 / max_len (a half of that: sums are rounded).  A factor is exact; as an addend of the weight's
    // exponent it would cost fp32 weights up to four bits (9 sequences of up to 945 rows off by 1.5e-7 instead of 7.9e-8).
    int lift = 15;
    if (desc->dtype != KVR_F16)
        for (lift = -1; ((int64_t)1 << (-1 - lift)) < max_len;) --lift;
    p.lift = ldexpf(1.f, lift);
    p.unlift = ldexpf(1.f, -lift);
    // (finite: no difference stays none)
    p.half_scale_log2 = fminf(eff_scale(desc) * (2.f * 1.4426950408889634f), 3.4028235e38f);
    return to_status(launch_decode(p, desc->head_dim, desc->dtype, (hipStream_t)stream));
}

}  // extern "C"
