// readers_api.hip -- host side of kvr_continue_shared, kvr_cache_weigh and
// kvr_cache_evict: argument validation (before any HIP call), work planning and
// workspaces, as kvr_api.hip does for the other entry points.
#include <math.h>
#include <string.h>

#include "kvr.h"
#include "readers_internal.hpp"

namespace kvr {
namespace {

constexpr int64_t kMaxTokens = (int64_t)1 << 30;
constexpr int64_t kMaxKeys = (int64_t)1 << 40;
constexpr int64_t kCus = 256;
constexpr int64_t kMaxRows = 0x7fffffff;   // cached rows and query rows of a call: 32-bit on the device
constexpr int64_t kMaxGrid = ((int64_t)1 << 24) - 1;   // workgroups of a launch: 2^32 threads are too many
constexpr int kWaves = 4;                  // of a workgroup

// The library's check of a descriptor: an update of no rows ends after it
int check_desc(const kvr_desc *d) { return kvr_cache_append(d, nullptr, nullptr, 0, nullptr, nullptr, 0, nullptr); }

float eff_scale(const kvr_desc *d) { return d->scale > 0.f ? d->scale : 1.f / sqrtf((float)d->head_dim); }
int elt_bytes(const kvr_desc *d) { return d->dtype == KVR_F32 ? 4 : 2; }

bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// keys of a stage (attn_direct.hpp)
int64_t stage_keys(const kvr_desc *d) { return d->dtype == KVR_F32 ? 16 : 32; }

// query rows of a workgroup (readers_internal.hpp)
int64_t way_rows(int way) { return way > kByRows ? 64 * (way - kByRows) : 16 * way; }

// ---- shared
// Workgroups are as many as there are compute units (256 and 512, items and merge: 2 readers
// of 32768 keys 26.9 + 4.2 and 27.1 + 5.4 us, 9 of 32768 31.2 + 4.0 and 35.6 + 5.5, 8 readers'
// 8000 own rows 48.4 + 4.8 and 47.8 + 4.8; 16 x 4 of 16384 35.2 + 6.1 and 36.3 + 9.0, but 64
// of 32768 without own rows 58.5 + 6.4 and 51.6 + 9.2), as long as each keeps this many keys.
// Prefix by keys: one stage for each wave; 128 and 256 measured 5.7 and 6.6 us with 255 keys
// and 2 readers, 6.1 and 7.4 us with 945 keys and 3 readers in fp32.  By rows it is 256:
// 128, 256 and 512 took 11.6, 11.0 and 13.7 us with 3774 keys and 9 readers, and a merge
// of more records.  Own rows: 128, 256 and 512 took 11.6, 11.2 and 10.3 us with 9 readers.
constexpr int64_t kMinKeysByKeys = 128, kMinKeysByRows = 256, kMinOwnKeys = 512;
// 2 readers of 8000 own rows: 4 and 16 splits 23.0 and 14.2 us; one of 16000: 16 and 32 splits
// 14.8 and 13.9
constexpr int64_t kMaxOwnSplits = 32;
// Prefix rows x keys from which a wave (fp32: an item) takes two tiles of query rows, which
// reads each key half as often, but leaves fewer items.  16-bit, one and two tiles: 256 rows of
// 3774 keys 18.4 + 4.0 and 20.0 + 5.5 us (items, merge), 128 of 3774 13.7 and 16.3, 68 of 32768
// 41.7 and 35.9, 256 of 16384 42.0 and 35.8.  fp32, 128 rows of 3774 keys 33.8 and 34.3, 64 of
// 16384 69.8 and 53.5; of head_dim 64, 192 of 945 6.3 and 8.3, 256 of 3774 12.8 and 12.8, 128 of
// 16384 20.6 and 18.0.
constexpr int64_t kWork2 = 3 << 19, kWork2F32 = 1 << 19;
// A call of at most this many stages of prefix and own rows is one launch (kAlone), not the
// items' and the merge's.  Us a call in a graph, and issued one by one (bf16, 32 / 8 heads of
// 128, one launch and two):
//     1 reader    10 stages   7.3 and 7.4   10.3 and 13.1     20 stages    9.8 and 7.5    10.4 and 13.0
//     32 readers  10          7.7 and 12.9  10.3 and 13.3     20          10.3 and 13.4   10.3 and 13.8
// fp32, 1 reader, 10 stages: 8.9 and 9.6, 10.4 and 13.1; 20: 11.6 and 9.8, 11.7 and 13.1; 32 readers,
// 10 stages: 9.7 and 13.4, 10.3 and 13.5.
constexpr int64_t kAloneStages = 20, kAloneStagesF32 = 10;
// Every reader reads the prefix anew, so there is a bound on stages times workgroups (one a reader
// and kv head; at head_dim 64 a compute unit holds two, and each needs half the bytes).  32 / 8 heads
// of 128, 512 workgroups: 13.4 and 14.6 us with 10 stages, 15.5 and 15.0 with 14, 18.5 and 15.8 with
// 20; 2048: 35.4 and 31.5 with 3, 67 and 36 with 20 (fp32, 512: 17.4 and 18.2 with 10; 2048: 52 and
// 42 with 3).  16 / 2 heads of 64, 512: 11.5 and 12.9 with 20; 2048: 26.1 and 30.6 with 10, 34.8 and
// 31.5 with 18.
constexpr int64_t kAloneWork = 20 * kCus, kAloneWork64 = 4 * kAloneWork;

struct SharedPlan {
    int pw, ow;
    int64_t p_tiles, t_tiles, np, nt, chunk, rows, octs_p, octs_o, octs_n;
    size_t ws_bytes;
};

// Row tiles, key splits and grid of a call: a pure function of the shape, its
// workspace non-decreasing in L_prefix and tail_capacity.
bool plan_shared(const kvr_desc *d, int64_t L, int64_t n, int64_t S, int64_t tcap, SharedPlan *out) {
    SharedPlan s;
    memset(&s, 0, sizeof s);
    const int64_t G = d->n_q_heads / d->n_kv_heads;
    if (n > kMaxRows || S > kMaxTokens || L > kMaxRows || tcap > kMaxRows) return false;
    if (n > 0 && S > kMaxRows / n / d->n_q_heads) return false;
    s.rows = n * S * d->n_q_heads;
    if (s.rows > 0) {
        const int64_t rows_p = n * S * G, rows_o = S * G;
        const bool f32 = d->dtype == KVR_F32;
        if (f32) s.pw = rows_p > 16 && rows_p * L > kWork2F32 ? 2 : 1;
        else s.pw = rows_p <= 16 ? 1 : kByRows + (rows_p > 64 && rows_p * L > kWork2 ? 2 : 1);
        s.ow = rows_o <= 16 || s.pw == 1 ? 1 : f32 ? 2 : kByRows + 1;
        s.p_tiles = ceil_div(rows_p, way_rows(s.pw));
        s.t_tiles = ceil_div(rows_o, way_rows(s.ow));
        int64_t want = 0;
        if (L > 0) {
            const int64_t base = s.p_tiles * d->n_kv_heads;
            const int64_t step = kWaves * stage_keys(d);
            want = ceil_div(kCus, base);
            const int64_t by_keys = ceil_div(L, s.pw > kByRows ? kMinKeysByRows : kMinKeysByKeys);
            if (want > by_keys) want = by_keys;
            s.chunk = ceil_div(ceil_div(L, want), step) * step;
            s.np = ceil_div(L, s.chunk);
        }
        const int64_t own = n * s.t_tiles * d->n_kv_heads;
        if (tcap > 0) {
            s.nt = ceil_div(kCus, own);
            const int64_t by_cap = ceil_div(tcap, kMinOwnKeys);
            if (s.nt > by_cap) s.nt = by_cap;
            if (s.nt > kMaxOwnSplits) s.nt = kMaxOwnSplits;
        }
        s.octs_p = ceil_div(s.np * d->n_kv_heads, 8) * s.p_tiles;
        s.octs_o = ceil_div(own * s.nt, 8);
        s.octs_n = ceil_div(n * ceil_div(rows_o, 16) * d->n_kv_heads, 8 * kWaves);
        if ((s.octs_p + s.octs_o + s.octs_n) * 8 > kMaxGrid || s.rows > kMaxGrid) return false;
        const int64_t stages = ceil_div(L, stage_keys(d)) + ceil_div(tcap, stage_keys(d));
        const int64_t work = (stages > 1 ? stages : 1) * n * d->n_kv_heads;
        if (rows_o <= 16 && stages <= (f32 ? kAloneStagesF32 : kAloneStages) && work <= (d->head_dim == 64 ? kAloneWork64 : kAloneWork))
            s.pw = kAlone;
        s.ws_bytes = (size_t)(want + s.nt + 1) * (size_t)s.rows * (d->head_dim + 2) * sizeof(float);
    }
    *out = s;
    return true;
}

// ---- weigh
// First pass.  16-bit, direct and by rows: 16 query rows of a kv head over 16384 keys 9.9 and
// 10.6 us, over 3774 4.3 and 5.2, 20 rows 13.2 and 10.8.  By rows, two and four tiles a wave:
// 512 rows of 16384 keys 28.6 and 25.9, 256 of 16384 16.9 and 17.1, 512 of 3774 11.4 and 12.7.
// fp32, one and two tiles: 16 rows of 4096 keys 6.6 and 7.9, 32 of 4096 10.8 and 9.0, 96 of
// 16384 66 and 50.
constexpr int64_t kStages4 = 256;
// Workgroups: 512, 768 and 1024 take 44, 48 and 47 us for 512 rows of 32640 keys
constexpr int64_t kStatsGroups = 2 * kCus;
constexpr int64_t kJoinAlone = 1024;   // splits x rows of a kv head from which they are joined once for all

struct WeighPlan {
    int way, held;
    bool join;
    int64_t nsplit, chunk, grid, norm_at;
    size_t ws_bytes;
};

bool plan_weigh(const kvr_desc *d, int64_t L, int64_t S, WeighPlan *out) {
    WeighPlan w;
    memset(&w, 0, sizeof w);
    const int64_t G = d->n_q_heads / d->n_kv_heads;
    if (L > kMaxRows || S > kMaxRows / G || L + S > kMaxRows) return false;
    if (S > 0) {
        const int64_t rows = S * G;
        const int64_t stages = ceil_div(L, stage_keys(d)) + ceil_div(S, stage_keys(d));
        const bool f32 = d->dtype == KVR_F32;
        w.way = rows <= 16 ? 1 : f32 ? 2 : kByRows + (rows > 256 && stages > kStages4 ? 4 : 2);
        const int64_t base = ceil_div(rows, way_rows(w.way)) * d->n_kv_heads;
        int64_t want = ceil_div(kStatsGroups, base);
        const int64_t most = ceil_div(stages, kWaves);
        if (want > most) want = most;
        const int64_t step = w.way > kByRows ? 1 : kWaves;      // the waves share a stage, or take one each
        w.chunk = ceil_div(ceil_div(stages, want), step) * step;
        w.nsplit = ceil_div(stages, w.chunk);
        w.grid = base * w.nsplit;
        // second pass in fp32: two stages held halve the reads of the query rows, as long as
        // the workgroups fill the part.  One and two: 24 rows of 16384 keys 69 and 49 us, of
        // 4096 23.8 and 21.1, of 1000 9.2 and 12.0.
        w.held = f32 && ceil_div(stages, kWaves * 2) * d->n_kv_heads >= kCus ? 2 : 1;
        if (w.grid > kMaxGrid || ceil_div(stages, kWaves) * d->n_kv_heads > kMaxGrid) return false;
        w.join = w.nsplit * rows > kJoinAlone;
        if (w.join && rows * d->n_kv_heads > kMaxGrid * 32) return false;      // (eight lanes a row: 32 a workgroup)
        w.norm_at = want * d->n_kv_heads * rows * 2 * (int64_t)sizeof(float);
        w.ws_bytes = (size_t)w.norm_at + (size_t)d->n_kv_heads * rows * sizeof(float);
    }
    *out = w;
    return true;
}

// ---- evict
// Kept rows, at least, of a workgroup that searches on its own: 512 of 1024 rows take 6.2, 6.2
// and 6.9 us with 4, 16 and 64
constexpr int64_t kRowsPerPart = 16;

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && na && nb && x < y + nb && y < x + na;
}

int to_status(hipError_t e) { return e == hipSuccess ? KVR_OK : KVR_ERR_DEVICE; }

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" {

size_t kvr_workspace_bytes_shared(const kvr_desc *desc, int64_t L_prefix, int32_t n, int32_t S, int64_t tail_capacity) {
    SharedPlan s;
    if (check_desc(desc) != KVR_OK || L_prefix < 0 || n < 0 || S < 0 || tail_capacity < 0) return (size_t)-1;
    return plan_shared(desc, L_prefix, n, S, tail_capacity, &s) ? s.ws_bytes : (size_t)-1;
}

int kvr_continue_shared(const kvr_desc *desc, const kvr_rope *rope, const void *Qs, const void *Ks, const void *Vs,
                        int32_t n, int32_t S, const void *kcache, const void *vcache, int64_t L_prefix, int64_t pos0,
                        void *ktail, void *vtail, int64_t tail_capacity, const int32_t *tail_len, int32_t append,
                        void *out, void *ws, size_t ws_bytes, void *stream) {
    int st = check_desc(desc);
    if (st) return st;
    if (n < 0 || S < 0 || L_prefix < 0 || tail_capacity < 0) return KVR_ERR_SHAPE;
    SharedPlan plan;
    if (!plan_shared(desc, L_prefix, n, S, tail_capacity, &plan)) return KVR_ERR_SHAPE;
    if (L_prefix > desc->capacity) return KVR_ERR_CAPACITY;
    if (append && S > tail_capacity) return KVR_ERR_CAPACITY;
    if (plan.rows == 0) return KVR_OK;
    if (!Qs || !Ks || !Vs || !out || !tail_len) return KVR_ERR_NULL;
    if (L_prefix > 0 && (!kcache || !vcache)) return KVR_ERR_NULL;
    if (tail_capacity > 0 && (!ktail || !vtail)) return KVR_ERR_NULL;
    if (rope) {
        if (pos0 < 0 || pos0 > kMaxKeys) return KVR_ERR_POSITION;
        if (!rope->cos_sin) return KVR_ERR_NULL;
        if (rope->n_pos < pos0 + tail_capacity + (append ? 0 : S)) return KVR_ERR_POSITION;
    }
    const void *const ptrs[] = {Qs, Ks, Vs, out, kcache, vcache, ktail, vtail, ws, rope ? rope->cos_sin : nullptr};
    for (const void *p : ptrs)
        if (!aligned(p, 16)) return KVR_ERR_ALIGN;
    if (!aligned(tail_len, 4)) return KVR_ERR_ALIGN;
    if (!ws || ws_bytes < plan.ws_bytes) return KVR_ERR_WORKSPACE;

    SharedParams p;
    memset(&p, 0, sizeof p);
    p.q = Qs; p.kn = Ks; p.vn = Vs; p.kc = kcache; p.vc = vcache; p.kt = ktail; p.vt = vtail;
    p.len = tail_len;
    p.out = out;
    p.ws = (float *)ws;
    p.rope = rope ? rope->cos_sin : nullptr;
    p.cap = desc->capacity;
    p.tcap = tail_capacity;
    p.L = L_prefix;
    p.pos0 = pos0;
    p.chunk = plan.chunk;
    p.rows = plan.rows;
    p.scale_log2 = eff_scale(desc) * 1.4426950408889634f;
    p.n = n;
    p.S = S;
    p.n_q_heads = desc->n_q_heads;
    p.n_kv_heads = desc->n_kv_heads;
    p.group = desc->n_q_heads / desc->n_kv_heads;
    p.append = append ? 1 : 0;
    p.np = (int32_t)plan.np;
    p.nt = (int32_t)plan.nt;
    p.nrec = p.np + p.nt + 1;
    p.p_tiles = (int32_t)plan.p_tiles;
    p.t_tiles = (int32_t)plan.t_tiles;
    p.oct_own = (uint32_t)plan.octs_p;
    p.oct_new = (uint32_t)(plan.octs_p + plan.octs_o);
    p.oct_all = (uint32_t)(plan.octs_p + plan.octs_o + plan.octs_n);
    return to_status(launch_shared(p, desc->head_dim, desc->dtype, plan.pw, plan.ow, (hipStream_t)stream));
}

size_t kvr_workspace_bytes_weigh(const kvr_desc *desc, int64_t L_prefix, int64_t S) {
    WeighPlan w;
    if (check_desc(desc) != KVR_OK || L_prefix < 0 || S < 0) return (size_t)-1;
    return plan_weigh(desc, L_prefix, S, &w) ? w.ws_bytes : (size_t)-1;
}

int kvr_cache_weigh(const kvr_desc *desc, const void *Qs, const void *Ks, const void *kcache, int64_t L_prefix,
                    int64_t S, float *weight, void *ws, size_t ws_bytes, void *stream) {
    const int st = check_desc(desc);
    if (st) return st;
    if (L_prefix < 0 || S < 0) return KVR_ERR_SHAPE;
    WeighPlan plan;
    if (!plan_weigh(desc, L_prefix, S, &plan)) return KVR_ERR_SHAPE;
    if (L_prefix + S > desc->capacity) return KVR_ERR_CAPACITY;
    if (S == 0) return KVR_OK;
    if (!Qs || !Ks || !weight || (L_prefix > 0 && !kcache)) return KVR_ERR_NULL;
    if (!aligned(Qs, 16) || !aligned(Ks, 16) || !aligned(kcache, 16) || !aligned(weight, 4) || !aligned(ws, 16))
        return KVR_ERR_ALIGN;
    if (!ws || ws_bytes < plan.ws_bytes) return KVR_ERR_WORKSPACE;

    WeighParams p;
    memset(&p, 0, sizeof p);
    p.q = Qs; p.kn = Ks; p.kc = kcache;
    p.weight = weight;
    p.ws = (float2 *)ws;
    p.norm = plan.join ? (float *)((char *)ws + plan.norm_at) : nullptr;
    p.cap = desc->capacity;
    p.L = L_prefix;
    p.S = (int32_t)S;
    p.n_q_heads = desc->n_q_heads;
    p.n_kv_heads = desc->n_kv_heads;
    p.group = desc->n_q_heads / desc->n_kv_heads;
    p.nsplit = (int32_t)plan.nsplit;
    p.chunk = (int32_t)plan.chunk;
    p.scale_log2 = eff_scale(desc) * 1.4426950408889634f;
    return to_status(launch_weigh(p, desc->head_dim, desc->dtype, plan.way, plan.held, (hipStream_t)stream));
}

size_t kvr_workspace_bytes_evict(const kvr_desc *desc, int64_t L) {
    if (check_desc(desc) != KVR_OK || L < 0 || L > kMaxRows) return (size_t)-1;
    return L <= kHeldRows ? 0 : (size_t)desc->n_kv_heads * (size_t)L * sizeof(int32_t);
}

int kvr_cache_evict(const kvr_desc *desc, const void *kcache, const void *vcache, int64_t L, const float *weight,
                    int64_t n_first, int64_t n_last, int64_t n_keep, void *kout, void *vout, int64_t capacity_out,
                    float *weight_out, int32_t *index, void *ws, size_t ws_bytes, void *stream) {
    const int st = check_desc(desc);
    if (st) return st;
    if (L < 0 || L > kMaxRows || n_first < 0 || n_last < 0 || n_keep < 0 || n_keep > L) return KVR_ERR_SHAPE;
    if (n_first > n_keep || n_last > n_keep - n_first) return KVR_ERR_SHAPE;
    if (capacity_out < 0 || capacity_out > kMaxKeys) return KVR_ERR_SHAPE;
    if (L > desc->capacity || n_keep > capacity_out) return KVR_ERR_CAPACITY;
    if (n_keep == 0) return KVR_OK;
    if (!kcache || !vcache || !weight || !kout || !vout) return KVR_ERR_NULL;
    const void *const ptrs[] = {kcache, vcache, kout, vout, ws};
    for (const void *p : ptrs)
        if (!aligned(p, 16)) return KVR_ERR_ALIGN;
    if (!aligned(weight, 4) || !aligned(weight_out, 4) || !aligned(index, 4)) return KVR_ERR_ALIGN;
    const size_t need = kvr_workspace_bytes_evict(desc, L);
    if (need && (!ws || ws_bytes < need)) return KVR_ERR_WORKSPACE;
    // rows move without an order: no output may share memory with anything else of the call
    const size_t hkv = (size_t)desc->n_kv_heads, row = (size_t)desc->head_dim * elt_bytes(desc);
    const struct { const void *p; size_t n; bool out; } buf[] = {
        {kcache, hkv * (size_t)desc->capacity * row, false}, {vcache, hkv * (size_t)desc->capacity * row, false},
        {weight, hkv * (size_t)desc->capacity * 4, false},   {kout, hkv * (size_t)capacity_out * row, true},
        {vout, hkv * (size_t)capacity_out * row, true},      {weight_out, hkv * (size_t)capacity_out * 4, true},
        {index, hkv * (size_t)n_keep * 4, true},             {ws, need, true}};
    for (size_t a = 0; a < sizeof buf / sizeof buf[0]; ++a)
        for (size_t b = 0; b < a; ++b)
            if ((buf[a].out || buf[b].out) && overlap(buf[a].p, buf[a].n, buf[b].p, buf[b].n)) return KVR_ERR_SHAPE;

    EvictParams p;
    memset(&p, 0, sizeof p);
    p.kc = kcache; p.vc = vcache; p.weight = weight;
    p.ko = kout; p.vo = vout; p.weight_out = weight_out; p.index = index;
    p.list = (int32_t *)ws;
    p.cap = desc->capacity;
    p.cap_out = capacity_out;
    p.L = (int32_t)L;
    p.n_first = (int32_t)n_first;
    p.n_last = (int32_t)n_last;
    p.n_keep = (int32_t)n_keep;
    p.n_kv_heads = desc->n_kv_heads;
    p.row_chunks = desc->head_dim * elt_bytes(desc) / 16;
    while ((1 << p.chunk_bits) < p.row_chunks) ++p.chunk_bits;
    // workgroups of a kv head: all compute units, unless that leaves one too few rows
    const int64_t parts = ceil_div(n_keep, kRowsPerPart), most = kCus / desc->n_kv_heads;
    p.parts = (int32_t)(parts < most ? parts : most > 1 ? most : 1);
    return to_status(launch_evict(p, (hipStream_t)stream));
}

}  // extern "C"
