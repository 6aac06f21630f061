// shared.hip -- attention of a batch of readers that share a long cached prefix
// and each have cached rows of their own.
//
//   out[r, i, h] = softmax over [prefix 0 .. L-1 | own rows 0 .. len_r - 1 | new rows 0 .. i]
//
// Three kinds of work in one launch, joined by a merge of log-sum-exp partials:
//   prefix  every reader sees the whole prefix, so the query rows of all readers of
//           a kv head are packed into tiles and the prefix is read once for all of
//           them (once for each row tile from the caches, once from HBM)
//   own     the rows of one reader and kv head over that reader's cached rows
//   new     the rows of one reader and kv head over its new rows, causally; the last
//           row tile stores these to the reader's cache
// Prefix and own items are a workgroup's over a range of cached keys, in one of two ways:
//   by keys   up to 16 query rows (fp32: 32 a tile): the four waves hold the same rows and
//             take the range's stages in turn, K and V straight from memory
//             (attn_direct.hpp), no barrier until their partials are joined
//   by rows   more rows, 16-bit: each wave holds 16 or 32 rows of its own and the
//             stages go through LDS once for all four (attn_ring.hpp)
// A new item is one wave's.  Each item's partial (M, l, O) is a record of the workspace.  A
// short call is a launch of its own (shared_alone_kernel): no records, no merge.
// The lengths are read on the device: a captured graph serves every step of a decode.
//
// Measured, items and merge, in us (32 query heads, 8 kv heads, head_dim 128, one MI355X):
//   64 readers of 32768 keys, 300 .. 1000 own rows   75.1 + 6.3   304 MB of keys and values, 4.0 TB/s
//   64 readers of 3774 keys, 24 .. 512 own rows      26.9 + 4.2   87 MB, 2.8 TB/s
//   16 readers x 4 tokens, 16384 keys                35.0 + 6.2   17.4 GFLOP, 0.50 PFLOP/s
//   9 readers of 3774 keys                           10.4 + 3.9   latency: lengths, rotation, first keys, records
//   3 readers x 5 tokens, 945 keys, head_dim 64, fp32   5.9 + 3.0   latency
//   8 readers x 256 tokens, 3774 keys, 100 own rows  230 + 33     a later turn's prompt: new items
//   8 readers x 24 tokens, the same                  30.4 + 7.4
// By rows, 32768 keys for 256 rows of a kv head take 58.5 us (0.59 PFLOP/s), of which 10 are
// the launch, the first stage and the records' writes, and 3 references that move in the
// first stages (55.6 with references that only move far below the maximum, which rounds
// weights that hold much of their row): a SIMD has one prefix wave, whose exponentials and
// matrix products (34 of 16 clocks a stage) are in order, one after the other; the other
// place on the SIMD is the own items'.  Twice the workgroups: 51.6 us, but twice the records to
// write and merge (9.2 instead of 6.4 us), 36.3 + 9.0 in the third line; eight waves in two
// teams that join in LDS took 18.5 us for 16384 keys instead of 23, but leave the own items no
// place: 89 us for the first line.
// A later turn's prompt is bound by its new items: a wave loads, rotates and takes 16 new keys at
// a time, one after the other.
#include "attn_ring.hpp"
#include "readers_internal.hpp"

namespace kvr {
namespace {

using namespace dev;

constexpr int WAVES = 4;

// 16-bit operations of both ways
template <class E, int D>
struct Op : Op16<E, D> {
    using Ring = Ring16<E, D>;
};

template <class OP, int RT>
struct Rows {
    typename OP::Q q[RT];
    f32x4 o[RT][OP::NT];
    float m[RT];             // reference of the row (log2 domain)
    typename OP::L l[RT];    // its sum
    typename OP::Mark t[RT]; // what its weights must not exceed
    int tok[RT];             // the row's token, of its reader's new ones
    int at[RT];              // the row in out, -1: none
};

// Cached rows of reader r, or -1 if it takes no part
__device__ __forceinline__ int reader_len(const SharedParams &p, int r) {
    const int len = p.len[r];
    return len >= 0 && (int64_t)len + (p.append ? p.S : 0) <= p.tcap ? len : -1;
}

// The query rows of a tile: row r0 + 16 rt + i of `nrows` rows, which are the heads
// of kv head hd for token tok0, then for the next token; past the last one it again, not
// to be stored.  len: the cached rows of the tokens' reader, where it is one (else -1)
template <class OP, int RT>
__device__ __forceinline__ void take_rows(const SharedParams &p, Rows<OP, RT> &R, int hd, int tok0, int r0, int nrows, int i,
                                          int g, int len) {
    const int G = p.group;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + 16 * rt + i;
        const int rr = min(r, nrows - 1);
        const int tk = rr / G;
        const int tok = tok0 + tk;
        const int at = tok * p.n_q_heads + hd * G + (rr - tk * G);
        OP::load_q(R.q[rt], (const unsigned char *)p.q + (int64_t)at * OP::ROWB, g);
        if (p.rope) {
            const int rd = tok / p.S;
            const int64_t pos = p.pos0 + (len >= 0 ? len : max(reader_len(p, rd), 0)) + (tok - rd * p.S);
            OP::rotate_q(R.q[rt], p.rope + pos * OP::DIM, g);
        }
        R.at[rt] = r < nrows ? at : -1;
        R.tok[rt] = tk;
    }
    __builtin_amdgcn_sched_barrier(0);      // the outputs' registers hold loads until here
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        R.m[rt] = -1e30f;
        R.l[rt] = OP::no_sum();
        R.t[rt] = OP::mark(R.l[rt]);
#pragma unroll
        for (int t = 0; t < OP::NT; ++t) R.o[rt][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
}

struct Nothing {
    __device__ __forceinline__ void operator()() const {}
};

// The scores of a stage of n cached keys become weights 2^(c2 s - m).
// The reference m does not follow the maximum (attn_direct.hpp: when it moves): whether a
// weight exceeds its row's mark is seen in the operands' bits, no maximum is taken
// otherwise.  A row's sum grows, its mark only here, so this is entered more often
// than a reference moves: on rows without peaks, in the first three or four stages.
// among(): work that does not depend on it, to be issued among the exponentials.
template <class OP, int RT, class AMONG>
__device__ __forceinline__ void softmax_step(Rows<OP, RT> &R, float (&s)[RT][OP::NS], typename OP::P (&w)[RT], int n,
                                             float c2, int g, AMONG among) {
    if (n < OP::KEYS) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int e = 0; e < OP::NS; ++e)
                if (OP::key_of(e, g) >= n) s[rt][e] = -INFINITY;
    }
    auto weights = [&](int rt) {      // lanes with a weight above their row's mark
        float p[OP::NS];
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e], c2, -R.m[rt]));
        OP::weights(w[rt], p);
        return __ballot(OP::above(OP::peak(w[rt]), R.t[rt]));
    };
    among();
    uint64_t above[RT], any = 0;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) any |= above[rt] = weights(rt);
    if (any) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (!above[rt]) continue;
            float mx = s[rt][0];
#pragma unroll
            for (int e = 0; e < OP::NS; ++e) mx = fmaxf(mx, s[rt][e]);
            mx = quad_max(mx);
            const bool moves = OP::moves(above[rt], threadIdx.x & 15, __builtin_amdgcn_exp2f(__builtin_fmaf(mx, c2, -R.m[rt])), R.l[rt]);
            if (!__ballot(moves)) continue;
            const float mn = moves ? mx * c2 - OP::kLift : R.m[rt];      // each row for itself
            const float alpha = __builtin_amdgcn_exp2f(R.m[rt] - mn);
            R.m[rt] = mn;
            R.l[rt] *= alpha;
#pragma unroll
            for (int t = 0; t < OP::NT; ++t) R.o[rt][t] *= alpha;
            weights(rt);
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) OP::add(R.l[rt], w[rt]);
    if (any) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) R.t[rt] = OP::mark(R.l[rt]);
    }
}

// Where row `at` of record `rec` keeps O, and (M, l)
template <class OP>
__device__ __forceinline__ float *record_o(const SharedParams &p, int64_t rec, int at) {
    return p.ws + (rec * p.rows + at) * OP::DIM;
}
template <class OP>
__device__ __forceinline__ float2 *record_ml(const SharedParams &p, int64_t rec, int at) {
    return (float2 *)(p.ws + (int64_t)p.nrec * p.rows * OP::DIM) + rec * p.rows + at;
}

// Valid rows of stage t of KEYS rows, of n rows (0 past the last stage)
template <int KEYS>
__device__ __forceinline__ int stage_rows(int64_t n, int t) {
    n -= (int64_t)t * KEYS;
    return (int)(n < 0 ? 0 : n > KEYS ? KEYS : n);
}

// ---- by keys
// Consecutive cached rows, in stages
template <class OP>
struct Range {
    uint64_t kb, vb;
    int64_t nkeys;
    __device__ __forceinline__ int stages() const { return (int)((nkeys + OP::KEYS - 1) / OP::KEYS); }
    __device__ __forceinline__ int count(int t) const { return stage_rows<OP::KEYS>(nkeys, t); }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t k(int t) const { return rows(kb, t); }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t v(int t) const { return rows(vb, t); }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t rows(uint64_t base, int t) const {
        return row_rsrc(base + (uint64_t)t * OP::KEYS * OP::ROWB, count(t), OP::ROWB, OP::ROWB);
    }
};

// One after the other
template <class OP>
struct Ranges {
    Range<OP> a, b;
    int na;      // stages of a
    __device__ __forceinline__ int stages() const { return na + b.stages(); }
    __device__ __forceinline__ int count(int t) const { return t < na ? a.count(t) : b.count(t - na); }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t k(int t) const { return t < na ? a.k(t) : b.k(t - na); }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t v(int t) const { return t < na ? a.v(t) : b.v(t - na); }
};

// A wave's stages first, first + STEP, ... of a range.  K and V have one set of registers
// each: the next stage's K is asked for when the scores are done, its V when the outputs
// are.  begin() asks for the first; the caller takes its rows meanwhile.
template <class OP, int RT, int STEP>
struct ByKeys {
    typename OP::K k;
    typename OP::V v;
    __device__ __forceinline__ void begin(const Range<OP> &r, int first, int i, int g) {
        OP::load_k(k, r.k(first), OP::ROWB, i, g);
        OP::load_v(v, r.v(first), OP::ROWB, i, g);
    }
    template <class RANGE>
    __device__ __forceinline__ void run(const RANGE &r, int first, Rows<OP, RT> &R, float c2, int i, int g) {
        const int nst = r.stages();
        for (int t = first; t < nst; t += STEP) {
            float s[RT][OP::NS];
            typename OP::P w[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) OP::scores(k, R.q[rt], s[rt]);
            __builtin_amdgcn_sched_barrier(0);
            OP::load_k(k, r.k(t + STEP), OP::ROWB, i, g);
            __builtin_amdgcn_sched_barrier(0);
            softmax_step<OP, RT>(R, s, w, r.count(t), c2, g, Nothing());
            OP::template accumulate<RT>(v, w, R.o);
            __builtin_amdgcn_sched_barrier(0);
            OP::load_v(v, r.v(t + STEP), OP::ROWB, i, g);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// LDS of the join of one row tile by W waves: O of every wave, component c of the lane's
// four in row c, then (m, l)
template <class OP, int W>
constexpr int obuf_floats() {
    return W * 4 * 64 * OP::NT;
}
template <class OP, int W>
constexpr int join_floats() {
    return obuf_floats<OP, W>() + 2 * W * 64;
}

// Every wave posts its partial of a row tile; after a barrier a wave joins, in wave order,
// component c of each row's outputs (head-dim indices NT (4 g + c) .. of the lane) over
// the larger reference M
template <class OP, int W>
__device__ __forceinline__ void post(const f32x4 (&o)[OP::NT], float m, float l, float *lds, int wave, int lane) {
    constexpr int NT = OP::NT;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int t = 0; t < NT; t += 4)
            *(f32x4 *)(lds + ((wave * 4 + c) * 64 + lane) * NT + t) = (f32x4){o[t][c], o[t + 1][c], o[t + 2][c], o[t + 3][c]};
    *(float2 *)(lds + obuf_floats<OP, W>() + (wave * 64 + lane) * 2) = make_float2(m, l);
}
template <class OP, int W>
__device__ __forceinline__ void joined(const float *lds, int c, int lane, f32x4 (&acc)[OP::NT / 4], float &M, float &l) {
    constexpr int NT = OP::NT;
    const float *ml = lds + obuf_floats<OP, W>();
    M = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < NT / 4; ++t) acc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < W; ++s) M = fmaxf(M, ml[(s * 64 + lane) * 2]);
#pragma unroll
    for (int s = 0; s < W; ++s) {
        const float2 w = *(const float2 *)(ml + (s * 64 + lane) * 2);
        const float a = __builtin_amdgcn_exp2f(w.x - M);
        l = __builtin_fmaf(a, w.y, l);
#pragma unroll
        for (int t = 0; t < NT / 4; ++t) {
            const f32x4 x = *(const f32x4 *)(lds + ((s * 4 + c) * 64 + lane) * NT + 4 * t);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] = __builtin_fmaf(a, x[e], acc[t][e]);
        }
    }
}

// The partials of the workgroup's waves to record `rec`
template <class OP, int RT>
__device__ __forceinline__ void join(const SharedParams &p, Rows<OP, RT> &R, float *lds, int64_t rec, int wave, int lane) {
    const int g = lane >> 4;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (rt) __syncthreads();
        post<OP, WAVES>(R.o[rt], R.m[rt], OP::total(R.l[rt]), lds, wave, lane);
        __syncthreads();
        f32x4 acc[OP::NT / 4];
        float M, l;
        joined<OP, WAVES>(lds, wave, lane, acc, M, l);
        if (R.at[rt] < 0) continue;
        float *po = record_o<OP>(p, rec, R.at[rt]) + OP::NT * (4 * g + wave);
#pragma unroll
        for (int t = 0; t < OP::NT / 4; ++t) *(f32x4 *)(po + 4 * t) = acc[t];
        if (wave == 0 && g == 0) *record_ml<OP>(p, rec, R.at[rt]) = make_float2(M, l);
    }
}

// ---- by rows
// Scores of a stage's keys, from LDS
template <class OP, class RG, int RT>
__device__ __forceinline__ void row_scores(const Rows<OP, RT> &R, const unsigned char *ks_, uint32_t ka, float (&s)[RT][OP::NS]) {
    static_assert(RG::KEYS == OP::KEYS, "one operand's keys in a stage");
    f32x4 a[RT][2];
#pragma unroll
    for (int ks = 0; ks < OP::NK; ++ks)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4 k = RG::row_frag(ks_, ka, h, ks);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                a[rt][h] = OP::mfma(k, R.q[rt].f[ks], ks ? a[rt][h] : (f32x4){0.f, 0.f, 0.f, 0.f});
        }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) s[rt][e] = a[rt][e >> 2][e & 3];
}

// The stages of `nkeys` cached rows at kb / vb, in SLOTS slots of LDS: the next stage's keys
// and one's values are read while the others are on their way.  begin() asks for the
// first; the caller takes its rows meanwhile, and run() first waits for all of it: loads
// that the compiler knows of must not be on their way when the loop begins, or it waits
// for every load in it.
constexpr int SLOTS = 4;

template <class OP, class RG, int RT>
struct ByRows {
    static_assert(SLOTS % 2 == 0, "two sets of scores take turns");
    using Scores = float[RT][OP::NS];
    uint64_t kb, vb;
    int64_t nkeys;
    unsigned char *lds;
    int nst, ragged, wave, lane;      // ragged: the stage that ends inside, or -1
    __device__ __forceinline__ void load(int t, int slot) const {
        const uint64_t off = (uint64_t)t * RG::KEYS * OP::ROWB;
        const int n = stage_rows<RG::KEYS>(nkeys, t);
        unsigned char *to = lds + slot * 2 * RG::HALF;
        if (n == RG::KEYS) {
            RG::template load_all<false>(kb + off, to, wave, lane);
            RG::template load_all<true>(vb + off, to + RG::HALF, wave, lane);
        } else {
            RG::template load<false>(kb + off, OP::ROWB, n, to, wave, lane);
            RG::template load<true>(vb + off, OP::ROWB, n, to + RG::HALF, wave, lane);
        }
    }
    __device__ __forceinline__ void begin(uint64_t kb_, uint64_t vb_, int64_t nkeys_, unsigned char *lds_, int wave_, int lane_) {
        kb = kb_; vb = vb_; nkeys = nkeys_; lds = lds_; wave = wave_; lane = lane_;
        nst = (int)((nkeys + RG::KEYS - 1) / RG::KEYS);
        ragged = nkeys % RG::KEYS ? nst - 1 : -1;
#pragma unroll
        for (int t = 0; t < SLOTS - 1; ++t)
            if (t < nst) load(t, t);
    }
    // Zeros in the place of values behind the last key, whose weights are 0: the row that
    // load() repeats there may hold an infinity.  Between the barrier behind which the stage has
    // landed and that of the stage itself.
    __device__ __forceinline__ void clean(int t, int slot) const {
        const int n = stage_rows<RG::KEYS>(nkeys, t);
        unsigned char *to = lds + (slot * 2 + 1) * RG::HALF;
        for (int at = n * OP::ROWB + 16 * (wave * 64 + lane); at < RG::HALF; at += 16 * 64 * WAVES)
            *(u32x4 *)(to + at) = (u32x4){0u, 0u, 0u, 0u};
    }
    // Stage t, in slot SLOT: its scores s become weights, while the matrix units make those of
    // the next stage.  32768 keys, 256 rows of a kv head, with references that hardly move: 61 us
    // one after the other, 57.5 so, and 55.6 with half of V asked for before the exponentials.
    template <int SLOT>
    __device__ __forceinline__ void stage(Rows<OP, RT> &R, int t, Scores &s, Scores &next, float c2, uint32_t ka, uint32_t va,
                                          int g) const {
        // this wave's part of stage t + 1 has landed (the SLOTS - 3 behind it may be on their
        // way); behind the barrier everybody's has, and nobody reads the slot of stage t - 1
        // any more
        if (t + SLOTS - 2 < nst) wait_vmcnt<(SLOTS - 3) * 2 * RG::LOADS>();
        else wait_vmcnt<0>();
        barrier_lds();
        if (t + SLOTS - 1 < nst) load(t + SLOTS - 1, (SLOT + SLOTS - 1) % SLOTS);
        if (t + 1 == ragged) clean(t + 1, (SLOT + 1) % SLOTS);
        const unsigned char *vs = lds + SLOT * 2 * RG::HALF + RG::HALF;
        const unsigned char *k1 = lds + (SLOT + 1) % SLOTS * 2 * RG::HALF;      // (behind the last stage: anything, not used)
        typename OP::P w[RT];
        constexpr int NT = OP::NT;
        u32x4 v[NT];      // half of it is asked for here, half when the weights' registers are free
        softmax_step<OP, RT>(R, s, w, stage_rows<RG::KEYS>(nkeys, t), c2, g, [&]() {
            row_scores<OP, RG, RT>(R, k1, ka, next);
#pragma unroll
            for (int u = 0; u < NT / 2; ++u) v[u] = RG::col_frag(vs, va, u);
        });
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = NT / 2; u < NT; ++u) v[u] = RG::col_frag(vs, va, u);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < OP::NT; ++u)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) R.o[rt][u] = OP::mfma(v[u], w[rt].f, R.o[rt][u]);
    }
    template <int SLOT>
    __device__ __forceinline__ void stages(Rows<OP, RT> &R, int t, Scores &s, Scores &next, float c2, uint32_t ka, uint32_t va,
                                           int g) const {
        if (t >= nst) return;
        stage<SLOT>(R, t, s, next, c2, ka, va, g);
        if constexpr (SLOT + 1 < SLOTS) stages<SLOT + 1>(R, t + 1, next, s, c2, ka, va, g);
    }
    __device__ __forceinline__ void run(Rows<OP, RT> &R, float c2) const {
        const int i = lane & 15, g = lane >> 4;
        const uint32_t ka = RG::row_at(i, g), va = RG::col_at(i, g);
        if (nst == 0) return;
        wait_vmcnt<0>();
        barrier_lds();
        if (ragged == 0) clean(0, 0);
        Scores s, next;
        row_scores<OP, RG, RT>(R, lds, ka, s);
        for (int t = 0; t < nst; t += SLOTS) stages<0>(R, t, s, next, c2, ka, va, g);
    }
};

// The partial of the wave's own rows
template <class OP, int RT>
__device__ __forceinline__ void put_rows(const SharedParams &p, const Rows<OP, RT> &R, int64_t rec, int g) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float l = OP::total(R.l[rt]);
        if (R.at[rt] < 0) continue;
        float *po = record_o<OP>(p, rec, R.at[rt]) + 4 * g;
#pragma unroll
        for (int t = 0; t < OP::NT; ++t) *(f32x4 *)(po + 16 * t) = R.o[rt][t];
        if (g == 0) *record_ml<OP>(p, rec, R.at[rt]) = make_float2(R.m[rt], l);
    }
}

// ---- items
// WAY: 1 or 2: by keys, that many 16-row tiles; kByRows + 1 or 2: by rows, that many in
// each wave
constexpr int tiles_of(int way) { return way > kByRows ? way - kByRows : way; }
constexpr int rows_of(int way) { return way > kByRows ? 64 * (way - kByRows) : 16 * way; }

template <class OP, int WAY>
constexpr int lds_bytes() {
    if constexpr (WAY > kByRows) return SLOTS * 2 * OP::Ring::HALF;
    else return join_floats<OP, WAVES>() * 4;
}

// Rows r0 .. of `nrows` query rows (take_rows) over `nkeys` cached rows at k / v, to record
// `rec`
struct Item {
    uint64_t k, v;
    int64_t nkeys, rec;
    int hd, tok0, r0, nrows, len;
};

template <class OP, int WAY>
__device__ __forceinline__ void attend(const SharedParams &p, const Item &it, unsigned char *lds, int wave, int lane) {
    constexpr int RT = tiles_of(WAY);
    const int i = lane & 15, g = lane >> 4;
    Rows<OP, RT> R;
    if constexpr (WAY > kByRows) {
        ByRows<OP, typename OP::Ring, RT> keys;
        keys.begin(it.k, it.v, it.nkeys, lds, wave, lane);
        take_rows(p, R, it.hd, it.tok0, it.r0 + wave * 16 * RT, it.nrows, i, g, it.len);
        keys.run(R, p.scale_log2);
        put_rows<OP, RT>(p, R, it.rec, g);
    } else {
        const Range<OP> range{it.k, it.v, it.nkeys};
        ByKeys<OP, RT, WAVES> keys;
        keys.begin(range, wave, i, g);
        take_rows(p, R, it.hd, it.tok0, it.r0, it.nrows, i, g, it.len);
        keys.run(range, wave, R, p.scale_log2, i, g);
        join<OP, RT>(p, R, (float *)lds, it.rec, wave, lane);
    }
}

// Prefix item (oct, in8): the (kv head, split) pairs in groups of eight, a group's row
// tiles one after the other.  Blocks eight apart share an XCD, so the tiles that read
// one range of prefix rows find it in one L2.
template <class OP, int WAY>
__device__ __forceinline__ void prefix_item(const SharedParams &p, uint32_t oct, uint32_t in8, unsigned char *lds, int wave,
                                            int lane) {
    const uint32_t pair = oct / p.p_tiles * 8 + in8;
    const int split = (int)(pair / p.n_kv_heads);
    if (split >= p.np) return;
    Item it;
    it.hd = (int)(pair % p.n_kv_heads);
    const int64_t kb = split * p.chunk;
    const uint64_t off = ((uint64_t)it.hd * p.cap + kb) * OP::ROWB;
    it.k = (uint64_t)(uintptr_t)p.kc + off;
    it.v = (uint64_t)(uintptr_t)p.vc + off;
    it.nkeys = min(p.chunk, p.L - kb);
    it.rec = split;
    it.tok0 = 0;
    it.r0 = (int)(oct % p.p_tiles) * rows_of(WAY);
    it.nrows = p.n * p.S * p.group;
    it.len = -1;
    attend<OP, WAY>(p, it, lds, wave, lane);
}

// Own item x: (split, reader, row tile, kv head), kv head
// fastest.  The splits have equal shares of the cached rows, in whole stages.
template <class OP, int WAY>
__device__ __forceinline__ void own_item(const SharedParams &p, uint32_t x, unsigned char *lds, int wave, int lane) {
    constexpr int KEYS = OP::KEYS;
    Item it;
    it.hd = (int)(x % p.n_kv_heads);
    x /= p.n_kv_heads;
    const int tile = (int)(x % p.t_tiles);
    x /= p.t_tiles;
    const int rd = (int)(x % p.n), split = (int)(x / p.n);
    if (split >= p.nt) return;
    it.len = reader_len(p, rd);
    if (it.len < 0) return;
    const uint32_t chunk = (((uint32_t)it.len + p.nt - 1) / p.nt + KEYS - 1) / KEYS * KEYS;
    const int64_t kb = min((int64_t)split * chunk, (int64_t)it.len);
    it.nkeys = min((int64_t)chunk, it.len - kb);
    if (it.nkeys == 0) {      // its rows' sums alone: the merge takes no output from a record with none
        const int r = tile * rows_of(WAY) + (int)threadIdx.x;
        if (threadIdx.x < rows_of(WAY) && r < p.S * p.group) {
            const int tk = r / p.group, at = (rd * p.S + tk) * p.n_q_heads + it.hd * p.group + (r - tk * p.group);
            *record_ml<OP>(p, p.np + split, at) = make_float2(-1e30f, 0.f);
        }
        return;
    }
    const uint64_t off = (((uint64_t)rd * p.n_kv_heads + it.hd) * p.tcap + kb) * OP::ROWB;
    it.k = (uint64_t)(uintptr_t)p.kt + off;
    it.v = (uint64_t)(uintptr_t)p.vt + off;
    it.rec = p.np + split;
    it.tok0 = rd * p.S;
    it.r0 = tile * rows_of(WAY);
    it.nrows = p.S * p.group;
    attend<OP, WAY>(p, it, lds, wave, lane);
}

// ---- new rows
// Rows r0 .. r0 + 15 of reader rd and kv head hd over its new rows, causally: a wave's
// partial, for done(R, g).  store: and these rows to the reader's cache, behind its len
// rows there.
template <class OP, class DONE>
__device__ __forceinline__ void attend_new(const SharedParams &p, int rd, int hd, int r0, int len, bool store, int lane, DONE done) {
    constexpr int KEYS = 16;      // (one part of a 16-bit stage: fewer registers)
    int i = lane & 15, g = lane >> 4;
    const int nrows = p.S * p.group;
    const int seen = min(p.S, (min(r0 + 16, nrows) - 1) / p.group + 1);      // new rows that a row sees
    const uint32_t nb = (uint32_t)p.n_kv_heads * OP::ROWB;
    const uint64_t src = ((uint64_t)rd * p.S * p.n_kv_heads + hd) * OP::ROWB;
    const uint64_t to = (((uint64_t)rd * p.n_kv_heads + hd) * p.tcap + len) * OP::ROWB;
    Rows<OP, 1> R;
    typename OP::K k;
    typename OP::V v;
    auto load = [&](int c0) {
        const int n = min(seen - c0, KEYS);
        const uint64_t at = src + (uint64_t)c0 * nb;
        OP::template load_k<1>(k, row_rsrc((uint64_t)(uintptr_t)p.kn + at, n, nb, OP::ROWB), nb, i, g);
        OP::template load_v<1>(v, row_rsrc((uint64_t)(uintptr_t)p.vn + at, n, nb, OP::ROWB), nb, i, g);
    };
    load(0);
    take_rows(p, R, hd, rd * p.S, r0, nrows, i, g, len);
    for (int c0 = 0; c0 < seen; c0 += KEYS) {
        const int n = min(seen - c0, KEYS);
        asm volatile("" : "+v"(i), "+v"(g));      // addresses are made in the loop: registers for all are not there
        if (c0) load(c0);
        if (p.rope) OP::template rotate_k<1>(k, p.rope + (p.pos0 + len + c0) * OP::DIM, n, i, g);
        if (store)
            OP::template store<1>(k, v, (unsigned char *)p.kt + to + (uint64_t)c0 * OP::ROWB,
                                  (unsigned char *)p.vt + to + (uint64_t)c0 * OP::ROWB, n, i, g);
        __builtin_amdgcn_sched_barrier(0);
        float s[OP::NS];
        typename OP::P w[1];
        OP::scores(k, R.q[0], s);
        const int lim = min(n - 1, R.tok[0] - c0);
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) {
            s[e] = OP::key_of(e, g) > lim ? -INFINITY : s[e];
            mx = fmaxf(mx, s[e]);
        }
        const float mn = fmaxf(R.m[0], quad_max(mx) * p.scale_log2 - OP::kLift);
        if (c0) {
            const float alpha = __builtin_amdgcn_exp2f(R.m[0] - mn);
            R.l[0] *= alpha;
#pragma unroll
            for (int t = 0; t < OP::NT; ++t) R.o[0][t] *= alpha;
        }
        R.m[0] = mn;
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], p.scale_log2, -mn));
        OP::weights(w[0], s);
        OP::add(R.l[0], w[0]);
        // A value that is no number must not reach the rows before it, whose weight for it is
        // 0: a stage that has one goes key by key, each for the rows that see it.
        if (__ballot(!OP::finite(v)) == 0) {
            OP::template accumulate<1>(v, w, R.o);
        } else {
            for (int c = 0; c < n; ++c) {
                const bool sees[1] = {c0 + c <= R.tok[0]};
                OP::template accumulate_key<1>(v, w, R.o, c, sees, g);
            }
        }
    }
    done(R, g);
}

// New item x, a wave's: (reader, 16-row tile, kv head), kv head fastest.  The last tile sees
// all new rows, and stores them.
template <class OP>
__device__ __forceinline__ void new_item(const SharedParams &p, uint32_t x, int lane) {
    constexpr int NT = OP::NT;
    const int hd = (int)(x % p.n_kv_heads);
    x /= p.n_kv_heads;
    const int tiles = (p.S * p.group + 15) / 16;
    const int tile = (int)(x % tiles), rd = (int)(x / tiles);
    if (rd >= p.n) return;
    const int len = reader_len(p, rd);
    if (len < 0) return;
    attend_new<OP>(p, rd, hd, tile * 16, len, p.append && tile == tiles - 1, lane, [&](const Rows<OP, 1> &R, int g) {
        const float l = OP::total(R.l[0]);
        if (R.at[0] < 0) return;
        float *po = record_o<OP>(p, p.nrec - 1, R.at[0]) + NT * 4 * g;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int t = 0; t < NT; t += 4)
                *(f32x4 *)(po + NT * c + t) = (f32x4){R.o[0][t][c], R.o[0][t + 1][c], R.o[0][t + 2][c], R.o[0][t + 3][c]};
        if (g == 0) *record_ml<OP>(p, p.nrec - 1, R.at[0]) = make_float2(R.m[0], l);
    });
}

// PW, OW: the ways of prefix and own items
template <class OP, int PW, int OW>
__global__ __launch_bounds__(256, 2) void shared_kernel(const SharedParams p) {
    constexpr int LP = lds_bytes<OP, PW>(), LO = lds_bytes<OP, OW>();
    __shared__ __attribute__((aligned(1024))) unsigned char lds[LP > LO ? LP : LO];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Blocks in groups of eight, one for each XCD: prefix items, own items, new items.
    const uint32_t oct = blockIdx.x / 8, in8 = blockIdx.x % 8;
    if (oct < p.oct_own) prefix_item<OP, PW>(p, oct, in8, lds, wave, lane);
    else if (oct < p.oct_new) own_item<OP, OW>(p, (oct - p.oct_own) * 8 + in8, lds, wave, lane);
    else new_item<OP>(p, ((oct - p.oct_new) * 8 + in8) * WAVES + wave, lane);
}

// ---- alone
// A short call in one launch: a workgroup does all that the rows of one reader and kv head
// see, the last wave the new rows, the others the stages of prefix and own rows in turn.
// Every reader reads the prefix anew, no partial goes through memory.  8.3 us for 2 readers of
// 255 keys: the launch, lengths, rotation, a few stages' round trips, the join.
constexpr int ALONE_WAVES = 8;

template <class OP>
__global__ __launch_bounds__(64 * ALONE_WAVES) void shared_alone_kernel(const SharedParams p) {
    constexpr int W = ALONE_WAVES;
    __shared__ __attribute__((aligned(16))) float lds[join_floats<OP, W>()];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hd = blockIdx.x % p.n_kv_heads, rd = blockIdx.x / p.n_kv_heads;
    Rows<OP, 1> R;
    int len;
    if (wave == W - 1) {
        len = reader_len(p, rd);
        if (len >= 0)
            attend_new<OP>(p, rd, hd, 0, len, p.append != 0, lane, [&](const Rows<OP, 1> &N, int) {
                post<OP, W>(N.o[0], N.m[0], OP::total(N.l[0]), lds, wave, lane);
            });
    } else {
        const uint64_t at = (uint64_t)hd * p.cap * OP::ROWB;
        Ranges<OP> keys;
        keys.a = Range<OP>{(uint64_t)(uintptr_t)p.kc + at, (uint64_t)(uintptr_t)p.vc + at, p.L};
        keys.na = keys.a.stages();
        ByKeys<OP, 1, W - 1> by;
        if (wave < keys.na) by.begin(keys.a, wave, i, g);
        len = reader_len(p, rd);
        const uint64_t own = ((uint64_t)rd * p.n_kv_heads + hd) * p.tcap * OP::ROWB;
        keys.b = Range<OP>{(uint64_t)(uintptr_t)p.kt + own, (uint64_t)(uintptr_t)p.vt + own, max(len, 0)};
        if (wave >= keys.na) by.begin(keys.b, wave - keys.na, i, g);
        if (len >= 0) {
            take_rows(p, R, hd, rd * p.S, 0, p.S * p.group, i, g, len);
            by.run(keys, wave, R, p.scale_log2, i, g);
            post<OP, W>(R.o[0], R.m[0], OP::total(R.l[0]), lds, wave, lane);
        }
    }
    if (len < 0) return;      // all waves
    __syncthreads();
    if (wave >= 4 || R.at[0] < 0) return;
    f32x4 acc[OP::NT / 4];
    float M, l;
    joined<OP, W>(lds, wave, lane, acc, M, l);
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int t = 0; t < OP::NT / 4; ++t)
        OP::put4((unsigned char *)p.out + (int64_t)R.at[0] * OP::ROWB, OP::NT * (4 * g + wave) + 4 * t, acc[t][0] * inv,
                 acc[t][1] * inv, acc[t][2] * inv, acc[t][3] * inv);
}

// out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over the records of a row: 17 records
// of 2048 rows, 18 MB, in 6.1 us, the launch and three round trips among them.  A wave
// takes 64 / (D / 4) rows, four values a lane; the workgroup's waves take the records in
// turn, and their sums are joined in wave order.
constexpr int MERGE_WAVES = 4;

template <class OP>
__global__ __launch_bounds__(64 * MERGE_WAVES) void shared_merge_kernel(const SharedParams p) {
    constexpr int D = OP::DIM, LANES = D / 4, BATCH = 4;
    __shared__ f32x4 sums[MERGE_WAVES][64];
    __shared__ float2 mls[MERGE_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t at_row = (int64_t)blockIdx.x * (64 / LANES) + lane / LANES, row = min(at_row, p.rows - 1);
    const int d = lane % LANES * 4;
    const bool on = at_row < p.rows && reader_len(p, (int)(row / ((int64_t)p.n_q_heads * p.S))) >= 0;
    const float *o = p.ws + row * D + d;
    const float *ml = p.ws + (int64_t)p.nrec * p.rows * D + row * 2;
    float M = -1e30f, l = 0.f;
    f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int s0 = wave; s0 < p.nrec; s0 += MERGE_WAVES * BATCH) {
        f32x4 x[BATCH];
        float2 w[BATCH];
#pragma unroll
        for (int s = 0; s < BATCH; ++s) {
            const int r = s0 + s * MERGE_WAVES;
            w[s] = make_float2(-1e30f, 0.f);
            x[s] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if (r < p.nrec) {
                x[s] = *(const f32x4 *)(o + r * p.rows * D);
                w[s] = *(const float2 *)(ml + r * p.rows * 2);
            }
        }
#pragma unroll
        for (int s = 0; s < BATCH; ++s)
            if (w[s].y == 0.f) x[s] = (f32x4){0.f, 0.f, 0.f, 0.f};      // no keys: what is there is no output
        float mx = M;
#pragma unroll
        for (int s = 0; s < BATCH; ++s) mx = fmaxf(mx, w[s].x);
        const float a = __builtin_amdgcn_exp2f(M - mx);
        M = mx;
        l *= a;
        acc *= a;
#pragma unroll
        for (int s = 0; s < BATCH; ++s) {
            const float b = __builtin_amdgcn_exp2f(w[s].x - M);
            l = __builtin_fmaf(b, w[s].y, l);
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = __builtin_fmaf(b, x[s][c], acc[c]);
        }
    }
    sums[wave][lane] = acc;
    mls[wave][lane] = make_float2(M, l);
    __syncthreads();
    if (wave || !on) return;
    float top = M;
#pragma unroll
    for (int s = 1; s < MERGE_WAVES; ++s) top = fmaxf(top, mls[s][lane].x);
    float a = __builtin_amdgcn_exp2f(M - top);
    l *= a;
    acc *= a;
#pragma unroll
    for (int s = 1; s < MERGE_WAVES; ++s) {
        a = __builtin_amdgcn_exp2f(mls[s][lane].x - top);
        l = __builtin_fmaf(a, mls[s][lane].y, l);
        acc += a * sums[s][lane];
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    OP::put4((unsigned char *)p.out + row * OP::ROWB, d, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}

template <class OP>
hipError_t launch_op(const SharedParams &p, int pw, int ow, hipStream_t s) {
    const dim3 grid((unsigned)(p.oct_all * 8)), block(256);
    constexpr int R = kByRows;
    if (pw == kAlone) {
        hipLaunchKernelGGL(shared_alone_kernel<OP>, dim3((unsigned)(p.n * p.n_kv_heads)), dim3(64 * ALONE_WAVES), 0, s, p);
        return hipGetLastError();
    }
    if (pw == 1) hipLaunchKernelGGL((shared_kernel<OP, 1, 1>), grid, block, 0, s, p);
    else if constexpr (OP::ELT == 2) {
        if (pw == R + 1 && ow == 1) hipLaunchKernelGGL((shared_kernel<OP, R + 1, 1>), grid, block, 0, s, p);
        else if (pw == R + 1) hipLaunchKernelGGL((shared_kernel<OP, R + 1, R + 1>), grid, block, 0, s, p);
        else if (ow == 1) hipLaunchKernelGGL((shared_kernel<OP, R + 2, 1>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((shared_kernel<OP, R + 2, R + 1>), grid, block, 0, s, p);
    } else {
        if (ow == 1) hipLaunchKernelGGL((shared_kernel<OP, 2, 1>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((shared_kernel<OP, 2, 2>), grid, block, 0, s, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int per = 64 / (OP::DIM / 4);
    hipLaunchKernelGGL(shared_merge_kernel<OP>, dim3((unsigned)((p.rows + per - 1) / per)), dim3(64 * MERGE_WAVES), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_shared(const SharedParams &p, int head_dim, int dtype, int pw, int ow, hipStream_t s) {
    if (dtype == KVR_F32) return head_dim == 128 ? launch_op<Op32<128>>(p, pw, ow, s) : launch_op<Op32<64>>(p, pw, ow, s);
    if (dtype == KVR_F16)
        return head_dim == 128 ? launch_op<Op<F16, 128>>(p, pw, ow, s) : launch_op<Op<F16, 64>>(p, pw, ow, s);
    return head_dim == 128 ? launch_op<Op<Bf16, 128>>(p, pw, ow, s) : launch_op<Op<Bf16, 64>>(p, pw, ow, s);
}

}  // namespace kvr
