// shared.hip -- attention of a batch of readers that share a long cached prefix
// and each have cached rows of their own.
//
//   out[r, i, h] = softmax over [prefix 0 .. L-1 | own rows 0 .. len_r - 1 | new rows 0 .. i]
//
// Two kinds of work in one launch, joined by a merge of log-sum-exp partials:
//   prefix  every reader sees the whole prefix, so the query rows of all readers of
//           a kv head are packed into tiles and the prefix is read once for all of
//           them (once for each row tile from the caches, once from HBM)
//   own     the rows of one reader and kv head over that reader's cached rows and,
//           causally, its new rows; the last row tile stores these to its cache
// A workgroup of four waves is one such item over a range of keys, in one of two ways:
//   by keys   up to 16 query rows (fp32: 32 a tile): every wave holds the same rows
//             and takes the range's stages in turn, K and V straight from memory
//             (attn_direct.hpp), no barrier until the four partials are joined
//   by rows   more rows, 16-bit: each wave holds 16 or 32 rows of its own and the
//             stages go through LDS once for all four (attn_ring.hpp)
// The item's partial (M, l, O) goes to the workspace.  The lengths are read on the
// device: a captured graph serves every step of a decode.
#include <type_traits>

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
    float m[RT], l[RT];      // reference (log2 domain) of the row; the lane's share of the sum
    int last[RT];            // own rows: the last new row that the lane's query row sees
};

// The scores of a stage become weights: keys with stage index >= n are masked, with
// CAUSAL also those beyond the row's own bound (c0: the stage's first new row).
template <class OP, int RT, bool CAUSAL>
__device__ __forceinline__ void softmax_step(Rows<OP, RT> &R, float (&s)[RT][OP::NS], typename OP::P (&w)[RT], int n,
                                             int c0, float c2, int g) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (CAUSAL || n < OP::KEYS) {
            const int lim = CAUSAL ? min(n - 1, R.last[rt] - c0) : n - 1;
#pragma unroll
            for (int e = 0; e < OP::NS; ++e)
                if (OP::key_of(e, g) > lim) s[rt][e] = -INFINITY;
        }
        float mx = s[rt][0];
#pragma unroll
        for (int e = 1; e < OP::NS; ++e) mx = fmaxf(mx, s[rt][e]);
        mx = quad_max(mx) * c2;
        // the reference is the running maximum: the largest weight is 2^0, which the
        // 16-bit operand holds without rounding
        if (__ballot(mx > R.m[rt])) {
            const float mn = fmaxf(R.m[rt], mx);
            const float alpha = __builtin_amdgcn_exp2f(R.m[rt] - mn);
            R.m[rt] = mn;
            R.l[rt] *= alpha;
#pragma unroll
            for (int t = 0; t < OP::NT; ++t) R.o[rt][t] *= alpha;
        }
        float p[OP::NS];
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) {
            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e], c2, -R.m[rt]));
            sum += p[e];
        }
        R.l[rt] += sum;
        OP::weights(w[rt], p);
    }
}

// O += P V of a stage of new rows.  A value that is no number must not reach the rows
// before it, whose weight for it is 0: a stage that has one goes key by key, each for
// the rows that see it.
template <class OP, int RT>
__device__ __forceinline__ void accumulate_new(Rows<OP, RT> &R, const typename OP::V &v,
                                               const typename OP::P (&w)[RT], int n, int c0, int g) {
    if (__ballot(!OP::finite(v)) == 0) {
        OP::template accumulate<RT>(v, w, R.o);
        return;
    }
    for (int c = 0; c < n; ++c) {
        bool sees[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) sees[rt] = c0 + c <= R.last[rt];
        OP::template accumulate_key<RT>(v, w, R.o, c, sees, g);
    }
}

// Stages first, first + WAVES, ... of `nkeys` consecutive cached rows at kb / vb.
// K and V have one set of registers each: the next stage's K is asked for when the
// scores are done, its V when the outputs are.
template <class OP, int RT>
__device__ __forceinline__ void cached_keys(Rows<OP, RT> &R, uint64_t kb, uint64_t vb, int64_t nkeys, int first,
                                            float c2, int i, int g) {
    constexpr int KEYS = OP::KEYS;
    const int nst = (int)((nkeys + KEYS - 1) / KEYS);
    if (first >= nst) return;
    auto left = [&](int t) {      // valid rows of stage t (0 past the last stage)
        const int64_t n = nkeys - (int64_t)t * KEYS;
        return (int)(n < 0 ? 0 : n > KEYS ? KEYS : n);
    };
    auto rows_of = [&](uint64_t base, int t) {
        return row_rsrc(base + (uint64_t)t * KEYS * OP::ROWB, left(t), OP::ROWB, OP::ROWB);
    };
    typename OP::K k;
    typename OP::V v;
    OP::load_k(k, rows_of(kb, first), OP::ROWB, i, g);
    OP::load_v(v, rows_of(vb, first), OP::ROWB, i, g);
    for (int t = first; t < nst; t += WAVES) {
        float s[RT][OP::NS];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) OP::scores(k, R.q[rt], s[rt]);
        __builtin_amdgcn_sched_barrier(0);
        OP::load_k(k, rows_of(kb, t + WAVES), OP::ROWB, i, g);
        __builtin_amdgcn_sched_barrier(0);
        typename OP::P w[RT];
        softmax_step<OP, RT, false>(R, s, w, left(t), 0, c2, g);
        OP::template accumulate<RT>(v, w, R.o);
        __builtin_amdgcn_sched_barrier(0);
        OP::load_v(v, rows_of(vb, t + WAVES), OP::ROWB, i, g);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// LDS of the join of one row tile: O of every wave, component c of the lane's four in
// row c, then (m, l)
template <class OP>
constexpr int obuf_floats() {
    return WAVES * 4 * 64 * OP::NT;
}
template <class OP>
constexpr int join_floats() {
    return obuf_floats<OP>() + 2 * WAVES * 64;
}

// The four waves' partials: every wave posts its own, then wave w joins component w
// of each row's outputs (NT consecutive head-dim indices a lane), in wave order, and
// stores it to record `rec` of the workspace.
template <class OP, int RT>
__device__ __forceinline__ void join(const SharedParams &p, Rows<OP, RT> &R, float *lds, int64_t rec,
                                     const int (&row)[RT], int wave, int lane) {
    constexpr int NT = OP::NT, D = OP::DIM;
    const int g = lane >> 4;
    float *ml = lds + obuf_floats<OP>();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (rt) __syncthreads();
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int t = 0; t < NT; t += 4)
                *(f32x4 *)(lds + ((wave * 4 + c) * 64 + lane) * NT + t) =
                    (f32x4){R.o[rt][t][c], R.o[rt][t + 1][c], R.o[rt][t + 2][c], R.o[rt][t + 3][c]};
        *(float2 *)(ml + (wave * 64 + lane) * 2) = make_float2(R.m[rt], R.l[rt]);
        __syncthreads();
        float2 w[WAVES];
        float M = -INFINITY;
#pragma unroll
        for (int s = 0; s < WAVES; ++s) {
            w[s] = *(const float2 *)(ml + (s * 64 + lane) * 2);
            M = fmaxf(M, w[s].x);
        }
        float l = 0.f;
        f32x4 acc[NT / 4];
#pragma unroll
        for (int t = 0; t < NT / 4; ++t) acc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < WAVES; ++s) {
            const float a = __builtin_amdgcn_exp2f(w[s].x - M);
            l = __builtin_fmaf(a, w[s].y, l);
#pragma unroll
            for (int t = 0; t < NT / 4; ++t) {
                const f32x4 x = *(const f32x4 *)(lds + ((s * 4 + wave) * 64 + lane) * NT + 4 * t);
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[t][c] = __builtin_fmaf(a, x[c], acc[t][c]);
            }
        }
        l = quad_sum(l);
        if (row[rt] < 0) continue;
        float *po = p.ws + (rec * p.rows + row[rt]) * D + NT * (4 * g + wave);
#pragma unroll
        for (int t = 0; t < NT / 4; ++t) *(f32x4 *)(po + 4 * t) = acc[t];
        if (wave == 0 && g == 0)
            *(float2 *)(p.ws + (int64_t)p.nrec * p.rows * D + (rec * p.rows + row[rt]) * 2) = make_float2(M, l);
    }
}

// Cached rows of reader r, or -1 if it takes no part
__device__ __forceinline__ int reader_len(const SharedParams &p, int r) {
    const int len = p.len[r];
    return len >= 0 && (int64_t)len + (p.append ? p.S : 0) <= p.tcap ? len : -1;
}

// The query rows of a tile: row r0 + 16 rt + i of `nrows` rows, which are the heads
// of kv head g for token tok0, then for the next token
template <class OP, int RT>
__device__ __forceinline__ void take_rows(const SharedParams &p, Rows<OP, RT> &R, int (&row)[RT], int head_g,
                                          int tok0, int r0, int nrows, int i, int g) {
    const int G = p.group;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + 16 * rt + i;
        const int rr = min(r, nrows - 1);         // rows past the last repeat it and are not stored
        const int tk = rr / G;
        const int tok = tok0 + tk;
        const int at = tok * p.n_q_heads + head_g * G + (rr - tk * G);
        OP::load_q(R.q[rt], (const unsigned char *)p.q + (int64_t)at * OP::ROWB, g);
        if (p.rope) {
            const int rd = tok / p.S;
            const int64_t pos = p.pos0 + max(reader_len(p, rd), 0) + (tok - rd * p.S);
            OP::rotate_q(R.q[rt], p.rope + pos * OP::DIM, g);
        }
        row[rt] = r < nrows ? at : -1;
        R.last[rt] = tk;
        R.m[rt] = -1e30f;
        R.l[rt] = 0.f;
#pragma unroll
        for (int t = 0; t < OP::NT; ++t) R.o[rt][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
}

// ---- by rows
constexpr int SLOTS = 3;      // stages in LDS: one read, one landed or landing, one asked for

// One stage from LDS.  CAUSAL: new rows, the first of which is row c0.
template <class OP, class RG, int RT, bool CAUSAL>
__device__ __forceinline__ void row_stage(Rows<OP, RT> &R, const unsigned char *ks_, const unsigned char *vs_, uint32_t ka,
                                          uint32_t va, int n, int c0, float c2, int g) {
    f32x4 a[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int h = 0; h < 2; ++h) a[rt][h] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < OP::NK; ++ks)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4 k = RG::row_frag(ks_, ka, h, ks);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) a[rt][h] = OP::mfma(k, R.q[rt].f[ks], a[rt][h]);
        }
    float s[RT][OP::NS];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) s[rt][e] = a[rt][e >> 2][e & 3];
    typename OP::P w[RT];
    softmax_step<OP, RT, CAUSAL>(R, s, w, n, c0, c2, g);
    if constexpr (CAUSAL) {
        // as accumulate_new: a value that is no number reaches the rows that see it alone
        bool ok = true;
#pragma unroll
        for (int t = 0; t < OP::NT; ++t) ok = ok && OP::finite_words(RG::col_frag(vs_, va, t));
        if (__ballot(!ok)) {
            for (int c = 0; c < n; ++c)
#pragma unroll
                for (int t = 0; t < OP::NT; ++t) {
                    const u32x4 v = OP::only_key(RG::col_frag(vs_, va, t), c, g);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const f32x4 x = OP::mfma(v, w[rt].f, R.o[rt][t]);
                        R.o[rt][t] = c0 + c <= R.last[rt] ? x : R.o[rt][t];
                    }
                }
            return;
        }
    }
#pragma unroll
    for (int t = 0; t < OP::NT; ++t) {
        const u32x4 v = RG::col_frag(vs_, va, t);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) R.o[rt][t] = OP::mfma(v, w[rt].f, R.o[rt][t]);
    }
}

// All stages of `nkeys` cached rows
template <class OP, class RG, int RT>
__device__ __forceinline__ void row_cached(Rows<OP, RT> &R, uint64_t kb, uint64_t vb, int64_t nkeys, unsigned char *lds,
                                           float c2, int wave, int lane) {
    const int i = lane & 15, g = lane >> 4;
    const uint32_t ka = RG::row_at(i, g), va = RG::col_at(i, g);
    const int nst = (int)((nkeys + RG::KEYS - 1) / RG::KEYS);
    auto count = [&](int t) { return (int)min(nkeys - (int64_t)t * RG::KEYS, (int64_t)RG::KEYS); };
    auto load = [&](int t, int slot) {
        const uint64_t off = (uint64_t)t * RG::KEYS * OP::ROWB;
        unsigned char *to = lds + slot * 2 * RG::HALF;
        RG::load(kb + off, OP::ROWB, count(t), to, wave, lane);
        RG::load(vb + off, OP::ROWB, count(t), to + RG::HALF, wave, lane);
    };
    if (nst > 0) load(0, 0);
    if (nst > 1) load(1, 1);
    int slot = 0;
    for (int t = 0; t < nst; ++t) {
        // this wave's part of stage t has landed (stage t + 1 may be on its way); behind the
        // barrier everybody's has, and nobody reads the slot of stage t - 1 any more
        if (t + 1 < nst) wait_vmcnt<2 * RG::LOADS>();
        else wait_vmcnt<0>();
        barrier_lds();
        if (t + 2 < nst) load(t + 2, slot == 0 ? 2 : slot - 1);
        const unsigned char *st = lds + slot * 2 * RG::HALF;
        row_stage<OP, RG, RT, false>(R, st, st + RG::HALF, ka, va, count(t), 0, c2, g);
        slot = slot == SLOTS - 1 ? 0 : slot + 1;
    }
    barrier_lds();
}

// The partial of the wave's own rows
template <class OP, int RT>
__device__ __forceinline__ void put_rows(const SharedParams &p, Rows<OP, RT> &R, int64_t rec, const int (&row)[RT], int g) {
    constexpr int D = OP::DIM;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float l = quad_sum(R.l[rt]);
        if (row[rt] < 0) continue;
        float *po = p.ws + (rec * p.rows + row[rt]) * D + 4 * g;
#pragma unroll
        for (int t = 0; t < OP::NT; ++t) *(f32x4 *)(po + 16 * t) = R.o[rt][t];
        if (g == 0) *(float2 *)(p.ws + (int64_t)p.nrec * p.rows * D + (rec * p.rows + row[rt]) * 2) = make_float2(R.m[rt], l);
    }
}

// ---- items
// WAY: 1 or 2: by keys, that many 16-row tiles; kByRows + 1 or 2: by rows, that many in
// each wave
constexpr int kTiles(int way) { return way > kByRows ? way - kByRows : way; }
constexpr int kRowsOf(int way) { return way > kByRows ? 64 * (way - kByRows) : 16 * way; }

template <class OP, int WAY>
constexpr int lds_bytes() {
    return WAY > kByRows ? SLOTS * 64 * OP::ROWB : join_floats<OP>() * 4;
}

// Prefix item (oct, in8): the (kv head, split) pairs in groups of eight, a group's row
// tiles one after the other.  Blocks eight apart share an XCD, so the tiles that read
// one range of prefix rows find it in one L2.
template <class OP, int WAY>
__device__ __forceinline__ void prefix_item(const SharedParams &p, uint32_t oct, uint32_t in8, unsigned char *lds) {
    constexpr int RT = kTiles(WAY);
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t pair = oct / p.p_tiles * 8 + in8;
    const int tile = (int)(oct % p.p_tiles);
    const int split = (int)(pair / p.n_kv_heads), hd = (int)(pair % p.n_kv_heads);
    if (split >= p.np) return;
    const int64_t kb = split * p.chunk, ke = min(kb + p.chunk, p.L);
    const uint64_t off = ((uint64_t)hd * p.cap + kb) * OP::ROWB;
    const uint64_t k0 = (uint64_t)(uintptr_t)p.kc + off, v0 = (uint64_t)(uintptr_t)p.vc + off;
    Rows<OP, RT> R;
    int row[RT];
    if constexpr (WAY > kByRows) {
        take_rows(p, R, row, hd, 0, tile * kRowsOf(WAY) + wave * 16 * RT, p.n * p.S * p.group, i, g);
        row_cached<OP, typename OP::Ring, RT>(R, k0, v0, ke - kb, lds, p.scale_log2, wave, lane);
        put_rows<OP, RT>(p, R, split, row, g);
    } else {
        take_rows(p, R, row, hd, 0, tile * 16 * RT, p.n * p.S * p.group, i, g);
        cached_keys<OP, RT>(R, k0, v0, ke - kb, wave, p.scale_log2, i, g);
        join<OP, RT>(p, R, (float *)lds, split, row, wave, lane);
    }
}

// Own item b: (split, reader, row tile, kv head), kv head fastest.  The splits have equal
// shares of the cached rows, in whole stages of four waves; the last has the new rows too.
template <class OP, int WAY>
__device__ __forceinline__ void own_item(const SharedParams &p, uint32_t b, unsigned char *lds) {
    constexpr int RT = kTiles(WAY), KEYS = OP::KEYS;
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hd = (int)(b % p.n_kv_heads);
    b /= p.n_kv_heads;
    const int tile = (int)(b % p.t_tiles);
    b /= p.t_tiles;
    const int rd = (int)(b % p.n), split = (int)(b / p.n);
    if (split >= p.nt) return;
    const int len = reader_len(p, rd);
    if (len < 0) return;
    const int r0 = tile * kRowsOf(WAY), nrows = p.S * p.group;
    const int share = (len + p.nt - 1) / p.nt;
    const int chunk = (share + KEYS - 1) / KEYS * KEYS;
    const int64_t kb = (int64_t)split * chunk;
    const int64_t nk = max((int64_t)0, min((int64_t)chunk, len - kb));
    const uint64_t head = (uint64_t)rd * p.n_kv_heads + hd;
    const uint64_t off = (head * p.tcap + kb) * OP::ROWB;
    const uint64_t k0 = (uint64_t)(uintptr_t)p.kt + off, v0 = (uint64_t)(uintptr_t)p.vt + off;
    // new rows that a row of this tile sees; the last tile sees all and stores them
    const int seen = split == p.nt - 1 ? min(p.S, (min(r0 + kRowsOf(WAY), nrows) - 1) / p.group + 1) : 0;
    const bool store = p.append && tile == p.t_tiles - 1;
    const uint32_t nb = (uint32_t)p.n_kv_heads * OP::ROWB;
    const uint64_t src = ((uint64_t)rd * p.S * p.n_kv_heads + hd) * OP::ROWB;
    const uint64_t kn = (uint64_t)(uintptr_t)p.kn + src, vn = (uint64_t)(uintptr_t)p.vn + src;
    const uint64_t to = (head * p.tcap + len) * OP::ROWB;
    unsigned char *kd = (unsigned char *)p.kt + to, *vd = (unsigned char *)p.vt + to;
    Rows<OP, RT> R;
    int row[RT];
    if constexpr (WAY > kByRows) {
        using RG = typename OP::Ring;
        take_rows(p, R, row, hd, rd * p.S, r0 + wave * 16 * RT, nrows, i, g);
        row_cached<OP, RG, RT>(R, k0, v0, nk, lds, p.scale_log2, wave, lane);
        for (int c0 = 0; c0 < seen; c0 += KEYS) {
            // the stage's rows through registers: a thread has chunk c of a row and the one
            // half a row further, whose dims are each other's partners in the rotation
            constexpr int PAIRS = RG::CH / 2;
            const int n = min(seen - c0, KEYS);
            const int r = threadIdx.x / PAIRS, c = threadIdx.x % PAIRS;
            if (r < KEYS) {
                u32x4 k[2], v[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) k[h] = v[h] = (u32x4){0u, 0u, 0u, 0u};
                if (r < n) {
                    const uint64_t at = (uint64_t)(c0 + r) * nb + 16 * c;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        k[h] = *(const u32x4 *)(uintptr_t)(kn + at + 16 * PAIRS * h);
                        v[h] = *(const u32x4 *)(uintptr_t)(vn + at + 16 * PAIRS * h);
                    }
                    if (p.rope) OP::rotate8(k[0], k[1], p.rope + (p.pos0 + len + c0 + r) * OP::DIM + 16 * c);
                    if (store) {
                        const uint64_t d = (uint64_t)(c0 + r) * OP::ROWB + 16 * c;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            *(u32x4 *)(kd + d + 16 * PAIRS * h) = k[h];
                            *(u32x4 *)(vd + d + 16 * PAIRS * h) = v[h];
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    unsigned char *l = lds + r * OP::ROWB + 16 * ((c + PAIRS * h) ^ RG::swz(r));
                    *(u32x4 *)l = k[h];
                    *(u32x4 *)(l + RG::HALF) = v[h];
                }
            }
            barrier_lds();
            row_stage<OP, RG, RT, true>(R, lds, lds + RG::HALF, RG::row_at(i, g), RG::col_at(i, g), n, c0, p.scale_log2, g);
            barrier_lds();
        }
        put_rows<OP, RT>(p, R, p.np + split, row, g);
    } else {
        take_rows(p, R, row, hd, rd * p.S, r0, nrows, i, g);
        // (16-bit: 16 query rows are 16 tokens at most, one part of a stage.)  Stage c of the
        // new rows goes to the wave whose turn follows the cached stages
        const int nst = (int)((nk + KEYS - 1) / KEYS);
        for (int c = (wave - nst) & (WAVES - 1); c * KEYS < seen; c += WAVES) {
            const int c0 = c * KEYS, n = min(seen - c0, KEYS);
            typename OP::K k;
            typename OP::V v;
            const uint64_t at = (uint64_t)c0 * nb;
            OP::template load_k<1>(k, row_rsrc(kn + at, n, nb, OP::ROWB), nb, i, g);
            OP::template load_v<1>(v, row_rsrc(vn + at, n, nb, OP::ROWB), nb, i, g);
            if (p.rope) OP::template rotate_k<1>(k, p.rope + (p.pos0 + len + c0) * OP::DIM, n, i, g);
            if (store) OP::template store<1>(k, v, kd + (uint64_t)c0 * OP::ROWB, vd + (uint64_t)c0 * OP::ROWB, n, i, g);
            float sc[RT][OP::NS];
            typename OP::P w[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) OP::scores(k, R.q[rt], sc[rt]);
            softmax_step<OP, RT, true>(R, sc, w, n, c0, p.scale_log2, g);
            accumulate_new<OP, RT>(R, v, w, n, c0, g);
        }
        cached_keys<OP, RT>(R, k0, v0, nk, wave, p.scale_log2, i, g);
        join<OP, RT>(p, R, (float *)lds, p.np + split, row, wave, lane);
    }
}

// PW, OW: the ways of prefix and own items
template <class OP, int PW, int OW>
__global__ __launch_bounds__(256, OP::ELT == 2 ? 3 : OW == 1 ? 2 : 1) void shared_kernel(const SharedParams p) {
    constexpr int LP = lds_bytes<OP, PW>(), LO = lds_bytes<OP, OW>();
    __shared__ __attribute__((aligned(1024))) unsigned char lds[LP > LO ? LP : LO];
    // blocks in groups of eight (one for each XCD), the own items' groups spread evenly
    // among the prefix items': the first are bound by memory, the second by the
    // matrix and vector units
    const uint32_t oct = blockIdx.x / 8, in8 = blockIdx.x % 8;
    const uint32_t before = (uint32_t)(oct * p.own_share >> 32), upto = (uint32_t)((oct + 1) * p.own_share >> 32);
    if (upto > before) own_item<OP, OW>(p, before * 8 + in8, lds);
    else prefix_item<OP, PW>(p, oct - upto, in8, lds);
}

// out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over the records of a row, in
// record order.  D / 4 lanes a row, four values a lane.
template <class OP>
__global__ __launch_bounds__(64) void shared_merge_kernel(const SharedParams p) {
    constexpr int D = OP::DIM, LANES = D / 4, BATCH = 8;
    const int64_t row = (int64_t)blockIdx.x * (64 / LANES) + threadIdx.x / LANES;
    const int d = threadIdx.x % LANES * 4;
    if (row >= p.rows) return;
    if (reader_len(p, (int)(row / ((int64_t)p.n_q_heads * p.S))) < 0) return;
    const float *o = p.ws + row * D + d;
    const float *ml = p.ws + (int64_t)p.nrec * p.rows * D + row * 2;
    float M = -1e30f, l = 0.f;
    f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < p.nrec; s0 += BATCH) {
        f32x4 x[BATCH];
        float2 w[BATCH];
#pragma unroll
        for (int s = 0; s < BATCH; ++s) {
            const int64_t at = (int64_t)min(s0 + s, p.nrec - 1) * p.rows;
            x[s] = *(const f32x4 *)(o + at * D);
            w[s] = *(const float2 *)(ml + at * 2);
        }
        float mx = M;
#pragma unroll
        for (int s = 0; s < BATCH; ++s) mx = fmaxf(mx, w[s].x);
        const float a = __builtin_amdgcn_exp2f(M - mx);
        M = mx;
        l *= a;
        acc *= a;
#pragma unroll
        for (int s = 0; s < BATCH; ++s) {
            const float b = s0 + s < p.nrec ? __builtin_amdgcn_exp2f(w[s].x - M) : 0.f;
            l = __builtin_fmaf(b, w[s].y, l);
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = __builtin_fmaf(b, x[s][c], acc[c]);
        }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    OP::put4((unsigned char *)p.out + row * OP::ROWB, d, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}

template <class OP>
hipError_t launch_op(const SharedParams &p, int pw, int ow, hipStream_t s) {
    const dim3 grid((unsigned)(p.oct_all * 8)), block(256);
    constexpr int R = kByRows;
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
    hipLaunchKernelGGL(shared_merge_kernel<OP>, dim3((unsigned)((p.rows + per - 1) / per)), dim3(64), 0, s, p);
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
