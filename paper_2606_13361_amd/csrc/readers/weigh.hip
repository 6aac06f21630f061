// weigh.hip -- the attention weight that each cached row receives, summed over the
// query rows and heads of its kv head:
//
//   weight[g][j] += sum_(i, h of g) 2^(c q_ih . k_j - M_ih) / l_ih,   c = scale log2(e)
//
// A row's normalizer (M, l) covers all its keys, so there are two passes over the
// keys, both matrix products of K and Q^T:
//   stats  a wave holds 16 RT query rows and walks keys; each lane keeps the running
//          reference and sum of its own keys, joined at the end.  Up to 16 rows of a kv
//          head (and fp32): the four waves hold the same rows and split the keys, K
//          straight from memory (attn_direct.hpp).  More: each wave has rows of its own
//          and the four share the keys' stages in LDS (attn_ring.hpp).
//   sums   a wave holds HELD stages of keys and walks all query rows of its kv head,
//          which the four waves share in LDS (fp32: straight from memory); the weights
//          of its keys add up in registers and are added to the buffer once
// Every sum has a fixed order and every buffer element one writer: results are
// reproducible bit for bit.
//
// Measured, in us (32 query heads, 8 kv heads, head_dim 128, one MI355X):
//   128 tokens over 32640 keys   stats 38.8, norms 4.7, sums 46.9   34.2 GFLOP a pass: 0.88 and 0.73 PFLOP/s
//   24 tokens over 16384 keys    11.0 + 3.9 + 11.7                  33 MB of keys a pass
//   1 token over 3774 keys       4.0 + 4.6                          latency
// (Medians of passes that follow each other; the first ones after a pause are 10 % slower.)
// Long calls are bound by what a wave issues: for 16 rows and 32 keys 8 products of 16 clocks of a
// SIMD, and beside them, by the counters, 33 vector instructions in the first pass and 45 in the
// second: 8 exponentials of 16 clocks, 8 fused multiplications and 8 additions of 4, which are
// the work, and masks, checks of the sums and, in the second pass, the addresses of the query
// rows.  That is 128 clocks of products and 228 and 276 of the rest; a unit takes about 290 and
// 350 at 1.9 GHz, more than the larger of the two: the SIMD's two and three waves overlap
// them in part.
// Scores of the next stage made among the exponentials, as in shared.hip, changed nothing (45
// and 53 us for 43 and 52).  The second pass holds one stage of keys a wave; two, for half the
// reads of the query rows, took 60 us instead of 55.
#include <type_traits>

#include "attn_ring.hpp"
#include "readers_internal.hpp"

namespace kvr {
namespace {

using namespace dev;

constexpr int WAVES = 4;

// K rows of stage t of a kv head's key sequence: its prefix stages, then the new rows'
template <class OP>
struct Keys {
    uint64_t kc, kn;
    int64_t L;
    uint32_t new_b;
    int S, n_pre;      // n_pre: prefix stages
    __device__ __forceinline__ Keys(const WeighParams &p, int hd) {
        kc = (uint64_t)(uintptr_t)p.kc + (uint64_t)hd * p.cap * OP::ROWB;
        kn = (uint64_t)(uintptr_t)p.kn + (uint64_t)hd * OP::ROWB;
        L = p.L;
        S = p.S;
        new_b = (uint32_t)p.n_kv_heads * OP::ROWB;
        n_pre = (int)((p.L + OP::KEYS - 1) / OP::KEYS);
    }
    __device__ __forceinline__ bool is_new(int t) const { return t >= n_pre; }
    // first row of the stage within its part, and its valid rows
    __device__ __forceinline__ int64_t first(int t) const { return (int64_t)(is_new(t) ? t - n_pre : t) * OP::KEYS; }
    __device__ __forceinline__ int count(int t) const {
        const int64_t n = (is_new(t) ? (int64_t)S : L) - first(t);
        return (int)(n < 0 ? 0 : n > OP::KEYS ? OP::KEYS : n);
    }
    __device__ __forceinline__ void load(typename OP::K &k, int t, int n, int i, int g) const {
        if (is_new(t)) OP::load_k(k, row_rsrc(kn + (uint64_t)first(t) * new_b, n, new_b, OP::ROWB), new_b, i, g);
        else OP::load_k(k, row_rsrc(kc + (uint64_t)first(t) * OP::ROWB, n, OP::ROWB, OP::ROWB), OP::ROWB, i, g);
    }
};

// Scores of keys beyond stage index `lim` leave the softmax
template <class OP>
__device__ __forceinline__ void mask(float (&s)[OP::NS], int lim, int g) {
#pragma unroll
    for (int e = 0; e < OP::NS; ++e)
        if (OP::key_of(e, g) > lim) s[e] = -INFINITY;
}

constexpr float kMost = 56.f, kSlack = 0x1p60f;

// A stage's scores of RT row tiles into the lane's running references and sums.  A
// reference need not be the maximum, only near enough: it moves there when a sum of
// terms 2^(c2 s - m) grows too large (or is no number), and nothing is rounded
// differently for it.  2^31 stages of up to kSlack (16 terms of 2^kMost) stay below the
// type's largest value.
template <class OP, int RT>
__device__ __forceinline__ void add_scores(const float (&s)[RT][OP::NS], float c2, float (&m)[RT], float (&l)[RT]) {
    float sum[RT];
    auto sums = [&]() {
        bool over = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float p[OP::NS];
#pragma unroll
            for (int e = 0; e < OP::NS; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e], c2, -m[rt]));
            sum[rt] = 0.f;
#pragma unroll
            for (int e = 0; e < OP::NS; ++e) sum[rt] += p[e];
            over |= !(sum[rt] <= kSlack);
        }
        return over;
    };
    if (__ballot(sums())) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float mx = s[rt][0];
#pragma unroll
            for (int e = 1; e < OP::NS; ++e) mx = fmaxf(mx, s[rt][e]);
            const float mn = mx * c2 > m[rt] + kMost ? mx * c2 : m[rt];      // each row for itself
            l[rt] *= __builtin_amdgcn_exp2f(m[rt] - mn);
            m[rt] = mn;
        }
        sums();
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) l[rt] += sum[rt];
}

// block: (row tile, split, kv head), kv head fastest.  A split's key range is p.chunk
// stages; the last one ends with the new rows.
template <class OP, int RT>
__global__ __launch_bounds__(256) void weigh_stats_kernel(const WeighParams p) {
    __shared__ float2 part[WAVES][RT][64];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t b = blockIdx.x;
    const int hd = b % p.n_kv_heads;
    b /= p.n_kv_heads;
    const int split = b % p.nsplit, tile = b / p.nsplit;
    const int G = p.group, rows = p.S * G;
    typename OP::Q q[RT];
    float m[RT], l[RT];
    int tok[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = min((tile * RT + rt) * 16 + i, rows - 1);
        tok[rt] = r / G;
        OP::load_q(q[rt], (const unsigned char *)p.q + ((int64_t)tok[rt] * p.n_q_heads + hd * G + (r - tok[rt] * G)) * OP::ROWB, g);
        m[rt] = -1e30f;
        l[rt] = 0.f;
    }
    const Keys<OP> keys(p, hd);
    const int last_tok = (min((tile + 1) * RT * 16, rows) - 1) / G;      // beyond it no new row is seen
    const int n_all = keys.n_pre + last_tok / OP::KEYS + 1;
    const int t0 = split * p.chunk;
    const int t1 = split == p.nsplit - 1 ? n_all : min(t0 + p.chunk, n_all);
    const float c2 = p.scale_log2;
    typename OP::K k[2];
    auto step = [&](const typename OP::K &kk, int t) {
        const int n = keys.count(t);
        float s[RT][OP::NS];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) OP::scores(kk, q[rt], s[rt]);
        if (keys.is_new(t) || n < OP::KEYS) {
            const int c0 = (int)keys.first(t);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) mask<OP>(s[rt], keys.is_new(t) ? min(n - 1, tok[rt] - c0) : n - 1, g);
        }
        add_scores<OP, RT>(s, c2, m, l);
    };
    int t = t0 + wave;
    if (t < t1) keys.load(k[0], t, keys.count(t), i, g);
    while (t < t1) {
        keys.load(k[1], t + WAVES, t + WAVES < t1 ? keys.count(t + WAVES) : 0, i, g);
        __builtin_amdgcn_sched_barrier(0);
        step(k[0], t);
        t += WAVES;
        if (t >= t1) break;
        keys.load(k[0], t + WAVES, t + WAVES < t1 ? keys.count(t + WAVES) : 0, i, g);
        __builtin_amdgcn_sched_barrier(0);
        step(k[1], t);
        t += WAVES;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) part[wave][rt][lane] = make_float2(m[rt], l[rt]);
    __syncthreads();
    // row r of the tile: 16 partials, in wave and lane order
    for (int r = threadIdx.x; r < RT * 16; r += 256) {
        const int row = tile * RT * 16 + r;
        if (row >= rows) break;
        float M = -1e30f, sum = 0.f;
#pragma unroll
        for (int x = 0; x < 4 * WAVES; ++x) M = fmaxf(M, part[x >> 2][r >> 4][(x & 3) * 16 + (r & 15)].x);
#pragma unroll
        for (int x = 0; x < 4 * WAVES; ++x) {
            const float2 v = part[x >> 2][r >> 4][(x & 3) * 16 + (r & 15)];
            sum = __builtin_fmaf(__builtin_amdgcn_exp2f(v.x - M), v.y, sum);
        }
        p.ws[((int64_t)hd * p.nsplit + split) * rows + row] = make_float2(M, sum);
    }
}

// The same with rows of its own for every wave (64 RT a workgroup) and the stages' K
// rows shared in LDS
template <class OP, class RG, int RT>
__global__ __launch_bounds__(256) void weigh_stats_rows_kernel(const WeighParams p) {
    constexpr int SLOTS = 3;      // one is read while the others are on their way
    __shared__ __attribute__((aligned(1024))) unsigned char lds[SLOTS * RG::HALF];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t b = blockIdx.x;
    const int hd = b % p.n_kv_heads;
    b /= p.n_kv_heads;
    const int split = b % p.nsplit, tile = b / p.nsplit;
    const int G = p.group, rows = p.S * G;
    typename OP::Q q[RT];
    float m[RT], l[RT];
    int tok[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = min(((tile * WAVES + wave) * RT + rt) * 16 + i, rows - 1);
        tok[rt] = r / G;
        OP::load_q(q[rt], (const unsigned char *)p.q + ((int64_t)tok[rt] * p.n_q_heads + hd * G + (r - tok[rt] * G)) * OP::ROWB, g);
        m[rt] = -1e30f;
        l[rt] = 0.f;
    }
    const Keys<OP> keys(p, hd);
    const int last_tok = (min((tile + 1) * WAVES * RT * 16, rows) - 1) / G;      // beyond it no new row is seen
    const int n_all = keys.n_pre + last_tok / OP::KEYS + 1;
    const int t0 = split * p.chunk;
    const int t1 = split == p.nsplit - 1 ? n_all : min(t0 + p.chunk, n_all);
    const uint32_t ka = RG::row_at(i, g);
    const float c2 = p.scale_log2;
    auto load = [&](int t, int slot) {
        const uint64_t first = (uint64_t)keys.first(t);
        if (keys.is_new(t)) RG::template load<false>(keys.kn + first * keys.new_b, keys.new_b, keys.count(t), lds + slot * RG::HALF, wave, lane);
        else RG::template load<false>(keys.kc + first * OP::ROWB, OP::ROWB, keys.count(t), lds + slot * RG::HALF, wave, lane);
    };
    for (int x = 0; x < SLOTS - 1 && t0 + x < t1; ++x) load(t0 + x, x);
    wait_vmcnt<0>();      // the query rows too: loads that the compiler knows of would be waited for in the loop
    int slot = 0;
    for (int t = t0; t < t1; ++t) {
        if (t + SLOTS - 2 < t1) wait_vmcnt<(SLOTS - 2) * RG::LOADS>();
        else wait_vmcnt<0>();
        barrier_lds();      // the stage has landed, the slot of the one before is free
        if (t + SLOTS - 1 < t1) load(t + SLOTS - 1, slot == 0 ? SLOTS - 1 : slot - 1);
        const unsigned char *st = lds + slot * RG::HALF;
        typename OP::K k;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ks = 0; ks < OP::NK; ++ks) k.f[h][ks] = RG::row_frag(st, ka, h, ks);
        float s[RT][OP::NS];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) OP::scores(k, q[rt], s[rt]);
        const int n = keys.count(t);
        if (keys.is_new(t) || n < OP::KEYS) {
            const int c0 = (int)keys.first(t);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) mask<OP>(s[rt], keys.is_new(t) ? min(n - 1, tok[rt] - c0) : n - 1, g);
        }
        add_scores<OP, RT>(s, c2, m, l);
        slot = slot == SLOTS - 1 ? 0 : slot + 1;
    }
    // the four lanes of a row
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float M = quad_max(m[rt]);
        const float sum = quad_sum(l[rt] * __builtin_amdgcn_exp2f(m[rt] - M));
        const int row = ((tile * WAVES + wave) * RT + rt) * 16 + i;
        if (g == 0 && row < rows) p.ws[((int64_t)hd * p.nsplit + split) * rows + row] = make_float2(M, sum);
    }
}

constexpr int ROWS_AT_ONCE = 1024;      // normalizers held in LDS

// M + log2(l) of a row, joined from its splits by eight lanes (lane j8 of them): a weight
// is one 2^x.  Rounding that exponent is an error of the size that the score has already.
__device__ __forceinline__ float join_norm(const float2 *src, int nsplit, int rows, int j8) {
    constexpr int AT_ONCE = 4;
    float M = -1e30f, sum = 0.f;
    for (int s0 = j8; s0 < nsplit; s0 += 8 * AT_ONCE) {
        float2 v[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            v[u] = src[(int64_t)min(s0 + 8 * u, nsplit - 1) * rows];
            if (s0 + 8 * u >= nsplit) v[u] = make_float2(-1e30f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const float mn = fmaxf(M, v[u].x);
            sum = sum * __builtin_amdgcn_exp2f(M - mn) + v[u].y * __builtin_amdgcn_exp2f(v[u].x - mn);
            M = mn;
        }
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        const float M2 = __shfl_xor(M, d), sum2 = __shfl_xor(sum, d), mn = fmaxf(M, M2);
        sum = sum * __builtin_amdgcn_exp2f(M - mn) + sum2 * __builtin_amdgcn_exp2f(M2 - mn);
        M = mn;
    }
    return M + __builtin_amdgcn_logf(sum);
}

// All rows' norms, for the second pass's workgroups to read instead of joining them each.
// 24 rows over 16384 keys, 43 splits: the second pass takes 23 us when it joins them, 13.6
// and 3.9 here.
__global__ __launch_bounds__(256) void weigh_norm_kernel(const WeighParams p) {
    const int64_t rows = (int64_t)p.S * p.group, x = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3;
    const int64_t at = min(x, rows * p.n_kv_heads - 1), hd = at / rows, r = at - hd * rows;
    const float nm = join_norm(p.ws + hd * p.nsplit * rows + r, p.nsplit, (int)rows, threadIdx.x & 7);
    if ((threadIdx.x & 7) == 0 && x == at) p.norm[x] = nm;
}

// norm[r] of rows r0 .. r0 + nr - 1 of a kv head into LDS.  Rows up to `padded` get weight 0.
__device__ __forceinline__ void take_norms(const WeighParams &p, float *norm, int hd, int rows, int r0, int nr, int padded) {
    if (p.norm) {
        for (int r = threadIdx.x; r < padded; r += 256)
            norm[r] = r < nr ? p.norm[(int64_t)hd * rows + r0 + r] : INFINITY;
        return;
    }
    for (int x = threadIdx.x; x < padded * 8; x += 256) {
        const int r = x >> 3;
        const float nm = join_norm(p.ws + (int64_t)hd * p.nsplit * rows + r0 + min(r, nr - 1), p.nsplit, rows, x & 7);
        if ((x & 7) == 0) norm[r] = r < nr ? nm : INFINITY;
    }
}

// The lane's place in the buffer for stage t of its wave's keys (t >= n_all: there is none):
// lane (i, g) has that of score i, after the sum over the sixteen lanes of a g; null for
// lanes beyond, and keys past the last
template <class OP>
__device__ __forceinline__ float *place_of(const WeighParams &p, const Keys<OP> &keys, int hd, int t, int n_all, int i, int g) {
    const int n = t < n_all ? keys.count(t) : 0, key = OP::key_of(i & (OP::NS - 1), g);
    if (i >= OP::NS || key >= n) return nullptr;
    return p.weight + (int64_t)hd * p.cap + (keys.is_new(t) ? p.L : 0) + keys.first(t) + key;
}

// The weights of a stage's keys, of each lane's rows, summed over the lanes of a key's 16
// rows and added to what the buffer held
template <class OP>
__device__ __forceinline__ void add_to(float *place, float held, const float (&acc)[OP::NS], int i) {
    float mine = 0.f;
#pragma unroll
    for (int e = 0; e < OP::NS; ++e) {
        float x = acc[e];
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) x += __shfl_xor(x, d);
        mine = i == e ? x : mine;
    }
    if (place) *place = held + mine;
}

// block: (group of WAVES stages, kv head), kv head fastest.  The query rows go through LDS
// in stages of 32.
template <class OP, class RG>
__global__ __launch_bounds__(256) void weigh_sum_rows_kernel(const WeighParams p) {
    constexpr int SLOTS = 3, ROWS = 32;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[SLOTS * RG::HALF];
    __shared__ float norm[ROWS_AT_ONCE];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hd = blockIdx.x % p.n_kv_heads;
    const int G = p.group, rows = p.S * G;
    const Keys<OP> keys(p, hd);
    const int n_all = keys.n_pre + (p.S + OP::KEYS - 1) / OP::KEYS;
    const int t = (int)(blockIdx.x / p.n_kv_heads) * WAVES + wave;
    const float c2 = p.scale_log2;
    const uint32_t qa = RG::row_at(i, g);
    const uint64_t q0 = (uint64_t)(uintptr_t)p.q + (uint64_t)hd * G * OP::ROWB;
    typename OP::K k;
    float acc[OP::NS];
    keys.load(k, t, t < n_all ? keys.count(t) : 0, i, g);
    float *const place = place_of(p, keys, hd, t, n_all, i, g);
    const float held = place ? *place : 0.f;      // (asked for here: not a round trip of its own at the end)
#pragma unroll
    for (int e = 0; e < OP::NS; ++e) acc[e] = 0.f;
    // This wave's quarter of each stage, rows of the kv head one after the other (past the
    // last: it again): from one stage to the next a row's head goes on by 32 mod G, its
    // token by 32 / G, and one more where the head passes the group's last.
    uint64_t src[RG::LOADS], last[RG::LOADS];
    int head[RG::LOADS];
    const int more = ROWS % G;
    const uint64_t step = ((uint64_t)(ROWS / G) * p.n_q_heads + more) * OP::ROWB;
    const uint64_t wrap = (uint64_t)(p.n_q_heads - G) * OP::ROWB;
#pragma unroll
    for (int x = 0; x < RG::LOADS; ++x) {
        const int row = (wave * RG::LOADS + x) * 1024 / OP::ROWB + lane / RG::CH;
        const uint64_t chunk = q0 + 16u * (uint32_t)((lane & (RG::CH - 1)) ^ RG::template swz<false>(row));
        head[x] = row % G;
        src[x] = chunk + ((uint64_t)(row / G) * p.n_q_heads + head[x]) * OP::ROWB;
        last[x] = chunk + ((uint64_t)(p.S - 1) * p.n_q_heads + G - 1) * OP::ROWB;
    }
    auto load = [&](int slot) {
#pragma unroll
        for (int x = 0; x < RG::LOADS; ++x) {
            dma16((const void *)(uintptr_t)min(src[x], last[x]), lds + slot * RG::HALF + (wave * RG::LOADS + x) * 1024);
            head[x] += more;
            src[x] += step + (head[x] >= G ? wrap : 0);
            head[x] -= head[x] >= G ? G : 0;
        }
    };
    // 32 query rows from LDS against the wave's keys; NEW: these are new rows
    auto stage = [&](auto is_new, const unsigned char *st, int r0, int rr) {
        constexpr bool NEW = decltype(is_new)::value;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            typename OP::Q q;
#pragma unroll
            for (int ks = 0; ks < OP::NK; ++ks) q.f[ks] = RG::row_frag(st, qa, part, ks);
            const float nm = norm[rr + 16 * part + i];
            float s[OP::NS];
            OP::scores(k, q, s);
            if constexpr (NEW) mask<OP>(s, (r0 + rr + 16 * part + i) / G - (int)keys.first(t), g);
#pragma unroll
            for (int e = 0; e < OP::NS; ++e) acc[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c2, -nm));
        }
    };
    for (int r0 = 0; r0 < rows; r0 += ROWS_AT_ONCE) {
        const int nr = min(rows - r0, ROWS_AT_ONCE), padded = (nr + ROWS - 1) / ROWS * ROWS;
        if (r0) barrier_lds();
        load(0);
        if (ROWS < padded) load(1);
        take_norms(p, norm, hd, rows, r0, nr, padded);
        wait_vmcnt<0>();      // the keys too: loads that the compiler knows of would be waited for in the loop
        auto walk = [&](auto is_new) {
            int slot = 0;
            for (int rr = 0; rr < padded; rr += ROWS) {
                if (rr + ROWS < padded) wait_vmcnt<RG::LOADS>();
                else wait_vmcnt<0>();
                barrier_lds();
                if (rr + 2 * ROWS < padded) load(slot == 0 ? 2 : slot - 1);
                stage(is_new, lds + slot * RG::HALF, r0, rr);
                slot = slot == SLOTS - 1 ? 0 : slot + 1;
            }
        };
        if (keys.is_new(t)) walk(std::true_type{});
        else walk(std::false_type{});
    }
    add_to<OP>(place, held, acc, i);
}

// The same with the query rows straight from memory
template <class OP, int HELD>
__global__ __launch_bounds__(256) void weigh_sum_kernel(const WeighParams p) {
    __shared__ float norm[ROWS_AT_ONCE];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hd = blockIdx.x % p.n_kv_heads;
    const int G = p.group, rows = p.S * G;
    const Keys<OP> keys(p, hd);
    const int n_all = keys.n_pre + (p.S + OP::KEYS - 1) / OP::KEYS;
    const int t0 = ((int)(blockIdx.x / p.n_kv_heads) * WAVES + wave) * HELD;
    const float c2 = p.scale_log2;
    typename OP::K k[HELD];
    float acc[HELD][OP::NS], *place[HELD], held[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        keys.load(k[h], t0 + h, t0 + h < n_all ? keys.count(t0 + h) : 0, i, g);
        place[h] = place_of(p, keys, hd, t0 + h, n_all, i, g);
        held[h] = place[h] ? *place[h] : 0.f;
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) acc[h][e] = 0.f;
    }
    // row r0 + i of the kv head is head `rem` of token `tok`; 16 rows on: (t16, r16) further
    const int t16 = 16 / G, r16 = 16 - t16 * G;
    for (int r0 = 0; r0 < rows; r0 += ROWS_AT_ONCE) {
        const int nr = min(rows - r0, ROWS_AT_ONCE), padded = (nr + 15) & ~15;
        if (r0) __syncthreads();
        take_norms(p, norm, hd, rows, r0, nr, padded);
        int tok = (r0 + i) / G, rem = (r0 + i) - tok * G;
        typename OP::Q q, next;
        auto load = [&](typename OP::Q &to) {      // (rows past the last: any row)
            const int t = min(tok, p.S - 1);
            OP::load_q(to, (const unsigned char *)p.q + ((int64_t)t * p.n_q_heads + hd * G + rem) * OP::ROWB, g);
        };
        load(q);
        __syncthreads();
        for (int rr = 0; rr < padded; rr += 16) {
            const int at = tok;
            tok += t16;
            rem += r16;
            if (rem >= G) {
                rem -= G;
                ++tok;
            }
            load(next);
            const float nm = norm[rr + i];
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                float s[OP::NS];
                OP::scores(k[h], q, s);
                const int t = t0 + h;
                if (keys.is_new(t)) mask<OP>(s, at - (int)keys.first(t), g);
#pragma unroll
                for (int e = 0; e < OP::NS; ++e) acc[h][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c2, -nm));
            }
            q = next;
        }
    }
#pragma unroll
    for (int h = 0; h < HELD; ++h) add_to<OP>(place[h], held[h], acc[h], i);
}

template <class E, int D>
struct Op : Op16<E, D> {
    using Ring = Ring16<E, D>;
};

template <class OP>
hipError_t launch_op(const WeighParams &p, int way, int held, hipStream_t s) {
    const int rows = p.S * p.group, per = way > kByRows ? 64 * (way - kByRows) : 16 * way;
    const dim3 grid((unsigned)((rows + per - 1) / per) * p.nsplit * p.n_kv_heads), block(256);
    if (way == 1) {
        hipLaunchKernelGGL((weigh_stats_kernel<OP, 1>), grid, block, 0, s, p);
    } else if constexpr (OP::ELT == 4) {
        hipLaunchKernelGGL((weigh_stats_kernel<OP, 2>), grid, block, 0, s, p);
    } else {
        if (way == kByRows + 2) hipLaunchKernelGGL((weigh_stats_rows_kernel<OP, typename OP::Ring, 2>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((weigh_stats_rows_kernel<OP, typename OP::Ring, 4>), grid, block, 0, s, p);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.norm) {
        hipLaunchKernelGGL(weigh_norm_kernel, dim3((unsigned)(((int64_t)rows * p.n_kv_heads + 31) / 32)), block, 0, s, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const int64_t stages = (p.L + OP::KEYS - 1) / OP::KEYS + (p.S + OP::KEYS - 1) / OP::KEYS;
    const dim3 wgs((unsigned)((stages + WAVES * held - 1) / (WAVES * held) * p.n_kv_heads));
    if constexpr (OP::ELT == 2) {
        hipLaunchKernelGGL((weigh_sum_rows_kernel<OP, typename OP::Ring>), wgs, block, 0, s, p);
    } else {
        if (held == 2) hipLaunchKernelGGL((weigh_sum_kernel<OP, 2>), wgs, block, 0, s, p);
        else hipLaunchKernelGGL((weigh_sum_kernel<OP, 1>), wgs, block, 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_weigh(const WeighParams &p, int head_dim, int dtype, int way, int held, hipStream_t s) {
    if (dtype == KVR_F32) return head_dim == 128 ? launch_op<Op32<128>>(p, way, held, s) : launch_op<Op32<64>>(p, way, held, s);
    if (dtype == KVR_F16) return head_dim == 128 ? launch_op<Op<F16, 128>>(p, way, held, s) : launch_op<Op<F16, 64>>(p, way, held, s);
    return head_dim == 128 ? launch_op<Op<Bf16, 128>>(p, way, held, s) : launch_op<Op<Bf16, 64>>(p, way, held, s);
}

}  // namespace kvr
