// decode.hip -- attention of one new token of each sequence over its pages.
//
//   out[r, h] = softmax_j(scale q[r, h] . k_j) v_j,  j < len[r] + n_new, j's page in the pool
//
// The lengths are read on the device, so the work is shared out there too: the keys of a sequence and kv
// head are units, a stage of 32 (fp32: 16) for each wave of a workgroup, and the units of the whole batch, one
// sequence and head after the other, are cut into equal ranges, one for each workgroup.  However ragged the
// batch, every workgroup reads as much.  A sequence and head that lie in one range are finished there; pieces
// of one that several ranges share are records (m, l, O) of the workspace, which a second launch joins in
// their order.  Short or many sequences: a workgroup, or a wave, takes one and nothing is joined (paged_api.hip).
//
// A wave's stages go from memory straight to the registers that the matrix instructions read
// (attn_direct.hpp); a stage's two halves of 16 rows lie in one page each, and a buffer
// resource ends with a half's last row, so rows behind a sequence's length, and all rows of a
// page that is not in the pool, read as zeros and touch no memory.  The next stage's keys
// are asked for when the scores are done, its values when the outputs are, across the
// ends of sequences too: its pages are looked up another stage ahead, with scalar loads, which
// do not wait behind the keys and values that are on their way.
//
// HBM bounds it: G operations for each byte of 16-bit keys and values, G query heads to a kv head.
// Measured, a range's kernel and the join, in us (32 / 8 heads of 128 where nothing else is said):
//   64 sequences of 300 to 32768 rows   619 + 4.6    4.3 GB, 7.0 TB/s, what a launch that only reads reaches
//   64 of up to 4096, fp16              83.4 + 4.7   538 MB, 6.5 TB/s (reading: 6.7)
//   one of 32768                        23.9 + 4.5   134 MB, 5.6 TB/s (reading: 6.3): four stages a wave
//   one of 3774                         7.0 + 3.5    latency: lengths, page, keys, records, the second launch
//   9 of up to 945, 16 / 2 heads of 64, fp32   5.4 + 3.6   latency
//   64 of 100 to 16000, fp32            740 in all   4.2 GB, 5.7 TB/s; 32 / 1 heads 124: 530 MB, 4.3 TB/s
// A stage of 32 bf16 keys of 128 dimensions is 16 loads, 32 matrix and 161 vector instructions, one wave on a SIMD.
// What it took, in a graph: records joined a query row a workgroup, one of 32768 38 -> 31.7 us; pages by scalar loads
// (vector loads wait behind the keys on their way), 32 of 10 to 480 rows shared out 17 -> 14.4 and fewer registers,
// 64 of up to 32768 768 -> 720; scores that wait for the keys only, 64 of 100 to 480 20.0 -> 19.5.
#include <float.h>

#include "paged/paged_internal.hpp"
#include "paged/walk.hpp"
#include "readers/attn_direct.hpp"

namespace kvr {
namespace {

using namespace dev;

// The two element kinds: a stage's weights as the second product's operands.  16-bit: the weight
// cut to the element type, and what that left over, rounded (fp16: 22 bits) or, in bf16, cut and rounded once more
// (24), so that outputs are off by their own rounding alone; the products are matrix instructions that wait for
// memory anyway.  With two operands in bf16 (16 bits) 0.39 % of the outputs of 64 sequences of 300 to 32768 rows are
// another bf16 number than the exact ones rounded, with three 0.06 %, and 32-bit arithmetic of weights rounded once has
// 0.1 %; in a graph 632 and 635 us, one sequence of 300 rows 6.3 and 6.6, of 32768 27.1 and 27.5.
// A cut is of a little less than its number: then all operands are positive, and an infinite value stays one, down to
// weights of 2^-36 (fp16: the rest, too, is at least the smallest number) or 2^-60 (bf16) of the largest.  Below, it is
// no number.
template <class OP, int N>
struct Weights {
    typename OP::P part[N];      // the largest first
};
template <class E, int D>
struct Dec16 : Op16<E, D> {
    using B = Op16<E, D>;
    static constexpr int PARTS = 2;
    // of the rest: it rounds to the smallest fp16 number (and less than that: a weight of zero is not cut to minus it)
    static constexpr float LEAST = std::is_same<E, F16>::value ? 0x1.fffp-25f : 0.f;
    static constexpr int WEIGHTS = std::is_same<E, F16>::value ? 2 : 3;
    using W = Weights<B, WEIGHTS>;
    // part h of a stage
    template <int HINT>
    __device__ static __forceinline__ void load_k(typename B::K &k, __amdgpu_buffer_rsrc_t r, int h, int i, int g) {
#pragma unroll
        for (int ks = 0; ks < B::NK; ++ks)
            k.f[h][ks] = __builtin_amdgcn_raw_buffer_load_b128(r, B::ROWB * i + 16 * g + 64 * ks, 0, HINT);
    }
    template <int HINT>
    __device__ static __forceinline__ void load_v(typename B::V &v, __amdgpu_buffer_rsrc_t r, int h, int i, int g) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int off = (4 * g + e) * B::ROWB + 2 * B::NT * i;
            if constexpr (B::NT == 8) v.r[4 * h + e] = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, HINT);
            else v.r[4 * h + e] = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, HINT);
        }
    }
    __device__ static __forceinline__ uint32_t cut2(float a, float b) {
        if constexpr (std::is_same<E, F16>::value) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
        else return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
    __device__ static __forceinline__ void pack(W &w, const float (&p)[B::NS], float lift) {
        const float cut = lift * (1.f - 0x1p-20f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a = __builtin_fmaf(p[2 * j], cut, -LEAST), b = __builtin_fmaf(p[2 * j + 1], cut, -LEAST);
            uint32_t x = cut2(a, b);
            w.part[0].f[j] = x;
            float r = __builtin_fmaf(p[2 * j], lift, -E::lo(x)), s = __builtin_fmaf(p[2 * j + 1], lift, -E::hi(x));
            if constexpr (WEIGHTS == 3) {
                x = cut2(r * (1.f - 0x1p-12f), s * (1.f - 0x1p-12f));
                w.part[1].f[j] = x;
                r -= E::lo(x);
                s -= E::hi(x);
            }
            w.part[WEIGHTS - 1].f[j] = E::pack2(r, s);
        }
    }
    template <int RT>
    __device__ static __forceinline__ void outputs(const typename B::V &v, const W (&w)[RT], f32x4 (&o)[RT][B::NT]) {
#pragma unroll
        for (int t = 0; t < B::NT; ++t) {
            const u32x4 a = B::column(v, t);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int n = WEIGHTS - 1; n >= 0; --n) o[rt][t] = B::mfma(a, w[rt].part[n].f, o[rt][t]);
            if (RT > 1 && t % 2) __builtin_amdgcn_sched_barrier(0);      // operands of two at a time
        }
    }
};
template <int D>
struct Dec32 : Op32<D> {
    using B = Op32<D>;
    static constexpr int PARTS = 1;
    using W = typename B::P;
    template <int HINT>
    __device__ static __forceinline__ void load_k(typename B::K &k, __amdgpu_buffer_rsrc_t r, int, int i, int g) {
#pragma unroll
        for (int ks = 0; ks < B::NK; ++ks) k.f[ks] = load<HINT>(r, B::ROWB * i + 16 * g + 64 * ks);
    }
    template <int HINT>
    __device__ static __forceinline__ void load_v(typename B::V &v, __amdgpu_buffer_rsrc_t r, int, int i, int g) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < B::NT / 4; ++j) v.r[e][j] = load<HINT>(r, B::ROWB * (4 * g + e) + 4 * B::NT * i + 16 * j);
    }
    template <int HINT>
    __device__ static __forceinline__ f32x4 load(__amdgpu_buffer_rsrc_t r, int off) {
        return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, HINT));
    }
    __device__ static __forceinline__ void pack(W &w, const float (&p)[B::NS], float lift) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w.f[e] = p[e] * lift;
    }
    template <int RT>
    __device__ static __forceinline__ void outputs(const typename B::V &v, const W (&w)[RT], f32x4 (&o)[RT][B::NT]) {
        B::template accumulate<RT>(v, w, o);
    }
};

// What the page table says for a stage's parts.  Asked for two stages ahead.
template <class OP, int WAVES>
struct Pages {
    int page[OP::PARTS];
    __device__ __forceinline__ void ask(const DecodeParams &p, const Unit &b, int wave) {
        const int key = (b.u * WAVES + wave) * OP::KEYS;
        int at = b.page, part = b.part;
#pragma unroll
        for (int h = 0; h < OP::PARTS; ++h) {
            // (a part without rows has no entry of its own)
            page[h] = scalar(p.table + (int64_t)b.r * p.max_pages + (key + 16 * h < b.rows ? at : 0));
            if (++part == p.page_size >> 4) part = 0, ++at;
        }
    }
};

// A wave's stage of a unit: its parts' first rows, and how many there are
template <class OP, int WAVES>
struct Stage {
    int rows[OP::PARTS];
    uint64_t at[OP::PARTS];      // bytes from the pool's first
    __device__ __forceinline__ Stage() {      // none
#pragma unroll
        for (int h = 0; h < OP::PARTS; ++h) rows[h] = at[h] = 0;
    }
    __device__ __forceinline__ Stage(const DecodeParams &p, const Unit &b, const Pages<OP, WAVES> &pages, int wave) {
        const uint64_t first = (uint64_t)(b.hd / p.tiles) * (uint32_t)p.page_size;
        const int key = (b.u * WAVES + wave) * OP::KEYS;
        int part = b.part;
#pragma unroll
        for (int h = 0; h < OP::PARTS; ++h) {
            const int n = min(b.rows - (key + 16 * h), 16);
            const bool there = n > 0 && (uint32_t)pages.page[h] < (uint32_t)p.n_pages;
            rows[h] = there ? n : 0;
            at[h] = there ? (uint64_t)pages.page[h] * (uint64_t)p.page_bytes + (first + 16 * (uint32_t)part) * OP::ROWB : 0;
            if (++part == p.page_size >> 4) part = 0;
        }
    }
    template <int HINT>
    __device__ __forceinline__ void load_k(const DecodeParams &p, typename OP::K &k, int i, int g) const {
#pragma unroll
        for (int h = 0; h < OP::PARTS; ++h)
            OP::template load_k<HINT>(k, row_rsrc((uint64_t)p.kp + at[h], rows[h], OP::ROWB, OP::ROWB), h, i, g);
    }
    template <int HINT>
    __device__ __forceinline__ void load_v(const DecodeParams &p, typename OP::V &v, int i, int g) const {
#pragma unroll
        for (int h = 0; h < OP::PARTS; ++h)
            OP::template load_v<HINT>(v, row_rsrc((uint64_t)p.vp + at[h], rows[h], OP::ROWB, OP::ROWB), h, i, g);
    }
};

// The sum of no weights.  Sums of it alone keep its sign, one with a weight of zero does not: keys whose scores
// are all -infinity leave +0, and their softmax is no number; no keys leave this, and give zeros.
constexpr float kNoKeys = -0.f;
// What makes a row's products its output
__device__ __forceinline__ float reciprocal(float l) {
    return l > 0.f ? 1.f / l : __float_as_uint(l) == __float_as_uint(kNoKeys) ? 0.f : __builtin_nanf("");
}

template <class OP, int RT>
struct Rows {
    f32x4 o[RT][OP::NT];
    float m[RT], l[RT];      // half the largest score; the lane's share of the row's sum
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -FLT_MAX;
            l[rt] = 0.f;
#pragma unroll
            for (int t = 0; t < OP::NT; ++t) o[rt][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
    }
};

// Scores become weights 2^(c2 (s / 2 - m)), m half the largest score so far.  The difference comes first: the largest
// score's is zero, however large it is (less a rounded reference of c2 s it is half a step of that, whole powers of two
// from scores of 1e7 on).  It is of halves: two finite scores may be an infinity apart.
template <class OP, int RT>
__device__ __forceinline__ void softmax_step(Rows<OP, RT> &R, float (&s)[RT][OP::NS], typename OP::W (&w)[RT],
                                             const int (&rows)[OP::PARTS], float c2, float lift, int g) {
    int all = rows[0];
#pragma unroll
    for (int h = 1; h < OP::PARTS; ++h) all += rows[h];
    if (all < OP::KEYS) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int e = 0; e < OP::NS; ++e)
                if (4 * g + (e & 3) >= rows[e >> 2]) s[rt][e] = -INFINITY;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float mx = s[rt][0];
#pragma unroll
        for (int e = 1; e < OP::NS; ++e) mx = fmaxf(mx, s[rt][e]);
        mx = fmaxf(0.5f * quad_max(mx), R.m[rt]);
        if (__ballot(mx > R.m[rt])) {
            const float a = __builtin_amdgcn_exp2f((R.m[rt] - mx) * c2);
            R.m[rt] = mx;
            R.l[rt] *= a;
#pragma unroll
            for (int t = 0; t < OP::NT; ++t) R.o[rt][t] *= a;
        }
        float p[OP::NS], sum = 0.f;
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) {
            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][e], 0.5f, -R.m[rt]) * c2);
            sum += p[e];
        }
        R.l[rt] += sum;
        OP::pack(w[rt], p, lift);
    }
}

// The query rows of a kv head's tile; past the last one it again, not to be stored
template <class OP, int RT>
__device__ __forceinline__ void take_queries(const DecodeParams &p, typename OP::Q (&q)[RT], int r, int hd, int i, int g) {
    const int kh = hd / p.tiles, row0 = (hd - kh * p.tiles) * 16 * RT;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = min(row0 + 16 * rt + i, p.group - 1);
        const int64_t at = r * p.q.token + (kh * p.group + row) * p.q.head;
        OP::load_q(q[rt], (const unsigned char *)p.q.p + at * OP::ELT, g);
    }
}

// Where record rec keeps O, and (m, l)
template <class OP>
__device__ __forceinline__ float *record_o(const DecodeParams &p, int64_t rec) {
    return p.ws + rec * p.rows * OP::DIM;
}
template <class OP>
__device__ __forceinline__ float2 *record_ml(const DecodeParams &p, int64_t rec) {
    return (float2 *)(p.ws + (int64_t)2 * p.grid * p.rows * OP::DIM) + rec * p.rows;
}
// The first and the last workgroup of a sequence and head
template <class OP>
__device__ __forceinline__ int2 *sharers_of(const DecodeParams &p, int r, int hd) {
    return (int2 *)(p.ws + (int64_t)2 * p.grid * p.rows * (OP::DIM + 2)) + (int64_t)r * p.n_kv_heads * p.tiles + hd;
}

// LDS of a join of one row tile by a workgroup's waves: O, component c of the lane's four apart, and (m, l)
template <class OP, int WAVES>
struct Join {
    static constexpr int NT = OP::NT;
    f32x4 o[WAVES][4][64][NT / 4];
    float2 ml[WAVES][64];
};

// The units from b on
template <class OP, int RT, int WAVES, int HINT>
__device__ __forceinline__ void decode_units(const DecodeParams &p, Walk<OP, WAVES> &walk, Unit b, int at, const Cut &cut, int wg,
                                             int wave, int lane) {
    constexpr int NT = OP::NT;
    using St = Stage<OP, WAVES>;
    const int i = lane & 15, g = lane >> 4;
    const float c2 = p.half_scale_log2, lift = p.lift;
    Unit n1, n2;       // the next unit, the one after it
    Pages<OP, WAVES> p1, p2;
    p1.ask(p, b, wave);
    typename OP::Q q[RT];
    typename OP::K k;
    typename OP::V v;
    Rows<OP, RT> R;
    // in this order, as the loop has it: it waits for the keys only, with the values on their way
    take_queries<OP, RT>(p, q, b.r, b.hd, i, g);
    St st(p, b, p1, wave);
    __builtin_amdgcn_sched_barrier(0);
    st.template load_k<HINT>(p, k, i, g);
    __builtin_amdgcn_sched_barrier(0);
    st.template load_v<HINT>(p, v, i, g);
    __builtin_amdgcn_sched_barrier(0);
    n1 = b;
    bool more = walk.next(p, n1, lane);
    if (more) p1.ask(p, n1, wave);
    int seg_u = b.u;      // the segment's first unit here
    int seen = 0;         // whether the wave has had any keys of it
    R.clear();

    for (;;) {
        float s[RT][OP::NS];
        typename OP::W w[RT];
        int rows[OP::PARTS];
#pragma unroll
        for (int h = 0; h < OP::PARTS; ++h) seen |= rows[h] = st.rows[h];
        if (more) st = St(p, n1, p1, wave);
        else st = St();
        n2 = n1;
        const bool more2 = walk.next(p, n2, lane);
        if (more2) p2.ask(p, n2, wave);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) OP::scores(k, q[rt], s[rt]);
        __builtin_amdgcn_sched_barrier(0);
        st.template load_k<HINT>(p, k, i, g);
        __builtin_amdgcn_sched_barrier(0);
        softmax_step<OP, RT>(R, s, w, rows, c2, lift, g);
        OP::template outputs<RT>(v, w, R.o);
        __builtin_amdgcn_sched_barrier(0);
        st.template load_v<HINT>(p, v, i, g);
        __builtin_amdgcn_sched_barrier(0);
        const bool seg_end = b.last();
        if (seg_end || !more) {
            if (more) take_queries<OP, RT>(p, q, n1.r, n1.hd, i, g);
            const bool whole = seg_end && seg_u == 0;
            const int kh = b.hd / p.tiles, row0 = (b.hd - kh * p.tiles) * 16 * RT;
            // a piece that begins its segment is the workgroup's last, its second record
            const int64_t rec = 2 * (int64_t)wg + (seg_u == 0 ? 1 : 0);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int row = row0 + 16 * rt + i;
                const bool on = row < p.group;
                const float l = seen ? quad_sum(R.l[rt]) : kNoKeys;
                // c: the component of the lane's four, head-dim indices NT (4 g + c) ..
                auto put = [&](int c, const f32x4 (&acc)[NT / 4], float M, float L) {
                    const int d = NT * (4 * g + c);
                    if (whole) {
                        const float inv = reciprocal(L) * p.unlift;
                        unsigned char *out = (unsigned char *)p.out + ((int64_t)b.r * p.n_q_heads + kh * p.group + row) * OP::ROWB;
#pragma unroll
                        for (int t = 0; t < NT / 4; ++t)
                            OP::put4(out, d + 4 * t, acc[t][0] * inv, acc[t][1] * inv, acc[t][2] * inv, acc[t][3] * inv);
                    } else {
                        float *po = record_o<OP>(p, rec) + (int64_t)(row - row0) * OP::DIM + d;
#pragma unroll
                        for (int t = 0; t < NT / 4; ++t) *(f32x4 *)(po + 4 * t) = acc[t];
                        if (c == 0 && g == 0) record_ml<OP>(p, rec)[row - row0] = make_float2(M, L);
                    }
                };
                if constexpr (WAVES == 1) {
                    if (on) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            f32x4 acc[NT / 4];
#pragma unroll
                            for (int t = 0; t < NT; t += 4) acc[t / 4] = (f32x4){R.o[rt][t][c], R.o[rt][t + 1][c], R.o[rt][t + 2][c], R.o[rt][t + 3][c]};
                            put(c, acc, R.m[rt], l);
                        }
                    }
                } else {
                    __shared__ Join<OP, WAVES> lds;
                    __syncthreads();      // the join before this one has been read
                    if (on) {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int t = 0; t < NT; t += 4)
                                lds.o[wave][c][lane][t / 4] = (f32x4){R.o[rt][t][c], R.o[rt][t + 1][c], R.o[rt][t + 2][c], R.o[rt][t + 3][c]};
                        lds.ml[wave][lane] = make_float2(R.m[rt], l);
                    }
                    __syncthreads();
                    if (on && wave < 4) {
                        float M = -FLT_MAX, L = kNoKeys;
                        f32x4 acc[NT / 4];
#pragma unroll
                        for (int t = 0; t < NT / 4; ++t) acc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int s = 0; s < WAVES; ++s) M = fmaxf(M, lds.ml[s][lane].x);
#pragma unroll
                        for (int s = 0; s < WAVES; ++s) {
                            const float2 ml = lds.ml[s][lane];
                            const float a = __builtin_amdgcn_exp2f((ml.x - M) * c2);
                            L = __builtin_fmaf(a, ml.y, L);
#pragma unroll
                            for (int t = 0; t < NT / 4; ++t)
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[t][e] = __builtin_fmaf(a, lds.o[s][wave][lane][t][e], acc[t][e]);
                        }
                        put(wave, acc, M, L);
                    }
                }
            }
            if (!p.alone && seg_u == 0 && threadIdx.x == 0) {
                const int last = at + b.units - 1;      // the segment's last unit
                *sharers_of<OP>(p, b.r, b.hd) = make_int2(wg, whole ? wg : cut.range_of(last));
            }
            R.clear();
            // the queries have landed: otherwise every stage's scores would wait for what was asked for before
            // these, its values among it
            wait_vmcnt<0>();
            at += b.u + 1 - seg_u;      // of the next segment's first unit
            seg_u = seen = 0;
        }
        if (!more) break;
        b = n1;
        n1 = n2;
        p1 = p2;
        more = more2;
    }
}

// The non-temporal hint of a buffer load
constexpr int kStream = 2;

// STREAM: the call may read so much that keys and values go around the caches.  How much it is is
// known here only; the loop stands twice, as waits for loads are counted in each path by itself.
template <class OP, int RT, int WAVES, bool STREAM>
__global__ __launch_bounds__(64 * WAVES, 2) void decode_kernel(const DecodeParams p) {
    const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : uniform(threadIdx.x >> 6), wg = blockIdx.x;
    Walk<OP, WAVES> walk(p, wave);
    Unit b;
    Cut cut;
    int at;
    if (!walk.first(p, b, at, wg, cut, wave, lane)) return;
    if constexpr (STREAM) {
        if (cut.total >= p.stream_units) {
            decode_units<OP, RT, WAVES, kStream>(p, walk, b, at, cut, wg, wave, lane);
            return;
        }
    }
    decode_units<OP, RT, WAVES, 0>(p, walk, b, at, cut, wg, wave, lane);
}

// The records of ROWS query rows of a sequence and head, joined in an order that the lengths fix:
// several ways take a row's records in turn, LANES lanes of four values each, and their sums are joined.
template <class OP, int ROWS>
__global__ __launch_bounds__(256) void decode_merge_kernel(const DecodeParams p) {
    constexpr int D = OP::DIM, LANES = D / 4, WAYS = 256 / LANES / ROWS, BATCH = 4;
    __shared__ f32x4 sums[256];
    __shared__ float2 mls[WAYS * ROWS];
    const int heads = p.n_kv_heads * p.tiles, groups = (p.rows + ROWS - 1) / ROWS;
    const int seg = blockIdx.x / groups, r = seg / heads, hd = seg - r * heads;
    int2 wgs = *sharers_of<OP>(p, r, hd);
    if (rows_of(p, scalar(p.len + r)) < 0 || wgs.x == wgs.y) return;
    wgs.x = max(wgs.x, 0);      // (anything, if the lengths are not what they were)
    wgs.y = min(wgs.y, p.grid - 1);
    const int slot = threadIdx.x / LANES, way = slot / ROWS, d = threadIdx.x % LANES * 4;
    const int kh = hd / p.tiles, row0 = (hd - kh * p.tiles) * p.rows, rows = min(p.rows, p.group - row0);
    const int at = (blockIdx.x - seg * groups) * ROWS + slot % ROWS, row = min(at, rows - 1);
    float M = -FLT_MAX, l = kNoKeys;
    f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int s0 = wgs.x + way; s0 <= wgs.y; s0 += WAYS * BATCH) {
        f32x4 x[BATCH];
        float2 w[BATCH];
        float mx = M;
#pragma unroll
        for (int s = 0; s < BATCH; ++s) {
            const int wg = s0 + s * WAYS;
            w[s] = make_float2(-FLT_MAX, kNoKeys);
            x[s] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if (wg <= wgs.y) {
                const int64_t rec = 2 * (int64_t)wg + (wg == wgs.x ? 1 : 0);
                x[s] = *(const f32x4 *)(record_o<OP>(p, rec) + (int64_t)row * D + d);
                w[s] = record_ml<OP>(p, rec)[row];
            }
        }
#pragma unroll
        for (int s = 0; s < BATCH; ++s) mx = fmaxf(mx, w[s].x);
        const float a = __builtin_amdgcn_exp2f((M - mx) * p.half_scale_log2);
        M = mx;
        l *= a;
        acc *= a;
#pragma unroll
        for (int s = 0; s < BATCH; ++s) {
            const float f = __builtin_amdgcn_exp2f((w[s].x - M) * p.half_scale_log2);
            l = __builtin_fmaf(f, w[s].y, l);
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = __builtin_fmaf(f, x[s][c], acc[c]);
        }
    }
    sums[threadIdx.x] = acc;
    if (d == 0) mls[slot] = make_float2(M, l);
    __syncthreads();
    if (way || at >= rows) return;
    float top = M;
#pragma unroll
    for (int s = 1; s < WAYS; ++s) top = fmaxf(top, mls[s * ROWS + slot].x);
    const float a = __builtin_amdgcn_exp2f((M - top) * p.half_scale_log2);
    l *= a;
    acc *= a;
#pragma unroll
    for (int s = 1; s < WAYS; ++s) {
        const float2 ml = mls[s * ROWS + slot];
        const float f = __builtin_amdgcn_exp2f((ml.x - top) * p.half_scale_log2);
        l = __builtin_fmaf(f, ml.y, l);
        const f32x4 x = sums[s * ROWS * LANES + threadIdx.x];
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = __builtin_fmaf(f, x[c], acc[c]);
    }
    const float inv = reciprocal(l) * p.unlift;
    const int64_t to = (int64_t)r * p.n_q_heads + kh * p.group + row0 + row;
    OP::put4((unsigned char *)p.out + to * OP::ROWB, d, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}

template <class OP>
hipError_t launch_op(const DecodeParams &p, hipStream_t s) {
    const dim3 grid((unsigned)p.grid);
    if (p.rows > 16) {
        if (p.waves == 4) hipLaunchKernelGGL((decode_kernel<OP, 2, 4, false>), grid, dim3(256), 0, s, p);
        else hipLaunchKernelGGL((decode_kernel<OP, 2, 1, false>), grid, dim3(64), 0, s, p);
    } else if (p.waves == 1) {
        hipLaunchKernelGGL((decode_kernel<OP, 1, 1, false>), grid, dim3(64), 0, s, p);
    } else if (p.stream_units) {
        hipLaunchKernelGGL((decode_kernel<OP, 1, 4, true>), grid, dim3(256), 0, s, p);
    } else {
        hipLaunchKernelGGL((decode_kernel<OP, 1, 4, false>), grid, dim3(256), 0, s, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.alone) return e;
    const int segs = p.n * p.n_kv_heads * p.tiles;
    if (p.merge_rows == 1) hipLaunchKernelGGL((decode_merge_kernel<OP, 1>), dim3((unsigned)(segs * p.rows)), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((decode_merge_kernel<OP, 4>), dim3((unsigned)(segs * ((p.rows + 3) / 4))), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_decode(const DecodeParams &p, int head_dim, int dtype, hipStream_t s) {
    if (dtype == KVR_F32) return head_dim == 128 ? launch_op<Dec32<128>>(p, s) : launch_op<Dec32<64>>(p, s);
    if (dtype == KVR_F16) return head_dim == 128 ? launch_op<Dec16<F16, 128>>(p, s) : launch_op<Dec16<F16, 64>>(p, s);
    return head_dim == 128 ? launch_op<Dec16<Bf16, 128>>(p, s) : launch_op<Dec16<Bf16, 64>>(p, s);
}

}  // namespace kvr
