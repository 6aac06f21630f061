// attn_direct.hpp -- attention tiles whose K and V rows go from memory straight
// to the registers that the matrix instructions read: no LDS and no barrier in
// the key loop.  Shared by shared.hip (attention of many readers) and weigh.hip
// (accumulated attention weight).
//
// Notation of one wave and one stage of KEYS keys; a tile is 16 query rows:
//   S^T[key][row]  = K Q^T      A = K: lane (i, g) = (lane % 16, lane / 16) holds 16
//                               consecutive bytes of key i's row (of every 64)
//   O^T[d][row]   += V^T P^T    B = P^T: the score accumulator itself.  It leaves lane
//                               (i, g) with row i and keys 4 g + e of each 16-key part,
//                               and the k-slots of a product only have to name the same
//                               key in A and B.
// A = V^T wants NT = D / 16 operands of one head-dim index and the lane's keys.
// Operand t of lane i is given head-dim index NT i + t, so a lane loads NT
// consecutive elements of each of its keys' V rows (16 lanes read a whole row)
// and, in 16-bit types, transposes them in registers: 4 byte permutes for each
// operand of 8 keys.  The output comes out alike: lane (row, g), operand t,
// component c is head-dim index NT (4 g + c) + t.
//
// Rows come through a buffer resource that ends with the last valid one: a lane
// past it reads zeros and touches no memory, so ragged ends need no address of
// their own, and their scores are masked by the key's index.
#pragma once

#include <type_traits>

#include "attn_common.hpp"

namespace kvr {
namespace dev {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Rows [0, n) of stride_b bytes from `base`, of which row_b are read: the resource
// that ends with row n - 1 (n <= 0: an empty one).  A row of all kv heads has at most 2 MB:
// strides are 24-bit numbers, and a stage of at most 32 rows ends below 2^31.
// All wave-uniform; said so, or the compiler loops over the lanes' resources.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_rsrc(uint64_t base, int n, uint32_t stride_b, uint32_t row_b) {
    const uint32_t bytes = n > 0 ? (uint32_t)(n - 1) * stride_b + row_b : 0u;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)base), hi = __builtin_amdgcn_readfirstlane((uint32_t)(base >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void *)(uintptr_t)((uint64_t)hi << 32 | lo), 0,
                                             __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// Maximum and sum over the four lanes of a query row (lanes i, i + 16, i + 32, i + 48;
// the same bits in each)
__device__ __forceinline__ float quad_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// 16-bit elements (E: Bf16 or F16): stages of 32 keys, two 16-key parts
template <class E, int D>
struct Op16 {
    static constexpr int DIM = D, KEYS = 32, NS = 8, NT = D / 16, NK = D / 32, ROWB = D * 2, ELT = 2;
    struct Q {
        u32x4 f[NK];
    };
    typedef uint32_t vrow __attribute__((ext_vector_type(NT / 2)));
    struct K {
        u32x4 f[2][NK];
    };
    struct V {
        vrow r[8];
    };
    // the lane's key of score e
    __device__ static __forceinline__ int key_of(int e, int g) { return 16 * (e >> 2) + 4 * g + (e & 3); }

    __device__ static __forceinline__ void load_q(Q &q, const void *row, int g) {
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) q.f[ks] = *(const u32x4 *)((const unsigned char *)row + 64 * ks + 16 * g);
    }
    // cs: the table row of the position
    __device__ static __forceinline__ void rotate_q(Q &q, const float *cs, int g) {
#pragma unroll
        for (int ks = 0; ks < NK / 2; ++ks) rope_rot8<E>(q.f[ks], q.f[ks + NK / 2], cs + 2 * (32 * ks + 8 * g));
    }
    // PARTS = 1: a stage of at most 16 rows, the other part zeros
    template <int PARTS = 2>
    __device__ static __forceinline__ void load_k(K &k, __amdgpu_buffer_rsrc_t r, uint32_t stride_b, int i, int g) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ks = 0; ks < NK; ++ks)
                k.f[h][ks] = h < PARTS ? buf_load16(r, __umul24(16 * h + i, stride_b) + 16 * g + 64 * ks)
                                       : (u32x4){0u, 0u, 0u, 0u};
    }
    template <int PARTS = 2>
    __device__ static __forceinline__ void load_v(V &v, __amdgpu_buffer_rsrc_t r, uint32_t stride_b, int i, int g) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t off = __umul24(key_of(e, g), stride_b) + 2 * NT * i;
            if (e >= 4 * PARTS) v.r[e] = vrow(0);
            else if constexpr (NT == 8) v.r[e] = buf_load16(r, off);
            else v.r[e] = __builtin_amdgcn_raw_buffer_load_b64(r, (int)off, 0, 0);
        }
    }
    // new key rows: position of key c of the stage is that of table row cs + c * D
    template <int PARTS = 2>
    __device__ static __forceinline__ void rotate_k(K &k, const float *cs, int n, int i, int g) {
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
            const int c = min(16 * h + i, n - 1);      // a row past the last is masked: any table row
#pragma unroll
            for (int ks = 0; ks < NK / 2; ++ks)
                rope_rot8<E>(k.f[h][ks], k.f[h][ks + NK / 2], cs + c * D + 2 * (32 * ks + 8 * g));
        }
    }
    // rows [0, n) of the stage into consecutive rows of a cache
    template <int PARTS = 2>
    __device__ static __forceinline__ void store(const K &k, const V &v, unsigned char *kd, unsigned char *vd, int n,
                                                 int i, int g) {
#pragma unroll
        for (int h = 0; h < PARTS; ++h)
            if (16 * h + i < n)
#pragma unroll
                for (int ks = 0; ks < NK; ++ks)
                    *(u32x4 *)(kd + (16 * h + i) * ROWB + 64 * ks + 16 * g) = k.f[h][ks];
#pragma unroll
        for (int e = 0; e < 4 * PARTS; ++e)
            if (key_of(e, g) < n) *(vrow *)(vd + key_of(e, g) * ROWB + 2 * NT * i) = v.r[e];
    }
    __device__ static __forceinline__ void scores(const K &k, const Q &q, float (&s)[NS]) {
        f32x4 a[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) a[h] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < NK; ++ks)
#pragma unroll
            for (int h = 0; h < 2; ++h) a[h] = mfma(k.f[h][ks], q.f[ks], a[h]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = a[e >> 2][e & 3];
    }
    // Weights as the second product's operand: the element type, rounded to nearest
    // even, each off by half a step at most.  The row's sum is taken from the rounded
    // ones, as one more product (with ones in the place of V^T: every component is the
    // row's sum over all the wave's keys), so that out = sum p v / sum p stays a mean of
    // the values: where one weight dominates, its rounding cancels.
    using L = f32x4;
    __device__ static __forceinline__ L no_sum() { return (f32x4){0.f, 0.f, 0.f, 0.f}; }
    __device__ static __forceinline__ float total(const L &l) { return l[0]; }
    struct P {
        u32x4 f;
    };
    __device__ static __forceinline__ void weights(P &w, const float (&p)[NS]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t x = E::pack2(p[2 * j], p[2 * j + 1]);
            asm("" : "+v"(x));      // one conversion of two: the halves' maxima below would split it
            w.f[j] = x;
        }
    }
    __device__ static __forceinline__ void add(L &l, const P &w) {
        constexpr uint32_t one = std::is_same<E, F16>::value ? 0x3c003c00u : 0x3f803f80u;
        l = mfma((u32x4){one, one, one, one}, w.f, l);
    }
    // When a row's reference moves, to where the largest weight is 2^kLift.  A weight that holds
    // much of its row must not be rounded, or results of two orders of keys differ by it: the
    // largest one so far is a power of two, and one that grows above it moves the reference as
    // soon as it is more than a third of the sum so far (a quarter of both), or the operand or
    // the sums do not hold it:
    //   bf16  above 1: a sum of weights times values is never larger than the same with the
    //         maximum as the reference.  2^-118 of the largest weight is a normal number yet.
    //   fp16  above the type's largest number: 2^31 weights below 2^16, each times a value below
    //         2^16, are far below the largest fp32 number.  There are 14 exponents below 1, and
    //         below them bits go: with the largest weight at 2^12 or more, weights of 2^-26 of it
    //         keep all of theirs.
    static constexpr int kLift = std::is_same<E, F16>::value ? 12 : -8;
    static constexpr float kLargest = std::is_same<E, F16>::value ? 0x1p12f : 0x1p-8f;      // 2^kLift
    typedef uint16_t Pair __attribute__((ext_vector_type(2)));
    // The weight that a row's must not exceed, in both halves, as the element type truncates
    // it; positive floats order as their bits do.  (l: the row's sum)
    using Mark = Pair;
    __device__ static __forceinline__ Mark mark(const L &l) {
        const float x = fmaxf(l[0] * (1.f / 3.f), kLargest);
        if constexpr (std::is_same<E, F16>::value) return __builtin_bit_cast(Pair, __builtin_amdgcn_cvt_pkrtz(x, x));
        const uint32_t u = __float_as_uint(fminf(x, 1.f));
        return __builtin_bit_cast(Pair, __builtin_amdgcn_perm(u, u, 0x07060706u));
    }
    using Peak = Pair;
    __device__ static __forceinline__ Peak peak(const P &w) {
        Peak k = __builtin_bit_cast(Peak, (uint32_t)w.f[0]);
#pragma unroll
        for (int j = 1; j < 4; ++j) k = __builtin_elementwise_max(k, __builtin_bit_cast(Peak, (uint32_t)w.f[j]));
        return k;
    }
    // one of the lane's weights exceeds the mark
    __device__ static __forceinline__ bool above(Peak k, Mark t) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(k, t)) != 0;
    }
    // one of the row's does, the largest of which is top.  A row decides by its own weights and
    // sum, and a mark made earlier is not larger, so it does not matter which of a tile's rows
    // asked.
    __device__ static __forceinline__ bool moves(uint64_t, int, float top, const L &l) {
        return above(__builtin_bit_cast(Peak, E::pack2(top, top)), mark(l));
    }
    // whether every value of the stage is a number (the exponent's bits are not all set)
    __device__ static __forceinline__ bool finite(const V &v) {
        bool ok = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) ok &= finite_words(v.r[e]);
        return ok;
    }
    template <class W>
    __device__ static __forceinline__ bool finite_words(const W &w) {
        constexpr uint32_t ex = std::is_same<E, F16>::value ? 0x7c00u : 0x7f80u;
        bool ok = true;
#pragma unroll
        for (int j = 0; j < (int)(sizeof(W) / 4); ++j) ok &= ((w[j] & ex) != ex) & ((w[j] >> 16 & ex) != ex);
        return ok;
    }
    // an operand of eight keys with zeros in the place of every key but c
    __device__ static __forceinline__ u32x4 only_key(u32x4 a, int c, int g) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            a[j] &= key_of(2 * j, g) == c ? 0xffffu : key_of(2 * j + 1, g) == c ? 0xffff0000u : 0u;
        return a;
    }
    // operand t of V^T: elements t of keys 2j (low half) and 2j + 1 (high half)
    __device__ static __forceinline__ u32x4 column(const V &v, int t) {
        u32x4 a;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            a[j] = __builtin_amdgcn_perm(v.r[2 * j + 1][t / 2], v.r[2 * j][t / 2], (t & 1) ? 0x07060302u : 0x05040100u);
        return a;
    }
    // o[rt][t] += V^T P^T of every tile
    template <int RT>
    __device__ static __forceinline__ void accumulate(const V &v, const P (&w)[RT], f32x4 (&o)[RT][NT]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const u32x4 a = column(v, t);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) o[rt][t] = mfma(a, w[rt].f, o[rt][t]);
        }
    }
    // the same of key c alone (zeros in the place of the others), for the rows that see it
    template <int RT>
    __device__ static __forceinline__ void accumulate_key(const V &v, const P (&w)[RT], f32x4 (&o)[RT][NT], int c,
                                                          const bool (&sees)[RT], int g) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const u32x4 a = only_key(column(v, t), c, g);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const f32x4 x = mfma(a, w[rt].f, o[rt][t]);
                o[rt][t] = sees[rt] ? x : o[rt][t];
            }
        }
    }
    __device__ static __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        if constexpr (std::is_same<E, F16>::value)
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c,
                                                          0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
    }
    // four consecutive outputs
    __device__ static __forceinline__ void put4(void *row, int d, float a, float b, float c, float e) {
        u32x2 v;
        v[0] = E::pack2(a, b);
        v[1] = E::pack2(c, e);
        *(u32x2 *)((uint16_t *)row + d) = v;
    }
};

// fp32: stages of 16 keys, one element for each lane of an operand
template <int D>
struct Op32 {
    static constexpr int DIM = D, KEYS = 16, NS = 4, NT = D / 16, NK = D / 16, ROWB = D * 4, ELT = 4;
    struct Q {
        f32x4 f[NK];
    };
    struct K {
        f32x4 f[NK];
    };
    struct V {
        f32x4 r[4][NT / 4];
    };
    struct P {
        float f[4];
    };
    __device__ static __forceinline__ int key_of(int e, int g) { return 4 * g + e; }

    __device__ static __forceinline__ f32x4 load(__amdgpu_buffer_rsrc_t r, uint32_t off) {
        return __builtin_bit_cast(f32x4, buf_load16(r, off));
    }
    __device__ static __forceinline__ void load_q(Q &q, const void *row, int g) {
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) q.f[ks] = *(const f32x4 *)((const unsigned char *)row + 64 * ks + 16 * g);
    }
    __device__ static __forceinline__ void turn(f32x4 &a, f32x4 &b, const float *cs) {
        const f32x4 c01 = *(const f32x4 *)cs, c23 = *(const f32x4 *)(cs + 4);
        float x[4], y[4];
        rope_rot(a[0], b[0], c01[0], c01[1], x[0], y[0]);
        rope_rot(a[1], b[1], c01[2], c01[3], x[1], y[1]);
        rope_rot(a[2], b[2], c23[0], c23[1], x[2], y[2]);
        rope_rot(a[3], b[3], c23[2], c23[3], x[3], y[3]);
        a = (f32x4){x[0], x[1], x[2], x[3]};
        b = (f32x4){y[0], y[1], y[2], y[3]};
    }
    __device__ static __forceinline__ void rotate_q(Q &q, const float *cs, int g) {
#pragma unroll
        for (int ks = 0; ks < NK / 2; ++ks) turn(q.f[ks], q.f[ks + NK / 2], cs + 2 * (16 * ks + 4 * g));
    }
    template <int PARTS = 1>
    __device__ static __forceinline__ void load_k(K &k, __amdgpu_buffer_rsrc_t r, uint32_t stride_b, int i, int g) {
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) k.f[ks] = load(r, __umul24(i, stride_b) + 16 * g + 64 * ks);
    }
    template <int PARTS = 1>
    __device__ static __forceinline__ void load_v(V &v, __amdgpu_buffer_rsrc_t r, uint32_t stride_b, int i, int g) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < NT / 4; ++j)
                v.r[e][j] = load(r, __umul24(key_of(e, g), stride_b) + 4 * NT * i + 16 * j);
    }
    template <int PARTS = 1>
    __device__ static __forceinline__ void rotate_k(K &k, const float *cs, int n, int i, int g) {
        const int c = min(i, n - 1);
#pragma unroll
        for (int ks = 0; ks < NK / 2; ++ks) turn(k.f[ks], k.f[ks + NK / 2], cs + c * D + 2 * (16 * ks + 4 * g));
    }
    template <int PARTS = 1>
    __device__ static __forceinline__ void store(const K &k, const V &v, unsigned char *kd, unsigned char *vd, int n,
                                                 int i, int g) {
        if (i < n)
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) *(f32x4 *)(kd + i * ROWB + 64 * ks + 16 * g) = k.f[ks];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (key_of(e, g) < n)
#pragma unroll
                for (int j = 0; j < NT / 4; ++j)
                    *(f32x4 *)(vd + key_of(e, g) * ROWB + 4 * NT * i + 16 * j) = v.r[e][j];
    }
    // four chains of sums, joined: a chain is NK long instead of D
    __device__ static __forceinline__ void scores(const K &k, const Q &q, float (&s)[NS]) {
        f32x4 a[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) a[c] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < NK; ++ks)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                a[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.f[ks][c], q.f[ks][c], a[c], 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = (a[0][e] + a[1][e]) + (a[2][e] + a[3][e]);
    }
    // the lane's share of the row's sum
    using L = float;
    __device__ static __forceinline__ L no_sum() { return 0.f; }
    __device__ static __forceinline__ float total(L l) { return quad_sum(l); }
    __device__ static __forceinline__ void weights(P &w, const float (&p)[NS]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w.f[e] = p[e];
    }
    __device__ static __forceinline__ void add(L &l, const P &w) { l += (w.f[0] + w.f[1]) + (w.f[2] + w.f[3]); }
    // As in bf16, but weights are not rounded: a row's reference moves when the four of one of
    // its lanes add up to more than 1 (or to no number).
    static constexpr int kLift = -10;
    struct Mark {};
    __device__ static __forceinline__ Mark mark(const L &) { return Mark(); }
    using Peak = float;
    __device__ static __forceinline__ Peak peak(const P &w) { return (w.f[0] + w.f[1]) + (w.f[2] + w.f[3]); }
    __device__ static __forceinline__ bool above(Peak k, Mark) { return !(k <= 1.f); }
    // lanes: those that are above
    __device__ static __forceinline__ bool moves(uint64_t lanes, int i, float, const L &) {
        const uint32_t x = (uint32_t)lanes | (uint32_t)(lanes >> 32);
        return ((x | x >> 16) >> i & 1) != 0;
    }
    __device__ static __forceinline__ bool finite(const V &v) {
        bool ok = true;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int d = 0; d < NT; ++d) ok &= (__float_as_uint(v.r[e][d / 4][d % 4]) & 0x7f800000u) != 0x7f800000u;
        return ok;
    }
    template <int RT>
    __device__ static __forceinline__ void accumulate_key(const V &v, const P (&w)[RT], f32x4 (&o)[RT][NT], int c,
                                                          const bool (&sees)[RT], int g) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float a = key_of(e, g) == c ? v.r[e][t / 4][t % 4] : 0.f;
                    const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x4f32(a, w[rt].f[e], o[rt][t], 0, 0, 0);
                    o[rt][t] = sees[rt] ? x : o[rt][t];
                }
    }
    template <int RT>
    __device__ static __forceinline__ void accumulate(const V &v, const P (&w)[RT], f32x4 (&o)[RT][NT]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.r[e][t / 4][t % 4], w[rt].f[e], o[rt][t], 0, 0, 0);
    }
    __device__ static __forceinline__ void put4(void *row, int d, float a, float b, float c, float e) {
        *(f32x4 *)((float *)row + d) = (f32x4){a, b, c, e};
    }
};

}  // namespace dev
}  // namespace kvr
