// rows.hip -- rows of new tokens on their way into a paged cache (kvr_paged_append)
// or to rows of their own (kvr_qk_norm_rope): the norm of each query and key head, the
// rotation at the token's position, one rounding; values are copied.
//
//   y = R(pos) (x / sqrt(mean(x^2) + eps) * w)
//
// A thread holds 16 bytes of a row's first half and the 16 bytes of their partners, so
// the rotation needs no exchange and a row's sum of squares goes over the D elt / 32
// lanes next to each other that share it.  The sums are added in the order of every
// kernel that normalizes heads (pair_sq), and values are rounded as those that rotate
// rows round them, so that a key has the same bits from each.
//
// A wave takes rows of one token at a time: its cosines and sines are read once, and up to
// BATCH rows of a lane are on their way at once.  The places of the wave's tokens are worked
// out by a lane each, while the first rows are on their way.
//
// HBM bounds it (a copy with the same store hint reaches 5.6 to 5.8 TB/s).  bf16, 32 / 8 heads of 128, read and written:
//   32768 tokens' norms and rotation 123 us, 5.6 TB/s
//   32 prompts, 32767 tokens, into pages 168 us, 4.8 TB/s; 3774 tokens' keys and values 9.2 us, 3.6 TB/s
//   one token 3.8 us: launch, length, page, rotation
// Waits for rows that are not on their way while others are worked out are filled by other waves: 3
// rows a lane (4 waves a SIMD) and 6 (3 waves) took 181 and 198 us for the prompts, 66 and 74 us for
// 32768 tokens' keys and values.  Written rows bypass the caches as far as a hint does that: 3774 tokens
// 10.9 us without, the norms 136.  A wave for the rows of one token instead of a workgroup for a few
// tokens' (cosines read for each row, places behind a barrier): the prompts 218 -> 170, the norms 196 -> 127.
#include "attn_common.hpp"
#include "paged/paged_internal.hpp"

namespace kvr {
namespace {

using namespace dev;

constexpr int WAVES = kRowWaves;
constexpr int BATCH = 3;      // rows of a lane that are on their way at once

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Chunk {
    u32x4 lo, hi;
};

template <class E>
struct Elt {
    static constexpr int BYTES = 2, N = 8;
    __device__ static __forceinline__ void widen(const u32x4 &w, float (&x)[N]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = E::lo(w[j]);
            x[2 * j + 1] = E::hi(w[j]);
        }
    }
    __device__ static __forceinline__ u32x4 narrow(const float (&x)[N]) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = E::pack2_f32(x[2 * j], x[2 * j + 1]);
        return w;
    }
    __device__ static __forceinline__ void rotate(Chunk &c, const float *cs) { rope_rot8<E>(c.lo, c.hi, cs); }
};
template <>
struct Elt<float> {
    static constexpr int BYTES = 4, N = 4;
    __device__ static __forceinline__ void widen(const u32x4 &w, float (&x)[N]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[j]);
    }
    __device__ static __forceinline__ u32x4 narrow(const float (&x)[N]) {
        return (u32x4){__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
    __device__ static __forceinline__ void rotate(Chunk &c, const float *cs) {
        float a[N], b[N], y[N], z[N];
        widen(c.lo, a);
        widen(c.hi, b);
#pragma unroll
        for (int j = 0; j < N; ++j) rope_rot(a[j], b[j], cs[2 * j], cs[2 * j + 1], y[j], z[j]);
        c.lo = narrow(y);
        c.hi = narrow(z);
    }
};

// Chunk of a lane among the LANES of its row.  Their bits are reversed, so that the sums' order
// (pairs that are D / 4, D / 8, ... apart first) goes over lanes 1, 2, 4, ... apart.
template <int LANES>
__device__ __forceinline__ int chunk_of(int lane) {
    int c = 0;
#pragma unroll
    for (int b = 1; b < LANES; b <<= 1) c = c << 1 | ((lane & b) ? 1 : 0);
    return c;
}

// The value of the lane B away (B = 4 and 8: of a lane whose value that lane has too)
template <int B>
__device__ __forceinline__ float from_lane(float x) {
    constexpr int ctrl = B == 1 ? 0xB1 : B == 2 ? 0x4E : B == 4 ? 0x141 : 0x140;      // quad_perm, row_half_mirror, row_mirror
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xf, 0xf, false));
}

// The row's sum, from each lane's N pairs
template <int LANES, int N>
__device__ __forceinline__ float row_sum(float (&s)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
        s[j] += from_lane<1>(s[j]);
        s[j] += from_lane<2>(s[j]);
        if constexpr (LANES >= 8) s[j] += from_lane<4>(s[j]);
        if constexpr (LANES >= 16) s[j] += from_lane<8>(s[j]);
    }
#pragma unroll
    for (int b = N / 2; b > 0; b >>= 1)
#pragma unroll
        for (int j = 0; j < b; ++j) s[j] += s[j + b];
    return s[0];
}

// Where a token goes: its position, and its slot in the pages in bytes
struct Place {
    int64_t slot;      // < 0: the token takes no part
    int64_t pos;
};
__device__ __forceinline__ int64_t lane_of(int64_t x, int l) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)x, l), hi = __builtin_amdgcn_readlane((int)(x >> 32), l);
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// How many of cu[1 .. n] are at most t (they are in order): 64 of them at a time
__device__ __forceinline__ int ended(const int32_t *cu, int n, int64_t t, int lane) {
    int lo = 0, cnt = n;
    while (cnt > 0) {
        const int step = (cnt + 63) / 64;
        const int at = (lane + 1) * step;
        const int c = __popcll(__ballot(at <= cnt && cu[lo + min(at, cnt)] <= t));      // whole steps that ended
        lo += c * step;
        cnt = min(step - 1, cnt - c * step);
    }
    return lo;
}

// The places of tokens t0 .. t0 + n - 1 (at most 64), one a lane
template <bool PAGED>
__device__ __forceinline__ Place places_of(const RowsParams &p, int64_t t0, int n, int row_bytes, int lane) {
    const int64_t t = t0 + lane;
    Place o;
    o.slot = -1;
    o.pos = 0;
    int r = lane < n ? 0 : p.n_seq;
    if constexpr (PAGED) {
        if (p.cu) {
            const int r0 = ended(p.cu, p.n_seq, t0, lane);
            const int64_t end = r0 + 1 + lane <= p.n_seq ? (int64_t)p.cu[r0 + 1 + lane] : (int64_t)1 << 40;
            for (int j = 0; j < n; ++j) {
                int c = r0 + __popcll(__ballot(end <= t0 + j));
                if (c == r0 + 64) c = ended(p.cu, p.n_seq, t0 + j, lane);      // (a row of sequences without tokens)
                if (lane == j) r = c;
            }
        } else if (lane < n) {
            r = (int)t;
        }
    }
    if (lane >= n || (PAGED && r >= p.n_seq)) return o;
    o.pos = p.pos ? (int64_t)p.pos[t] : p.pos0 + t;
    int64_t slot = 0;
    if constexpr (PAGED) {
        const int64_t first = p.cu ? p.cu[r] : t;
        const int32_t len = p.len[r];
        if (first < 0 || first > t || len < 0) return o;
        const int64_t row = (int64_t)len + (t - first);
        if (row >= (int64_t)p.max_pages * p.page_size) return o;
        const int32_t at = (int32_t)row / p.page_size;
        const int32_t page = p.table[(int64_t)r * p.max_pages + at];
        if ((uint32_t)page >= (uint32_t)p.n_pages) return o;
        if (!p.pos) o.pos = row;
        slot = page * p.page_bytes + (int64_t)((int32_t)row - at * p.page_size) * row_bytes;
    }
    if (!p.cs || (o.pos >= 0 && o.pos < p.n_pos)) o.slot = slot;
    return o;
}

template <class T, int D, bool PAGED>
__global__ __launch_bounds__(64 * WAVES) void rows_kernel(const RowsParams p) {
    using EL = Elt<T>;
    constexpr int N = EL::N, LANES = D / (2 * N), ROWS = 64 / LANES, ROWB = D * EL::BYTES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = chunk_of<LANES>(lane % LANES);
    const int per = p.n_q + p.n_k + p.n_v, n_qk = p.n_q + p.n_k;
    const uint32_t id = blockIdx.x * WAVES + wave, group = id / (uint32_t)p.parts;
    const int64_t t0 = (int64_t)group * p.tokens, t1 = min(t0 + p.tokens, p.n_tok);
    const int first = (int)(id - group * p.parts) * p.part_rows, last = min(first + p.part_rows, per);

    // weights of the lane's elements
    u32x4 w[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned char *n = (const unsigned char *)(i ? p.kn : p.qn) + 16 * c;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            w[i][h] = (i ? p.kn : p.qn) ? *(const u32x4 *)(n + h * (ROWB / 2)) : (u32x4){0u, 0u, 0u, 0u};
    }

    Place at;
    for (int64_t t = t0; t < t1; ++t) {
        int64_t slot;
        float cs[2 * N];
        for (int r0 = first; r0 < last; r0 += BATCH * ROWS) {
            Chunk x[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (r0 + b * ROWS >= last) break;
                const int r = min(r0 + b * ROWS + lane / LANES, last - 1);
                const RowsAt &a = r < p.n_q ? p.q : r < n_qk ? p.k : p.v;
                const int h = r - (r < p.n_q ? 0 : r < n_qk ? p.n_q : n_qk);
                const unsigned char *s = (const unsigned char *)a.p + (t * a.token + h * a.head) * EL::BYTES + 16 * c;
                x[b].lo = *(const u32x4 *)s;
                x[b].hi = *(const u32x4 *)(s + ROWB / 2);
            }
            if (r0 == first) {
                if (t == t0) at = places_of<PAGED>(p, t0, (int)(t1 - t0), ROWB, lane);
                slot = lane_of(at.slot, (int)(t - t0));
                if (slot < 0) break;
                if (p.cs) {
                    const float *s = p.cs + lane_of(at.pos, (int)(t - t0)) * D + 2 * N * c;
#pragma unroll
                    for (int j = 0; j < 2 * N; ++j) cs[j] = s[j];
                }
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (r0 + b * ROWS >= last) break;
                const int r = r0 + b * ROWS + lane / LANES;
                const bool is_q = r < p.n_q, is_v = r >= n_qk;
                const bool norm = !is_v && (is_q ? p.qn : p.kn);
                Chunk y = x[b];
                if (p.cs && __ballot(!is_v && !norm)) {
                    EL::rotate(y, cs);
                    if (norm || is_v) y = x[b];
                }
                if (__ballot(norm)) {
                    float a[N], e[N], s[N], wa[N], we[N];
                    EL::widen(x[b].lo, a);
                    EL::widen(x[b].hi, e);
                    EL::widen(is_q ? w[0][0] : w[1][0], wa);
                    EL::widen(is_q ? w[0][1] : w[1][1], we);
#pragma unroll
                    for (int j = 0; j < N; ++j) s[j] = pair_sq(a[j], e[j]);
                    const float inv = 1.0f / sqrtf(row_sum<LANES, N>(s) / (float)D + p.eps);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        a[j] = a[j] * inv * wa[j];
                        e[j] = e[j] * inv * we[j];
                    }
                    if (p.cs) {
#pragma unroll
                        for (int j = 0; j < N; ++j) {
                            const float f = a[j], g = e[j];
                            rope_rot(f, g, cs[2 * j], cs[2 * j + 1], a[j], e[j]);
                        }
                    }
                    const u32x4 lo = EL::narrow(a), hi = EL::narrow(e);
                    if (norm) { y.lo = lo; y.hi = hi; }
                }
                if (r >= last) continue;
                const int h = r - (is_q ? 0 : is_v ? n_qk : p.n_q);
                unsigned char *d;
                if (PAGED && !is_q)
                    d = (is_v ? p.vp : p.kp) + slot + (int64_t)h * p.page_size * ROWB;
                else
                    d = (unsigned char *)(is_q ? p.qo.p : p.ko.p) +
                        (t * (is_q ? p.qo.token : p.ko.token) + h * (is_q ? p.qo.head : p.ko.head)) * EL::BYTES;
                __builtin_nontemporal_store(y.lo, (u32x4 *)(d + 16 * c));
                __builtin_nontemporal_store(y.hi, (u32x4 *)(d + ROWB / 2 + 16 * c));
            }
        }
    }
}

template <class T>
hipError_t launch_t(const RowsParams &p, int head_dim, int64_t grid, hipStream_t s) {
    const dim3 g((unsigned)grid), b(64 * WAVES);
    if (p.kp) {
        if (head_dim == 128) hipLaunchKernelGGL((rows_kernel<T, 128, true>), g, b, 0, s, p);
        else hipLaunchKernelGGL((rows_kernel<T, 64, true>), g, b, 0, s, p);
    } else {
        if (head_dim == 128) hipLaunchKernelGGL((rows_kernel<T, 128, false>), g, b, 0, s, p);
        else hipLaunchKernelGGL((rows_kernel<T, 64, false>), g, b, 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rows(const RowsParams &p, int head_dim, int dtype, int64_t grid, hipStream_t s) {
    if (dtype == KVR_F32) return launch_t<float>(p, head_dim, grid, s);
    return dtype == KVR_F16 ? launch_t<F16>(p, head_dim, grid, s) : launch_t<Bf16>(p, head_dim, grid, s);
}

}  // namespace kvr
