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
// rows round them, so that a key has the same bits from each.  A workgroup takes a few
// tokens: their places are worked out by a thread each while the first rows are on
// their way.
//
// HBM bounds it.
#include "attn_common.hpp"
#include "paged/paged_internal.hpp"

namespace kvr {
namespace {

using namespace dev;

constexpr int NT = 256;
constexpr int BATCH = 2;      // rows of a thread that are on their way at once

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

template <bool PAGED>
__device__ __forceinline__ Place place_of(const RowsParams &p, int64_t t, const int32_t *cu_lds, int row_bytes) {
    Place o;
    o.slot = 0;
    o.pos = p.pos ? (int64_t)p.pos[t] : p.pos0 + t;
    if constexpr (PAGED) {
        const Place none = {-1, 0};
        int r = (int)t;
        int64_t first = t;
        if (p.cu) {
            // sequences that end at t or before
            int lo = 0, hi = p.n_seq;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                const int32_t end = p.n_seq <= NT ? cu_lds[mid + 1] : p.cu[mid + 1];
                if (end <= t) lo = mid + 1; else hi = mid;
            }
            r = lo;
            if (r == p.n_seq) return none;
            first = p.n_seq <= NT ? cu_lds[r] : p.cu[r];
            if (first < 0 || first > t) return none;
        }
        const int32_t len = p.len[r];
        if (len < 0) return none;
        const int64_t row = (int64_t)len + (t - first);
        if (row >= (int64_t)p.max_pages * p.page_size) return none;
        const int32_t at = (int32_t)row / p.page_size;
        const int32_t page = p.table[(int64_t)r * p.max_pages + at];
        if ((uint32_t)page >= (uint32_t)p.n_pages) return none;
        if (!p.pos) o.pos = row;
        o.slot = page * p.page_bytes + (int64_t)((int32_t)row - at * p.page_size) * row_bytes;
    }
    if (p.cs && (o.pos < 0 || o.pos >= p.n_pos)) o.slot = -1;
    return o;
}

template <class T, int D, bool PAGED>
__global__ __launch_bounds__(NT) void rows_kernel(const RowsParams p) {
    using EL = Elt<T>;
    constexpr int N = EL::N, LANES = D / (2 * N), ROWS = NT / LANES, ROWB = D * EL::BYTES;
    __shared__ Place places[kRowTokens];
    __shared__ int32_t cu_lds[NT + 1];
    const int tid = threadIdx.x;
    const int c = chunk_of<LANES>(tid % LANES);
    const int per = p.n_q + p.n_k + p.n_v;
    const int64_t t0 = (int64_t)blockIdx.x * p.tokens;
    const int nt = (int)min((int64_t)p.tokens, p.n_tok - t0);
    const int total = nt * per;

    Chunk x[BATCH];
    auto load = [&](int r0) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int r = r0 + b * ROWS;
            if (r >= total) continue;
            const int tk = (int)__umulhi((uint32_t)r, p.by_rows);
            int h = r - tk * per;
            const RowsAt &a = h < p.n_q ? p.q : h < p.n_q + p.n_k ? p.k : p.v;
            h -= h < p.n_q ? 0 : h < p.n_q + p.n_k ? p.n_q : p.n_q + p.n_k;
            const unsigned char *s = (const unsigned char *)a.p + ((t0 + tk) * a.token + h * a.head) * EL::BYTES + 16 * c;
            x[b].lo = *(const u32x4 *)s;
            x[b].hi = *(const u32x4 *)(s + ROWB / 2);
        }
    };
    load(tid / LANES);
    if constexpr (PAGED) {
        if (p.cu && p.n_seq <= NT) {
            for (int j = tid; j <= p.n_seq; j += NT) cu_lds[j] = p.cu[j];
            __syncthreads();
        }
    }
    if (tid < nt) places[tid] = place_of<PAGED>(p, t0 + tid, cu_lds, ROWB);
    __syncthreads();

    for (int r0 = tid / LANES; r0 < total; r0 += BATCH * ROWS) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int r = r0 + b * ROWS;
            if (r >= total) continue;      // all lanes of a row alike
            const int tk = (int)__umulhi((uint32_t)r, p.by_rows);
            int h = r - tk * per;
            const Place at = places[tk];
            if (at.slot < 0) continue;
            const bool is_q = h < p.n_q, is_v = h >= p.n_q + p.n_k;
            h -= is_q ? 0 : is_v ? p.n_q + p.n_k : p.n_q;
            if (!is_v) {
                const void *nw = is_q ? p.qn : p.kn;
                const float *cs = p.cs ? p.cs + at.pos * D + 2 * N * c : nullptr;
                if (nw) {
                    float a[N], e[N], s[N], wa[N], we[N];
                    EL::widen(x[b].lo, a);
                    EL::widen(x[b].hi, e);
                    EL::widen(*(const u32x4 *)((const unsigned char *)nw + 16 * c), wa);
                    EL::widen(*(const u32x4 *)((const unsigned char *)nw + ROWB / 2 + 16 * c), we);
#pragma unroll
                    for (int j = 0; j < N; ++j) s[j] = pair_sq(a[j], e[j]);
                    const float inv = 1.0f / sqrtf(row_sum<LANES, N>(s) / (float)D + p.eps);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        a[j] = a[j] * inv * wa[j];
                        e[j] = e[j] * inv * we[j];
                    }
                    if (cs) {
#pragma unroll
                        for (int j = 0; j < N; ++j) {
                            const float y = a[j], z = e[j];
                            rope_rot(y, z, cs[2 * j], cs[2 * j + 1], a[j], e[j]);
                        }
                    }
                    x[b].lo = EL::narrow(a);
                    x[b].hi = EL::narrow(e);
                } else if (cs) {
                    EL::rotate(x[b], cs);
                }
            }
            unsigned char *d;
            if (PAGED && !is_q)
                d = (is_v ? p.vp : p.kp) + at.slot + (int64_t)h * p.page_size * ROWB;
            else
                d = (unsigned char *)(is_q ? p.qo.p : p.ko.p) +
                    ((t0 + tk) * (is_q ? p.qo.token : p.ko.token) + h * (is_q ? p.qo.head : p.ko.head)) * EL::BYTES;
            *(u32x4 *)(d + 16 * c) = x[b].lo;
            *(u32x4 *)(d + ROWB / 2 + 16 * c) = x[b].hi;
        }
        load(r0 + BATCH * ROWS);
    }
}

template <class T>
hipError_t launch_t(const RowsParams &p, int head_dim, int64_t grid, hipStream_t s) {
    const dim3 g((unsigned)grid), b(NT);
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
