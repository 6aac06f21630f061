// weigh.hip -- the attention weight that each cached row receives, summed over the
// query rows and heads of its kv head:
//
//   weight[g][j] += sum_(i, h of g) 2^(c q_ih . k_j - M_ih) / l_ih,   c = scale log2(e)
//
// A row's normalizer (M, l) covers all its keys, so there are two passes over the
// keys, both matrix products of K and Q^T (attn_direct.hpp: K straight to registers):
//   stats  a wave holds 16 RT query rows and walks its share of the keys; each lane
//          keeps the running maximum and sum of its own keys, joined at the end
//   sums   a wave holds 64 keys and walks all query rows of its kv head; the weights
//          of its keys add up in registers and are added to the buffer once
// Every sum has a fixed order and every buffer element one writer: results are
// reproducible bit for bit.
#include <type_traits>

#include "attn_direct.hpp"
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
        const bool nw = keys.is_new(t);
        const int c0 = (int)keys.first(t);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float s[OP::NS];
            OP::scores(kk, q[rt], s);
            if (nw || n < OP::KEYS) mask<OP>(s, nw ? min(n - 1, tok[rt] - c0) : n - 1, g);
            float mx = s[0];
#pragma unroll
            for (int e = 1; e < OP::NS; ++e) mx = fmaxf(mx, s[e]);
            const float mn = fmaxf(m[rt], mx * c2);
            l[rt] *= __builtin_amdgcn_exp2f(m[rt] - mn);
            m[rt] = mn;
#pragma unroll
            for (int e = 0; e < OP::NS; ++e) l[rt] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c2, -mn));
        }
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

constexpr int ROWS_AT_ONCE = 1024;      // normalizers held in LDS
constexpr int HELD = 2;                 // stages of keys that a wave holds

template <class OP>
__global__ __launch_bounds__(256) void weigh_sum_kernel(const WeighParams p) {
    __shared__ float2 norm[ROWS_AT_ONCE];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hd = blockIdx.x % p.n_kv_heads;
    const int G = p.group, rows = p.S * G;
    const Keys<OP> keys(p, hd);
    const int n_all = keys.n_pre + (p.S + OP::KEYS - 1) / OP::KEYS;
    const int t0 = ((int)(blockIdx.x / p.n_kv_heads) * WAVES + wave) * HELD;
    const float c2 = p.scale_log2;
    typename OP::K k[HELD];
    float acc[HELD][OP::NS];
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        keys.load(k[h], t0 + h, t0 + h < n_all ? keys.count(t0 + h) : 0, i, g);
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) acc[h][e] = 0.f;
    }
    for (int r0 = 0; r0 < rows; r0 += ROWS_AT_ONCE) {
        const int nr = min(rows - r0, ROWS_AT_ONCE);
        if (r0) __syncthreads();
        for (int r = threadIdx.x; r < nr; r += 256) {
            const float2 *src = p.ws + (int64_t)hd * p.nsplit * rows + r0 + r;
            float M = -1e30f, sum = 0.f;
            for (int s = 0; s < p.nsplit; ++s) {
                const float2 v = src[(int64_t)s * rows];
                const float mn = fmaxf(M, v.x);
                sum = sum * __builtin_amdgcn_exp2f(M - mn) + v.y * __builtin_amdgcn_exp2f(v.x - mn);
                M = mn;
            }
            norm[r] = make_float2(M, 1.f / sum);
        }
        __syncthreads();
        for (int rr = 0; rr < nr; rr += 16) {
            const int r = rr + i;
            const bool valid = r < nr;
            const int at = r0 + min(r, nr - 1);
            const int tok = at / G;
            typename OP::Q q;
            OP::load_q(q, (const unsigned char *)p.q + ((int64_t)tok * p.n_q_heads + hd * G + (at - tok * G)) * OP::ROWB, g);
            const float2 nm = norm[min(r, nr - 1)];
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                float s[OP::NS];
                OP::scores(k[h], q, s);
                const int t = t0 + h;
                if (keys.is_new(t)) mask<OP>(s, tok - (int)keys.first(t), g);
#pragma unroll
                for (int e = 0; e < OP::NS; ++e) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c2, -nm.x)) * nm.y;
                    acc[h][e] += valid ? w : 0.f;
                }
            }
        }
    }
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        const int t = t0 + h;
        const int n = t < n_all ? keys.count(t) : 0;
        const int64_t first = (keys.is_new(t) ? p.L : 0) + keys.first(t);
#pragma unroll
        for (int e = 0; e < OP::NS; ++e) {
            float x = acc[h][e];
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) x += __shfl_xor(x, d);
            const int key = OP::key_of(e, g);
            if (i == e && key < n) p.weight[(int64_t)hd * p.cap + first + key] += x;
        }
    }
}

template <class OP>
hipError_t launch_op(const WeighParams &p, int rt, hipStream_t s) {
    const int rows = p.S * p.group;
    const unsigned tiles = (unsigned)((rows + 16 * rt - 1) / (16 * rt));
    const dim3 grid(tiles * p.nsplit * p.n_kv_heads);
    if (rt == 1) hipLaunchKernelGGL((weigh_stats_kernel<OP, 1>), grid, dim3(256), 0, s, p);
    else if (rt == 2) hipLaunchKernelGGL((weigh_stats_kernel<OP, 2>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((weigh_stats_kernel<OP, 4>), grid, dim3(256), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t stages = (p.L + OP::KEYS - 1) / OP::KEYS + (p.S + OP::KEYS - 1) / OP::KEYS;
    const unsigned wgs = (unsigned)((stages + WAVES * HELD - 1) / (WAVES * HELD));
    hipLaunchKernelGGL(weigh_sum_kernel<OP>, dim3(wgs * p.n_kv_heads), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_weigh(const WeighParams &p, int head_dim, int dtype, int rt, hipStream_t s) {
    if (dtype == KVR_F32) return head_dim == 128 ? launch_op<Op32<128>>(p, rt, s) : launch_op<Op32<64>>(p, rt, s);
    if (dtype == KVR_F16) return head_dim == 128 ? launch_op<Op16<F16, 128>>(p, rt, s) : launch_op<Op16<F16, 64>>(p, rt, s);
    return head_dim == 128 ? launch_op<Op16<Bf16, 128>>(p, rt, s) : launch_op<Op16<Bf16, 64>>(p, rt, s);
}

}  // namespace kvr
