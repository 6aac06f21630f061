// evict.hip -- a smaller cache of the rows with the most accumulated weight.
//
// Of rows 0 .. L - 1 of a kv head the first n_first and the last n_last stay, and of
// those between (the candidates) the `pick` ones with the largest weight, the lower row
// where weights are equal.  Weights are compared as integers: key_of() maps a float to
// an unsigned number of the same order.
//   select  one workgroup per kv head: the pick-th largest key by a radix search over
//           its bytes, then the kept rows' indices in ascending order
//   copy    the kept rows, their weights and indices
#include "readers_internal.hpp"

namespace kvr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 1024;
constexpr int NWAVES = THREADS / 64;

// Order of floats as unsigned numbers; -0 as 0, and a weight that is no number above
// all others, so that its row is kept and seen
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    if ((u & 0x7fffffffu) == 0) return 0x80000000u;
    return (u >> 31) ? ~u : u | 0x80000000u;
}

// Sum of x over the threads before this one, and of all threads
__device__ __forceinline__ uint32_t scan(uint32_t x, uint32_t *tmp, uint32_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t v = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(v, d);
        if (lane >= d) v += y;
    }
    __syncthreads();      // tmp of the scan before is read
    if (lane == 63) tmp[wave] = v;
    __syncthreads();
    uint32_t base = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NWAVES; ++w) {
        if (w < wave) base += tmp[w];
        all += tmp[w];
    }
    total = all;
    return base + v - x;
}

__global__ __launch_bounds__(THREADS) void evict_select_kernel(const EvictParams p) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t tmp[NWAVES];
    __shared__ uint32_t found[2];
    const int hd = blockIdx.x;
    const float *w = p.weight + (int64_t)hd * p.cap;
    int32_t *out = p.list + (int64_t)hd * p.n_keep;
    const int lo = p.n_first, hi = p.L - p.n_last;      // the candidates
    uint32_t pick = (uint32_t)(p.n_keep - p.n_first - p.n_last);
    // largest key T with at least `pick` candidates >= T, byte by byte from the top
    uint32_t T = 0, need = pick;      // need: of those equal to T in the bytes so far
    if (pick > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) hist[threadIdx.x] = 0;
            __syncthreads();
            for (int j = lo + threadIdx.x; j < hi; j += THREADS) {
                const uint32_t k = key_of(w[j]);
                if (shift == 24 || (k >> (shift + 8)) == (T >> (shift + 8))) atomicAdd(&hist[k >> shift & 255], 1u);
            }
            __syncthreads();
            // bin b is the one where the count from the top passes `need`
            const uint32_t mine = threadIdx.x < 256 ? hist[255 - threadIdx.x] : 0u;
            uint32_t all;
            const uint32_t before = scan(mine, tmp, all);
            if (threadIdx.x < 256 && before < need && before + mine >= need) {
                found[0] = 255 - threadIdx.x;
                found[1] = need - before;
            }
            __syncthreads();
            T |= found[0] << shift;
            need = found[1];
            __syncthreads();
        }
    }
    for (int j = threadIdx.x; j < lo; j += THREADS) out[j] = j;
    // candidates above T, and the first `need` of those equal to it
    uint32_t above = 0, equal = 0;
    for (int j0 = lo; j0 < hi; j0 += THREADS) {
        const int j = j0 + threadIdx.x;
        const uint32_t k = j < hi ? key_of(w[j]) : 0u;
        const bool in = j < hi && pick > 0;
        const uint32_t a = in && k > T, e = in && k == T;
        uint32_t ta, te;
        const uint32_t ca = above + scan(a, tmp, ta), ce = equal + scan(e, tmp, te);
        if (a || (e && ce < need)) out[lo + ca + min(ce, need)] = j;
        above += ta;
        equal += te;
    }
    for (int j = threadIdx.x; j < p.n_last; j += THREADS) out[lo + pick + j] = hi + j;
}

__global__ __launch_bounds__(256) void evict_copy_kernel(const EvictParams p) {
    const int64_t total = (int64_t)p.n_kv_heads * p.n_keep * p.row_chunks;
    for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
        const int c = (int)(x % p.row_chunks);
        const int64_t r = x / p.row_chunks;
        const int hd = (int)(r / p.n_keep);
        const int64_t to = r % p.n_keep;
        const int32_t from = p.list[r];
        const int64_t s = ((int64_t)hd * p.cap + from) * p.row_chunks + c;
        const int64_t d = ((int64_t)hd * p.cap_out + to) * p.row_chunks + c;
        const u32x4 k = ((const u32x4 *)p.kc)[s], v = ((const u32x4 *)p.vc)[s];
        ((u32x4 *)p.ko)[d] = k;
        ((u32x4 *)p.vo)[d] = v;
        if (c == 0) {
            if (p.index) p.index[r] = from;
            if (p.weight_out) p.weight_out[(int64_t)hd * p.cap_out + to] = p.weight[(int64_t)hd * p.cap + from];
        }
    }
}

}  // namespace

hipError_t launch_evict(const EvictParams &p, hipStream_t s) {
    hipLaunchKernelGGL(evict_select_kernel, dim3(p.n_kv_heads), dim3(THREADS), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t blocks = ((int64_t)p.n_kv_heads * p.n_keep * p.row_chunks + 255) / 256;
    hipLaunchKernelGGL(evict_copy_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace kvr
