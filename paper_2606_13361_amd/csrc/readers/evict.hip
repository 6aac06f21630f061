// evict.hip -- a smaller cache of the rows with the most accumulated weight.
//
// Of rows 0 .. L - 1 of a kv head the first n_first and the last n_last stay, and of
// those between the ones with the largest weight, the lower row where weights are equal.
// Weights are compared as integers: key_of() maps a float to an unsigned number of the
// same order, and the rows that stay anyway have the largest key of all.  With T the
// n_keep-th largest key and `need` the number of rows with exactly that key that are
// still to be taken, row j is kept if its key is above T, or if it is T and fewer than
// `need` rows before it have that key; its place is the number of kept rows before it.
//
// T comes from a histogram of the keys' top bits in LDS: the bin where the count from
// the top reaches n_keep holds it.  Of the bin's keys, up to kFew are ranked against each
// other; more of them go through histograms of the bits below, in two rounds.
//
//   evict_kernel (up to kHeldRows rows)  one launch.  Every workgroup of a kv head holds
//           all its keys in registers, finds T by itself, and copies its share of the
//           kept rows: no second launch, no list in memory.
//   evict_select_kernel, evict_copy_kernel (longer caches)  one workgroup per kv head
//           reads the weights again for each histogram and writes the list of kept
//           rows; the copy is a launch of its own.
#include "readers_internal.hpp"

namespace kvr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 1024;
constexpr int NWAVES = THREADS / 64;
constexpr uint32_t kZero = 0x80000000u;      // the key of weight 0
constexpr uint32_t kFew = 256;

// Order of floats as unsigned numbers, by parts: the order itself (-0 is added to 0 by
// the caller), a weight that is no number above all others, so that its row is kept and
// seen, above it the rows that stay anyway, below all (-infinity is 0x007fffff) no row.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
constexpr uint32_t kNan = 0xfffffffeu, kStays = 0xffffffffu, kNoRow = 0u;

// Sum of x over the threads before this one, and of all threads
__device__ __forceinline__ uint32_t scan(uint32_t x, uint32_t *tmp, uint32_t &total) {
    const int wave = threadIdx.x >> 6;
    // inclusive over the wave's lanes by data-parallel moves: within rows of 16 lanes,
    // then the rows' totals to the rows behind them
    uint32_t v = x;
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast 15, 31
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
    __syncthreads();      // tmp of the scan before is read
    if ((threadIdx.x & 63) == 63) tmp[wave] = v;
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

template <int BITS>
struct Search {
    uint32_t hist[1 << BITS];
    uint32_t few[kFew];
    uint32_t tmp[NWAVES];
    uint32_t found[3], n_few;
};

// Histogram of the keys' bits `shift` .. `shift` + BITS - 1, of those that agree with T above
// them; then the bin where the count from the top reaches `need`: its bits into T, what
// is left to take of its keys into `need`, and how many they are.
template <int BITS, int SBITS, bool TOP, class EACH>
__device__ __forceinline__ uint32_t narrow(Search<SBITS> &s, int shift, uint32_t &T, uint32_t &need, EACH each) {
    constexpr uint32_t bins = 1u << BITS;
    constexpr int PER = bins > THREADS ? bins / THREADS : 1;
    for (uint32_t b = threadIdx.x; b < bins; b += THREADS) s.hist[b] = 0;
    __syncthreads();
    // zeros are the one weight that many rows share: counted by wave, not one by one
    uint32_t zeros = 0;
    each([&](uint32_t k) {
        const bool mine = TOP ? k != kNoRow : k != kNoRow && k >> (shift + BITS) == T >> (shift + BITS);
        zeros += __popcll(__ballot(mine && k == kZero));
        if (mine && k != kZero) atomicAdd(&s.hist[(k >> shift) & (bins - 1)], 1u);
    });
    if ((threadIdx.x & 63) == 0 && zeros) atomicAdd(&s.hist[(kZero >> shift) & (bins - 1)], zeros);
    __syncthreads();
    uint32_t h[PER], sum = 0;
#pragma unroll
    for (int c = 0; c < PER; ++c) {
        const uint32_t b = threadIdx.x * PER + c;
        h[c] = b < bins ? s.hist[bins - 1 - b] : 0u;
        sum += h[c];
    }
    uint32_t all;
    uint32_t before = scan(sum, s.tmp, all);
#pragma unroll
    for (int c = 0; c < PER; ++c) {
        if (before < need && before + h[c] >= need) {
            s.found[0] = bins - 1 - (threadIdx.x * PER + c);
            s.found[1] = need - before;
            s.found[2] = h[c];
        }
        before += h[c];
    }
    __syncthreads();
    T |= s.found[0] << shift;
    need = s.found[1];
    return s.found[2];
}

// The pick-th largest key T (pick > 0), and how many of the keys equal to it are taken.
// each(f) calls f(key) for the thread's keys, all lanes of a wave together.
template <int BITS, class EACH>
__device__ __forceinline__ uint32_t find(Search<BITS> &s, uint32_t pick, uint32_t &need, EACH each) {
    uint32_t T = 0;
    need = pick;
    if (threadIdx.x == 0) s.n_few = 0;
    const uint32_t n = narrow<BITS, BITS, true>(s, 32 - BITS, T, need, each);
    if (n > kFew) {
        constexpr int HALF = (32 - BITS) / 2;
        narrow<HALF, BITS, false>(s, HALF, T, need, each);
        narrow<HALF, BITS, false>(s, 0, T, need, each);
        return T;
    }
    each([&](uint32_t k) {
        if (k != kNoRow && k >> (32 - BITS) == T >> (32 - BITS)) s.few[atomicAdd(&s.n_few, 1u)] = k;
    });
    __syncthreads();
    if (threadIdx.x < n) {
        const uint32_t k = s.few[threadIdx.x];
        uint32_t above = 0, equal = 0;
        for (uint32_t x = 0; x < n; ++x) {
            above += s.few[x] > k;
            equal += s.few[x] == k;
        }
        if (above < need && above + equal >= need) {      // the same from every thread with this key
            s.found[0] = k;
            s.found[1] = need - above;
        }
    }
    __syncthreads();
    need = s.found[1];
    return s.found[0];
}

__device__ __forceinline__ uint32_t lanes_before(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

constexpr int LIST = 2048;      // kept rows that a workgroup copies at a time

// PER: keys per thread.  Wave w holds rows 64 PER w .. 64 PER (w + 1) - 1, its lanes
// side by side: a wave counts its kept rows with ballots, and only the waves that hold
// rows of the workgroup's share place them.
template <int PER, int BITS>
__global__ __launch_bounds__(THREADS) void evict_kernel(const EvictParams p) {
    __shared__ Search<BITS> s;
    __shared__ uint32_t count[NWAVES][2];
    __shared__ int32_t list[LIST];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int hd = blockIdx.x % p.n_kv_heads, part = blockIdx.x / p.n_kv_heads;
    const float *w = p.weight + (int64_t)hd * p.cap;
    const int w0 = __builtin_amdgcn_readfirstlane(wave) * 64 * PER, j0 = w0 + lane;
    float x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = w[min(j0 + 64 * i, p.L - 1)];
    uint32_t key[PER];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        odd |= x[i] != x[i];
        key[i] = key_of(x[i] + 0.f);
    }
    if (__ballot(odd)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = x[i] != x[i] ? kNan : key[i];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = w0 + 64 * i, j = b + lane;
        if (b < p.n_first || b + 64 > p.L - p.n_last) {      // one of the wave's 64 may be no candidate
            if (j < p.n_first || j >= p.L - p.n_last) key[i] = kStays;
            if (j >= p.L) key[i] = kNoRow;
        }
    }
    uint32_t need;
    const uint32_t T = find<BITS>(s, (uint32_t)p.n_keep, need, [&](auto f) {
#pragma unroll
        for (int i = 0; i < PER; ++i) f(key[i]);
    });
    // keys above T, and equal to it, of each wave
    uint32_t a = 0, e = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        a += __popcll(__ballot(key[i] > T));
        e += __popcll(__ballot(key[i] == T));
    }
    if (lane == 0) {
        count[wave][0] = a;
        count[wave][1] = e;
    }
    __syncthreads();
    uint32_t a0 = 0, e0 = 0;      // of the waves before
    for (int x = 0; x < wave; ++x) {
        a0 += count[x][0];
        e0 += count[x][1];
    }
    const uint32_t first = a0 + min(e0, need), last = a0 + a + min(e0 + e, need);      // places of this wave's rows
    const int share = (p.n_keep + p.parts - 1) / p.parts;
    const int r_end = min(p.n_keep, (part + 1) * share);
    for (int r0 = part * share; r0 < r_end; r0 += LIST) {
        const int n = min(LIST, r_end - r0);
        if ((int)last > r0 && (int)first < r0 + n) {
            uint32_t ca = a0, ce = e0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                asm volatile("" : "+v"(key[i]));      // compared anew: 4 PER registers of masks are more than there are
                const uint64_t ma = __ballot(key[i] > T), me = __ballot(key[i] == T);
                const uint32_t eq = ce + lanes_before(me);
                const int at = (int)(ca + lanes_before(ma) + min(eq, need)) - r0;
                if ((key[i] > T || (key[i] == T && eq < need)) && at >= 0 && at < n) list[at] = j0 + 64 * i;
                ca += __popcll(ma);
                ce += __popcll(me);
            }
        }
        __syncthreads();
        // the rows, 16 bytes a thread, several in flight
        constexpr int BATCH = 4;
        const int total = n * p.row_chunks;
        for (int x0 = threadIdx.x; x0 < total; x0 += BATCH * THREADS) {
            u32x4 k[BATCH], v[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int x = min(x0 + b * THREADS, total - 1);
                const int r = x >> p.chunk_bits;
                const int64_t src = (((int64_t)hd * p.cap + list[r]) << p.chunk_bits) + (x & (p.row_chunks - 1));
                k[b] = ((const u32x4 *)p.kc)[src];
                v[b] = ((const u32x4 *)p.vc)[src];
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int x = x0 + b * THREADS;
                if (x >= total) break;
                const int64_t dst = (((int64_t)hd * p.cap_out + r0) << p.chunk_bits) + x;
                ((u32x4 *)p.ko)[dst] = k[b];
                ((u32x4 *)p.vo)[dst] = v[b];
            }
        }
        for (int r = threadIdx.x; r < n; r += THREADS) {
            if (p.index) p.index[(int64_t)hd * p.n_keep + r0 + r] = list[r];
            if (p.weight_out) p.weight_out[(int64_t)hd * p.cap_out + r0 + r] = w[list[r]];
        }
        __syncthreads();      // the list is read
    }
}

__global__ __launch_bounds__(THREADS) void evict_select_kernel(const EvictParams p) {
    __shared__ Search<14> s;
    const int hd = blockIdx.x;
    const float *w = p.weight + (int64_t)hd * p.cap;
    int32_t *out = p.list + (int64_t)hd * p.n_keep;
    const int64_t L = p.L;
    auto key = [&](int64_t j) {
        const float x = w[min(j, L - 1)];
        if (j >= L) return kNoRow;
        if (j < p.n_first || j >= L - p.n_last) return kStays;
        return x != x ? kNan : key_of(x + 0.f);
    };
    uint32_t need;
    const uint32_t T = find<14>(s, (uint32_t)p.n_keep, need, [&](auto f) {
        for (int64_t j0 = 0; j0 < L; j0 += THREADS) f(key(j0 + threadIdx.x));
    });
    uint32_t above = 0, equal = 0;
    for (int64_t j0 = 0; j0 < L; j0 += THREADS) {
        const int64_t j = j0 + threadIdx.x;
        const uint32_t k = key(j), a = k > T, e = k == T;
        uint32_t ta, te;
        const uint32_t ca = above + scan(a, s.tmp, ta), ce = equal + scan(e, s.tmp, te);
        if (a || (e && ce < need)) out[ca + min(ce, need)] = (int)j;
        above += ta;
        equal += te;
    }
}

__global__ __launch_bounds__(256) void evict_copy_kernel(const EvictParams p) {
    const int64_t total = (int64_t)p.n_kv_heads * p.n_keep * p.row_chunks;
    for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
        const int c = (int)(x & (p.row_chunks - 1));
        const int64_t r = x >> p.chunk_bits;
        const int hd = (int)(r / p.n_keep);
        const int64_t to = r - (int64_t)hd * p.n_keep;
        const int32_t from = p.list[r];
        const int64_t src = (((int64_t)hd * p.cap + from) << p.chunk_bits) + c;
        const int64_t dst = (((int64_t)hd * p.cap_out + to) << p.chunk_bits) + c;
        const u32x4 k = ((const u32x4 *)p.kc)[src], v = ((const u32x4 *)p.vc)[src];
        ((u32x4 *)p.ko)[dst] = k;
        ((u32x4 *)p.vo)[dst] = v;
        if (c == 0) {
            if (p.index) p.index[r] = from;
            if (p.weight_out) p.weight_out[(int64_t)hd * p.cap_out + to] = p.weight[(int64_t)hd * p.cap + from];
        }
    }
}

}  // namespace

hipError_t launch_evict(const EvictParams &p, hipStream_t s) {
    if (p.L <= kHeldRows) {
        const dim3 grid((unsigned)(p.n_kv_heads * p.parts)), block(THREADS);
        if (p.L <= 2 * THREADS) hipLaunchKernelGGL((evict_kernel<2, 12>), grid, block, 0, s, p);
        else if (p.L <= 8 * THREADS) hipLaunchKernelGGL((evict_kernel<8, 12>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((evict_kernel<32, 14>), grid, block, 0, s, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(evict_select_kernel, dim3(p.n_kv_heads), dim3(THREADS), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t blocks = ((int64_t)p.n_kv_heads * p.n_keep * p.row_chunks + 255) / 256;
    hipLaunchKernelGGL(evict_copy_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace kvr
