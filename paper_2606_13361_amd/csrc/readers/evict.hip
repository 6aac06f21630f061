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
//           8192 of 32768 rows (67 MB): 26.4 us, of which the copy is 7 and the search about
//           14: weights 1.6, keys 1, histogram 2.6, its bin 1.3, the bin's keys 2.2 and
//           their ranks 1.1, counts and places 2.5.  945 of 3798: 8.4 us, 512 of 1024: 6.2 us.
//   evict_select_kernel, evict_copy_kernel (longer caches)  one workgroup per kv head
//           reads the weights again for each histogram and writes the list of kept
//           rows; the copy is a launch of its own.  8192 of 40000 rows: 34 + 13 us, of 131072:
//           96 + 14 us.
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

// Sum of x over the threads before this one, and of all threads.  Callers have a barrier
// between the last use of tmp and this one.
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
    if ((threadIdx.x & 63) == 63) tmp[wave] = v;
    __syncthreads();
    uint32_t base = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NWAVES; ++w) {
        const uint32_t t = tmp[w];
        base += w < wave ? t : 0u;
        all += t;
    }
    total = all;
    return base + v - x;
}

template <int BITS>
struct Search {
    __attribute__((aligned(16))) uint32_t hist[1 << BITS];
    __attribute__((aligned(16))) uint32_t few[kFew];
    uint32_t rank[kFew];
    uint32_t tmp[NWAVES];
    uint32_t found[3], n_few, zeros;
};

template <int BITS, int SBITS>
__device__ __forceinline__ void clear(Search<SBITS> &s) {
    constexpr int n = (1 << BITS) / 4;
#pragma unroll
    for (int b = threadIdx.x; b < n; b += THREADS) ((u32x4 *)s.hist)[b] = (u32x4){0, 0, 0, 0};
}

// Before find(), apart from it: the weights may be on their way meanwhile
template <int BITS>
__device__ __forceinline__ void prepare(Search<BITS> &s) {
    clear<BITS>(s);
    if (threadIdx.x < kFew) {
        s.few[threadIdx.x] = kNoRow;
        s.rank[threadIdx.x] = 0;
    }
    if (threadIdx.x == 0) s.n_few = s.zeros = 0;
    __syncthreads();
}

// Histogram (cleared) of bits `shift` .. `shift` + BITS - 1 of the keys with among(key); then
// the bin where the count from the top reaches `need`: its bits into T, what is left to
// take of its keys into `need`, and how many they are.  If all of them are fewer than
// `need`, that many, and `need` and T as they were.
template <int BITS, int SBITS, class AMONG, class EACH>
__device__ __forceinline__ uint32_t narrow(Search<SBITS> &s, int shift, uint32_t &T, uint32_t &need, AMONG among, EACH each) {
    constexpr uint32_t bins = 1u << BITS;
    constexpr int PER = bins > THREADS ? bins / THREADS : 1;
    each([&](uint32_t k) {
        if (among(k)) atomicAdd(&s.hist[(k >> shift) & (bins - 1)], 1u);
    });
    __syncthreads();
    uint32_t h[PER], sum = 0;
    if constexpr (PER >= 4) {
        const u32x4 *at = (const u32x4 *)(s.hist + bins - PER * (threadIdx.x + 1));
#pragma unroll
        for (int c = 0; c < PER; c += 4) {
            const u32x4 x = at[c / 4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[PER - 1 - c - e] = x[e];
        }
    } else {
        h[0] = threadIdx.x < bins ? s.hist[bins - 1 - threadIdx.x] : 0u;
    }
#pragma unroll
    for (int c = 0; c < PER; ++c) sum += h[c];
    uint32_t all;
    uint32_t before = scan(sum, s.tmp, all);
    if (all < need) {
        __syncthreads();      // the histogram is read
        return all;
    }
    if (before < need && before + sum >= need) {      // one thread
#pragma unroll
        for (int c = 0; c < PER; ++c) {
            if (before < need && before + h[c] >= need) {
                s.found[0] = bins - 1 - (threadIdx.x * PER + c);
                s.found[1] = need - before;
                s.found[2] = h[c];
            }
            before += h[c];
        }
    }
    __syncthreads();
    T |= s.found[0] << shift;
    need = s.found[1];
    return s.found[2];
}

// The pick-th largest key T (pick > 0; keys of no row apart), how many of the keys equal to
// it are taken, and whether these are all.  each(f) calls f(key) for the thread's keys,
// all lanes of a wave together.  Zeros, the one weight that many rows share, would all add
// to one bin: the weights above them are counted first, zeros and those below only if
// that is not enough.
template <int BITS, class EACH>
__device__ __forceinline__ uint32_t find(Search<BITS> &s, uint32_t pick, uint32_t &need, bool &all, EACH each) {
    constexpr int TOP = 32 - BITS, HALF = TOP / 2;
    uint32_t T = 0;
    need = pick;
    uint32_t n = narrow<BITS>(s, TOP, T, need, [](uint32_t k) { return k > kZero; }, each);
    if (n < need) {
        need -= n;
        uint32_t zeros = 0;
        each([&](uint32_t k) { zeros += __popcll(__ballot(k == kZero)); });
        if ((threadIdx.x & 63) == 0) atomicAdd(&s.zeros, zeros);
        clear<BITS>(s);
        __syncthreads();
        if (s.zeros >= need) {
            all = s.zeros == need;
            return kZero;
        }
        need -= s.zeros;
        n = narrow<BITS>(s, TOP, T, need, [](uint32_t k) { return k < kZero && k != kNoRow; }, each);
    }
    if (n > kFew) {
        clear<HALF>(s);
        __syncthreads();
        narrow<HALF>(s, HALF, T, need, [=](uint32_t k) { return k >> TOP == T >> TOP; }, each);
        clear<HALF>(s);
        __syncthreads();
        n = narrow<HALF>(s, 0, T, need, [=](uint32_t k) { return k >> HALF == T >> HALF; }, each);
        all = n == need;
        return T;
    }
    each([&](uint32_t k) {
        if (k >> TOP == T >> TOP && k != kZero) {      // (the least weights share zero's bin)
            const uint32_t at = atomicAdd(&s.n_few, 1u);
            if (at < kFew) s.few[at] = k;      // always, unless the weights change during the call
        }
    });
    __syncthreads();
    // the keys above a key (low half) and equal to it (high half), by four threads
    const uint32_t c = threadIdx.x % kFew;
    const uint32_t k = s.few[c];
    if (c < n) {
        uint32_t above = 0, equal = 0;
        for (uint32_t x = threadIdx.x / kFew * 16; x < n; x += THREADS / kFew * 16) {      // (behind the last: no row's key)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const u32x4 f = ((const u32x4 *)s.few)[x / 4 + y];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    above += f[e] > k;
                    equal += f[e] == k;
                }
            }
        }
        atomicAdd(&s.rank[c], above | equal << 16);
    }
    __syncthreads();
    if (threadIdx.x < n) {
        const uint32_t above = s.rank[c] & 0xffff, equal = s.rank[c] >> 16;
        if (above < need && above + equal >= need) {      // the same from every thread with this key
            s.found[0] = k;
            s.found[1] = need - above;
            s.found[2] = equal;
        }
    }
    __syncthreads();
    need = s.found[1];
    all = s.found[2] == need;
    return s.found[0];
}

__device__ __forceinline__ uint32_t lanes_before(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// Whether this is lane i, without a comparison
__device__ __forceinline__ bool lane_is(int i) { return __builtin_amdgcn_inverse_ballot_w64(1ull << i); }

// A thread's keys: those of rows j0 + threadIdx.x + THREADS i, so that blocks of 64 rows,
// in order, are those of wave 0, wave 1, ... for i = 0, then for i = 1, ...
template <int PER>
struct Keys {
    uint32_t k[PER];
    __device__ __forceinline__ void load(const EvictParams &p, const float *w, uint32_t j0) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            k[i] = __float_as_uint(w[min(j0 + THREADS * i + threadIdx.x, (uint32_t)p.L - 1)]);
    }
    __device__ __forceinline__ void make(const EvictParams &p, uint32_t j0) {
        const uint32_t lane = threadIdx.x & 63, b0 = j0 + 64 * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) most = max(most, k[i]);
        if (__ballot(most > 0x7f800000u)) {      // a sign or no number
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float x = __uint_as_float(k[i]);
                k[i] = x != x ? kNan : key_of(x + 0.f);
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) k[i] |= 0x80000000u;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t b = b0 + THREADS * i, first = p.n_first, last = p.L - p.n_last;
            if (b < first || b + 64 > last) {      // one of the block may be no candidate
                const uint32_t j = b + lane;
                if (j < first || j >= last) k[i] = j < (uint32_t)p.L ? kStays : kNoRow;
            }
        }
    }
};

// Keys above T (low half) and equal to it (high half), up to 2^15 each: lane i gets the
// counts of the wave's block i, and of all blocks before it.  all: nothing equal is to be
// told apart, T is the largest key that goes.
template <int PER>
__device__ __forceinline__ void count(Keys<PER> &keys, uint32_t T, bool all, uint32_t *counts, uint32_t *tmp, uint32_t &mine,
                                      uint32_t &before, uint32_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    mine = 0;
    if (all) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t a = __popcll(__ballot(keys.k[i] > T));
            mine = lane_is(i) ? a : mine;
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t a = __popcll(__ballot(keys.k[i] > T)), e = __popcll(__ballot(keys.k[i] == T)), ae = a | e << 16;
            mine = lane_is(i) ? ae : mine;
        }
    }
    if (lane < PER) counts[lane * NWAVES + wave] = mine;
    __syncthreads();
    const bool one = threadIdx.x < PER * NWAVES;
    const uint32_t b = scan(one ? counts[threadIdx.x] : 0u, tmp, total);
    if (one) counts[threadIdx.x] = b;
    __syncthreads();
    before = lane < PER ? counts[lane * NWAVES + wave] : 0u;
}

// put(place, row) for the kept rows with places r0 .. r0 + n - 1.  above, equal: keys before
// those that count() saw
template <int PER, class PUT>
__device__ __forceinline__ void place(Keys<PER> &keys, uint32_t T, uint32_t need, uint32_t j0, uint32_t mine, uint32_t before,
                                      uint32_t above, uint32_t equal, int r0, int n, PUT put) {
    const int lane = threadIdx.x & 63;
    const uint32_t a0 = above + (before & 0xffff), e0 = equal + (before >> 16);
    const int first = (int)(a0 + min(e0, need)), last = (int)(a0 + (mine & 0xffff) + min(e0 + (mine >> 16), need));
    const uint64_t blocks = __ballot(lane < PER && last > r0 && first < r0 + n && last > first);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (!(blocks >> i & 1)) continue;
        asm volatile("" : "+v"(keys.k[i]));      // compared anew: 4 PER registers of masks are more than there are
        const uint64_t ma = __ballot(keys.k[i] > T), me = __ballot(keys.k[i] == T);
        const uint32_t eq = __builtin_amdgcn_readlane(e0, i) + lanes_before(me);
        const int at = (int)(__builtin_amdgcn_readlane(a0, i) + lanes_before(ma) + min(eq, need)) - r0;
        if ((keys.k[i] > T || (keys.k[i] == T && eq < need)) && at >= 0 && at < n) put(at, (int)(j0 + THREADS * i + threadIdx.x));
    }
}

constexpr int LIST = 2048;      // kept rows that a workgroup copies at a time

// PER: keys per thread
template <int PER, int BITS>
__global__ __launch_bounds__(THREADS) void evict_kernel(const EvictParams p) {
    __shared__ Search<BITS> s;
    __shared__ uint32_t counts[PER * NWAVES];
    __shared__ int32_t list[LIST];
    const int hd = blockIdx.x % p.n_kv_heads, part = blockIdx.x / p.n_kv_heads;
    const float *w = p.weight + (int64_t)hd * p.cap;
    Keys<PER> keys;
    keys.load(p, w, 0);
    prepare(s);
    keys.make(p, 0);
    uint32_t need, mine, before, total;
    bool all;
    uint32_t T = find<BITS>(s, (uint32_t)p.n_keep, need, all, [&](auto f) {
#pragma unroll
        for (int i = 0; i < PER; ++i) f(keys.k[i]);
    });
    if (all) --T, need = 0;
    count(keys, T, all, counts, s.tmp, mine, before, total);
    const int share = (p.n_keep + p.parts - 1) / p.parts;
    const int r_end = min(p.n_keep, (part + 1) * share);
    for (int r0 = part * share; r0 < r_end; r0 += LIST) {
        const int n = min(LIST, r_end - r0);
        place(keys, T, need, 0, mine, before, 0, 0, r0, n, [&](int at, int j) { list[at] = j; });
        __syncthreads();
        for (int r = threadIdx.x; r < n; r += THREADS) {
            if (p.index) p.index[(int64_t)hd * p.n_keep + r0 + r] = list[r];
            if (p.weight_out) p.weight_out[(int64_t)hd * p.cap_out + r0 + r] = w[list[r]];
        }
        // the rows, 16 bytes a thread, several in flight
        constexpr int BATCH = 4;
        const int chunks = n * p.row_chunks;
        for (int x0 = threadIdx.x; x0 < chunks; x0 += BATCH * THREADS) {
            u32x4 k[BATCH], v[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int x = min(x0 + b * THREADS, chunks - 1);
                const int r = x >> p.chunk_bits;
                const int64_t src = (((int64_t)hd * p.cap + list[r]) << p.chunk_bits) + (x & (p.row_chunks - 1));
                k[b] = ((const u32x4 *)p.kc)[src];
                v[b] = ((const u32x4 *)p.vc)[src];
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int x = x0 + b * THREADS;
                if (x >= chunks) break;
                const int64_t dst = (((int64_t)hd * p.cap_out + r0) << p.chunk_bits) + x;
                ((u32x4 *)p.ko)[dst] = k[b];
                ((u32x4 *)p.vo)[dst] = v[b];
            }
        }
        __syncthreads();      // the list is read
    }
}

__global__ __launch_bounds__(THREADS) void evict_select_kernel(const EvictParams p) {
    constexpr int PER = 8;
    __shared__ Search<14> s;
    __shared__ uint32_t counts[PER * NWAVES];
    const int hd = blockIdx.x;
    const float *w = p.weight + (int64_t)hd * p.cap;
    int32_t *out = p.list + (int64_t)hd * p.n_keep;
    prepare(s);
    Keys<PER> keys;
    uint32_t need;
    bool all;
    uint32_t T = find<14>(s, (uint32_t)p.n_keep, need, all, [&](auto f) {
        for (uint32_t j0 = 0; j0 < (uint32_t)p.L; j0 += PER * THREADS) {
            keys.load(p, w, j0);
            keys.make(p, j0);
#pragma unroll
            for (int i = 0; i < PER; ++i) f(keys.k[i]);
        }
    });
    if (all) --T, need = 0;
    uint32_t above = 0, equal = 0;
    for (uint32_t j0 = 0; j0 < (uint32_t)p.L; j0 += PER * THREADS) {
        uint32_t mine, before, total;
        keys.load(p, w, j0);
        keys.make(p, j0);
        count(keys, T, all, counts, s.tmp, mine, before, total);
        place(keys, T, need, j0, mine, before, above, equal, 0, p.n_keep, [&](int at, int j) { out[at] = j; });
        above += total & 0xffff;
        equal += total >> 16;
    }
}

__global__ __launch_bounds__(256) void evict_copy_kernel(const EvictParams p) {
    const int64_t total = (int64_t)p.n_kv_heads * p.n_keep * p.row_chunks;
    for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
        const int c = (int)(x & (p.row_chunks - 1));
        const int64_t r = x >> p.chunk_bits;
        const int hd = (int)(r / p.n_keep);
        const int64_t to = r - (int64_t)hd * p.n_keep;
        const int32_t from = (int32_t)min((uint32_t)p.list[r], (uint32_t)p.L - 1);      // (also if the weights change during the call)
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
        // as few keys a thread as hold them: 1024 rows take 6.2, 7.7 and 14.6 us with 2, 8 and 32,
        // 3798 rows 8.4 and 15.2 with 8 and 32
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
