// attn_ring.hpp -- stages of 32 K (or V, or Q) rows that the four waves of a workgroup
// share in LDS, 16-bit elements.  Shared by shared.hip and weigh.hip.
//
// Fragments loaded straight from memory (attn_direct.hpp) take 16 rows' lines at each
// instruction, about 75 clocks a kilobyte and compute unit; where several waves need
// the same rows, loading them once in whole rows costs the caches a quarter of the
// lines and a wave's reads come from LDS.
//
// Row r of a stage lies at r ROWB, its 16-byte chunk c in slot c ^ swz(r).  LDS gives 256
// bytes a clock.  K and Q: 16 lanes at a time read a chunk of 16 different rows, which swz
// spreads over 16 places of a 256-byte line.  V, transposed: 32 lanes at a time read two
// neighbouring chunks of eight rows, four consecutive ones from each of two 16-lane groups.
#pragma once

#include "attn_direct.hpp"

namespace kvr {
namespace dev {

template <class E, int D>
struct Ring16 {
    using OP = Op16<E, D>;
    static constexpr int ROWB = D * 2, CH = D / 8, NK = D / 32, NT = D / 16;
    static constexpr int KEYS = 32, HALF = KEYS * ROWB;      // one operand's rows of a stage
    static constexpr int LOADS = HALF / 4096;                // wave-wide 1 KB loads of a wave for them

    template <bool IS_V>
    __device__ static __forceinline__ int swz(int row) {
        const int half = ((row >> 2) ^ (row >> 3)) & 1;      // of the groups' rows 4 g ..
        if (IS_V) return D == 128 ? (row & 3) << 1 | half << 3 : (row & 2) | half << 2;
        return D == 128 ? row & 15 : (row >> 1) & 7;
    }
    // This wave's quarter of the rows [0, n) (n > 0) of stride_b bytes from base into the
    // stage at lds; rows past the last repeat it.  A key there is masked by its index; a value
    // has weight 0, and shared.hip clears it, as the last row's may be infinite.
    template <bool IS_V>
    __device__ static __forceinline__ void load(uint64_t base, uint32_t stride_b, int n, const unsigned char *lds, int wave,
                                                int lane) {
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int at = (wave * LOADS + x) * 1024;
            const int row = at / ROWB + lane / CH;
            const uint32_t off = (uint32_t)min(row, n - 1) * stride_b + 16u * (uint32_t)((lane & (CH - 1)) ^ swz<IS_V>(row));
            dma16_s(base, off, lds + at);
        }
    }
    // The same of KEYS rows that follow each other: offsets that are the same for every stage
    template <bool IS_V>
    __device__ static __forceinline__ void load_all(uint64_t base, const unsigned char *lds, int wave, int lane) {
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int at = (wave * LOADS + x) * 1024;
            const int row = at / ROWB + lane / CH;
            dma16_s(base, (uint32_t)(row * ROWB) + 16u * (uint32_t)((lane & (CH - 1)) ^ swz<IS_V>(row)), lds + at);
        }
    }
    // lane (i, g)'s LDS offset of chunk g of row i (swz has a row's last four bits: the same
    // 16 rows further, at + 16 ROWB); chunk 4 ks + g lies at this ^ 64 ks
    __device__ static __forceinline__ uint32_t row_at(int i, int g) { return (uint32_t)(i * ROWB + 16 * (g ^ swz<false>(i))); }
    // what lane (i, g) passes to the transposing read of rows 4 g .. 4 g + 3, columns 0 .. 15;
    // columns 16 t .. at this ^ 32 t
    __device__ static __forceinline__ uint32_t col_at(int i, int g) {
        const int row = 4 * g + (i >> 2);
        return (uint32_t)(row * ROWB + 16 * (((i & 3) >> 1) ^ swz<true>(row)) + 8 * (i & 1));
    }
    // K (or Q) rows of a 16-row part as an operand
    __device__ static __forceinline__ u32x4 row_frag(const unsigned char *lds, uint32_t at, int part, int ks) {
        return *(const u32x4 *)(lds + part * 16 * ROWB + (at ^ (64u * ks)));
    }
    // V^T of columns 16 t .. as an operand: lane (i, g) holds column 16 t + i of the keys of
    // Op16::key_of
    __device__ static __forceinline__ u32x4 col_frag(const unsigned char *lds, uint32_t at, int t) {
        const unsigned char *a = lds + (at ^ (32u * t));
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)a));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(a + 16 * ROWB)));
        return (u32x4){lo[0], lo[1], hi[0], hi[1]};
    }
};

// This wave's LDS reads are done; then all waves' are
__device__ __forceinline__ void barrier_lds() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace dev
}  // namespace kvr
