// readers_internal.hpp -- launch parameters shared by the host entry points
// (readers_api.hip) and the kernels for many readers of one cached document.  Not
// part of the public ABI (include/kvr.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvr.h"

namespace kvr {

// Many readers of one prefix, each with cached rows of its own (shared.hip)
struct SharedParams {
    const void *q;          // [n][S][n_q_heads][D]
    const void *kn, *vn;    // new rows [n][S][n_kv_heads][D]
    const void *kc, *vc;    // prefix [n_kv_heads][cap][D]
    void *kt, *vt;          // the readers' own rows [n][n_kv_heads][tcap][D]
    const int32_t *len;     // device [n]: cached own rows
    void *out;
    float *ws;              // partials: O [nrec][rows][D], then (m, l) [nrec][rows][2]; rows as in out
    const float *rope;      // table, or null
    int64_t cap, tcap, L, pos0;
    int64_t chunk;          // prefix keys per split
    int64_t rows;           // n S n_q_heads
    uint32_t oct_own, oct_new, oct_all;   // groups of eight blocks: where own and new items begin, all
    float scale_log2;
    int32_t n, S, n_q_heads, n_kv_heads, group;
    int32_t append;
    int32_t np, nt, nrec;   // splits of the prefix and of own rows; np + nt + 1, the last for the new rows
    int32_t p_tiles, t_tiles;   // row tiles of a kv head over the prefix, of a reader's kv head over its own rows
};
// pw, ow: the ways of prefix and own items, ow <= pw.  1, 2: the four waves share 16 or 32
// query rows and split the keys (2: fp32 only); kByRows + 1, + 2: each wave has 16 or 32
// rows of its own (16-bit only; own items: + 1).  pw kAlone: one launch, a workgroup for
// each reader and kv head, at most 16 rows each
constexpr int kByRows = 10, kAlone = 0;
hipError_t launch_shared(const SharedParams &p, int head_dim, int dtype, int pw, int ow, hipStream_t s);

// Attention weight received by each cached row (weigh.hip)
struct WeighParams {
    const void *q;        // [S][n_q_heads][D]
    const void *kn;       // new keys [S][n_kv_heads][D]
    const void *kc;       // [n_kv_heads][cap][D]
    float *weight;        // [n_kv_heads][cap], added to
    float2 *ws;           // (M, l) [n_kv_heads][nsplit][rows], rows = S group
    float *norm;          // [n_kv_heads][rows] behind them where a launch of its own joins the splits, or null
    int64_t cap, L;
    int32_t S, n_q_heads, n_kv_heads, group;
    int32_t nsplit, chunk;   // key splits of the first pass, of `chunk` stages each
    float scale_log2;
};
// way of the first pass: 1, 2: the four waves share that many 16-row tiles and split the keys
// (2: fp32 only); kByRows + 2, + 4: each wave has that many of its own (16-bit only).  held: key
// stages that a wave of the second pass holds, 1 or 2 (fp32 only)
hipError_t launch_weigh(const WeighParams &p, int head_dim, int dtype, int way, int held, hipStream_t s);

// The cache of the rows with the most weight (evict.hip)
struct EvictParams {
    const void *kc, *vc;     // [n_kv_heads][cap][row]
    const float *weight;     // [n_kv_heads][cap]
    void *ko, *vo;           // [n_kv_heads][cap_out][row]
    float *weight_out;       // [n_kv_heads][cap_out], or null
    int32_t *index;          // [n_kv_heads][n_keep], or null
    int32_t *list;           // L > kHeldRows: workspace, the kept rows [n_kv_heads][n_keep]
    int64_t cap, cap_out;
    int32_t L, n_first, n_last, n_keep;
    int32_t n_kv_heads;
    int32_t parts;                    // L <= kHeldRows: workgroups per kv head
    int32_t row_chunks, chunk_bits;   // 16-byte chunks per row, 2^chunk_bits
};
constexpr int64_t kHeldRows = 32768;   // longest cache whose weights a workgroup holds in registers
hipError_t launch_evict(const EvictParams &p, hipStream_t s);

}  // namespace kvr
