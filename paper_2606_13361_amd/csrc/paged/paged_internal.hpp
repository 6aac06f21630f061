// paged_internal.hpp -- launch parameters shared by the host entry points of the
// paged cache (paged_api.hip) and its kernels (rows.hip, decode.hip).
#pragma once

#include "kvr_internal.hpp"

namespace kvr {

// Rows [token][head] of an array, strides in elements
struct RowsAt {
    void *p;
    int64_t token, head;
};

// kvr_paged_append and kvr_qk_norm_rope.  A token's rows: n_q query, n_k key, n_v value rows.
struct RowsParams {
    RowsAt q, k, v;          // in
    RowsAt qo, ko;           // out (ko: rows to rows only)
    const void *qn, *kn;     // norm weights [D], or null
    float eps;
    const float *cs;         // rotary table, or null
    int64_t n_pos;
    const int32_t *pos;      // positions of the tokens, or null
    int64_t pos0;            // rows to rows, pos null: token t is at pos0 + t
    // pages (kp null: rows to rows)
    unsigned char *kp, *vp;
    int64_t page_bytes;      // between pages
    const int32_t *table, *cu, *len;
    int32_t n_pages, page_size, max_pages, n_seq;
    int64_t n_tok;
    int32_t n_q, n_k, n_v;
    int32_t tokens;          // of a wave, one after the other, at most 64
    int32_t parts;           // waves that share a token's rows
    int32_t part_rows;       // rows of one of them
};
constexpr int kRowWaves = 4;       // of a workgroup
hipError_t launch_rows(const RowsParams &p, int head_dim, int dtype, int64_t grid, hipStream_t s);

// kvr_paged_decode
struct DecodeParams {
    RowsAt q;                // n tokens, n_q_heads
    void *out;               // [n][n_q_heads][D]
    const unsigned char *kp, *vp;
    int64_t page_bytes;
    const int32_t *table, *len;
    float *ws;               // records, then the segments' workgroups
    int32_t n, n_new, max_len;
    int32_t n_pages, page_size, max_pages;
    int32_t n_q_heads, n_kv_heads, group;
    int32_t tiles;           // of 16 (32) query rows of a kv head
    int32_t rows;            // of a record
    int32_t grid;            // workgroups that share the units
    int32_t stream_units;    // units from which keys and values are loaded with the non-temporal hint (0: never)
    int32_t waves;           // of a workgroup
    int32_t merge_rows;      // query rows of a workgroup that joins records, 1 or 4
    int32_t alone;           // a workgroup takes one sequence and head, nothing is joined
    uint32_t part_shift;     // 16-row parts of a page, as a divisor: (part * part_mul) >> part_shift
    uint64_t part_mul;
    float half_scale_log2;   // the scale in log2, of half a score: twice as large
    float lift, unlift;      // factor of the weights in the second product, a power of two, and 1 / lift
};
// keys of a wave's stage: a unit of work is one for each of the workgroup's 1 or 4 waves
constexpr int kStageKeys = 32, kStageKeysF32 = 16;
hipError_t launch_decode(const DecodeParams &p, int head_dim, int dtype, hipStream_t s);

}  // namespace kvr
