// walk.hpp -- how decode.hip shares the work of a call out: the units of all sequences and heads, one after
// the other, cut into ranges, and a workgroup's walk over its range.
//
// Lengths are read from memory that the caller may write, more than once where a batch has more than 64
// sequences.  Lengths that change while the call runs give no sensible outputs, but every unit is one of
// a sequence of the batch: a range that finds no more of them ends.
#pragma once

#include "paged/paged_internal.hpp"

namespace kvr {
namespace {

// Rows of a sequence that its token sees; -1: the sequence takes no part
__device__ __forceinline__ int rows_of(const DecodeParams &p, int32_t len) {
    const int64_t n = (int64_t)len + p.n_new;
    return len >= 0 && n <= p.max_len ? (int)n : -1;
}
// Units of a sequence (of each of its heads): an empty one has one, which finds no keys
template <int UNIT>
__device__ __forceinline__ int units_of(int rows) {
    return rows < 0 ? 0 : rows == 0 ? 1 : (rows - 1) / UNIT + 1;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int lane_of(int x, int l) { return __builtin_amdgcn_readlane(x, l); }

// Inclusive sum over the lanes before
__device__ __forceinline__ int scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8: within 16 lanes
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // the sums of rows 0 and 2 to 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // of the first two to the others
    return x;
}

// `total` units cut into ranges of nearly one length, the longer ones first
struct Cut {
    int total, n, each, more;      // ranges; units of one; how many have one unit more
    __device__ __forceinline__ int start(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int range_of(int u) const {
        const int longer = more * (each + 1);
        return u < longer ? u / (each + 1) : more + (u - longer) / each;
    }
};

// Memory that no kernel of the call writes, read with scalar loads
template <class T>
__device__ __forceinline__ T scalar(const T *x) {
    return *(const __attribute__((address_space(4))) T *)(uintptr_t)x;
}

// A unit of one sequence and head, and the wave's stage of it
struct Unit {
    int r, hd;        // sequence; kv head and row tile
    int rows, units;  // of the sequence
    int u;
    int page, part;   // the stage's first part: entry of the page table, and which of the page's
    __device__ __forceinline__ bool last() const { return u + 1 == units; }
};

// The workgroup's units, one after the other
template <class OP, int WAVES>
struct Walk {
    static constexpr int UNIT = OP::KEYS * WAVES, PARTS = UNIT / 16;      // keys, and parts of 16, of a unit
    int heads, left;       // units behind the one returned last
    int lens_at, lens;     // rows_of 64 sequences, one a lane
    int page0, part0;      // of the wave's stage of a sequence's first unit
    int pages, parts;      // from one unit to the next

    __device__ __forceinline__ Walk(const DecodeParams &p, int wave) {
        heads = p.n_kv_heads * p.tiles;
        page_of(p, wave * OP::PARTS, page0, part0);
        page_of(p, PARTS, pages, parts);
    }
    __device__ __forceinline__ static void page_of(const DecodeParams &p, int part, int &page, int &rest) {
        page = (int)((part * p.part_mul) >> p.part_shift);
        rest = part - page * (p.page_size >> 4);
    }
    __device__ __forceinline__ void look(const DecodeParams &p, int r, int lane) {
        lens_at = r;
        lens = r + lane < p.n ? rows_of(p, p.len[r + lane]) : -1;
    }
    __device__ __forceinline__ int rows(const DecodeParams &p, int r, int lane) {
        if (r - lens_at >= 64) look(p, r, lane);
        return lane_of(lens, r - lens_at);
    }
    // The unit after b; false: there is none
    __device__ __forceinline__ bool next(const DecodeParams &p, Unit &b, int lane) {
        if (left <= 0) return false;
        --left;
        if (b.last()) {
            b.u = 0;
            b.page = page0;
            b.part = part0;
            if (++b.hd == heads) {
                b.hd = 0;
                do {
                    if (++b.r >= p.n) {      // (the lengths are not what they were)
                        left = 0;
                        return false;
                    }
                    b.rows = rows(p, b.r, lane);
                    b.units = units_of<UNIT>(b.rows);
                } while (b.units == 0);
            }
        } else {
            ++b.u;
            b.page += pages;
            b.part += parts;
            if (b.part >= p.page_size >> 4) {
                b.part -= p.page_size >> 4;
                ++b.page;
            }
        }
        return true;
    }
    // The workgroup's first unit, and the `at` of it among all; false: it has none.  The sequence is found
    // by sums over 64 groups of sequences, then over 64 groups of the right one's, ...
    __device__ __forceinline__ bool first(const DecodeParams &p, Unit &b, int &at, int wg, Cut &cut, int wave, int lane) {
        if (p.alone) {
            b.r = wg / heads;
            b.hd = wg - b.r * heads;
            b.rows = rows_of(p, scalar(p.len + b.r));
            b.units = units_of<UNIT>(b.rows);
            if (b.units == 0) return false;
            b.u = at = 0;
            b.page = page0;
            b.part = part0;
            left = b.units - 1;
            return true;
        }
        int lo = 0, cnt = p.n, want = 0, before = 0, mine, sum, step;
        for (bool top = true;; top = false) {
            step = (cnt + 63) / 64;
            mine = 0;
            if (step == 1) {
                look(p, lo, lane);
                mine = lane < cnt ? units_of<UNIT>(lens) : 0;
            } else {
                const int r0 = lo + lane * step, r1 = min(r0 + step, lo + cnt);
                for (int r = r0; r < r1; ++r) mine += units_of<UNIT>(rows_of(p, p.len[r]));
            }
            sum = scan(mine);
            if (top) {
                cut.total = lane_of(sum, 63) * heads;
                cut.n = min(p.grid, cut.total);
                if (wg >= cut.n) return false;
                cut.each = cut.total / cut.n;
                cut.more = cut.total - cut.each * cut.n;
                at = cut.start(wg);
                left = cut.start(wg + 1) - at - 1;
                want = at / heads;
            }
            const uint64_t over = __ballot(before + sum > want);
            if (over == 0) return false;      // (the lengths are not what they were)
            const int l = __builtin_ctzll(over);
            before += lane_of(sum, l) - lane_of(mine, l);
            const int start = lo + l * step;
            cnt = min(step, lo + cnt - start);
            lo = start;
            if (step == 1) break;
        }
        b.r = lo;
        b.rows = lane_of(lens, lo - lens_at);
        b.units = units_of<UNIT>(b.rows);
        const int rest = at - before * heads;
        b.hd = rest / b.units;
        b.u = rest - b.hd * b.units;
        page_of(p, (b.u * WAVES + wave) * OP::PARTS, b.page, b.part);
        return true;
    }
};

}  // namespace
}  // namespace kvr
