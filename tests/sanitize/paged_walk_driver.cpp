// Runs the device code that shares the units of kvr_paged_decode out (paged/walk.hpp) on the CPU: a wave is 64
// contexts that take turns and meet at each operation between lanes.  Checked: the workgroups' units are all units of the batch, each
// once and in order; and where lengths change behind the first unit, every unit is still one of a sequence of
// the batch, with rows, and a walk ends.
#include <stdint.h>
#include <stdio.h>
#include <string.h>
#include <ucontext.h>

#include <algorithm>
#include <functional>
#include <vector>

#include <hip/hip_runtime.h>

static ucontext_t g_wave, g_lanes[64];
static int g_lane_value[64], t_lane;
static bool g_done[64];
static std::function<void(int)> g_main;
static int g_bad = 0;
#define BAD(...) (++g_bad, fprintf(stderr, __VA_ARGS__), fputc('\n', stderr))

// Every lane goes on when all have come here
static void meet() {
    const int l = t_lane;
    swapcontext(&g_lanes[l], &g_wave);
}
static void lane_entry(int l) {
    g_main(l);
    g_done[l] = true;
}
static void run_wave(std::function<void(int)> f) {
    static std::vector<std::vector<char>> stacks(64, std::vector<char>(256 << 10));
    g_main = f;
    for (int l = 0; l < 64; ++l) {
        g_done[l] = false;
        getcontext(&g_lanes[l]);
        g_lanes[l].uc_stack.ss_sp = stacks[l].data();
        g_lanes[l].uc_stack.ss_size = stacks[l].size();
        g_lanes[l].uc_link = &g_wave;
        makecontext(&g_lanes[l], (void (*)())lane_entry, 1, l);
    }
    for (int left = 64; left > 0;) {
        left = 0;
        for (t_lane = 0; t_lane < 64; ++t_lane) {
            swapcontext(&g_wave, &g_lanes[t_lane]);
            left += !g_done[t_lane];
        }
        if (left != 0 && left != 64) {
            BAD("lanes go different ways");
            return;
        }
    }
}

template <class F>
static auto together(int x, F f) {
    g_lane_value[t_lane] = x;
    meet();
    const auto y = f();
    meet();
    return y;
}
static int lane_read(int x, int l) {
    return together(x, [&] { return g_lane_value[l]; });
}
// row_shr n: 0x110 + n; 0x142: lane 15 of the row before; 0x143: lane 31 for the rows behind.  Lanes without a source, or of rows
// that the mask leaves out, keep `old`
static int dpp(int old, int x, int ctrl, int row_mask) {
    return together(x, [&] {
        const int row = t_lane / 16;
        if (!(row_mask >> row & 1)) return old;
        if (ctrl > 0x110 && ctrl < 0x120) return t_lane % 16 < ctrl - 0x110 ? old : g_lane_value[t_lane - (ctrl - 0x110)];
        if (ctrl == 0x142) return row == 0 ? old : g_lane_value[16 * row - 1];
        return row < 2 ? old : g_lane_value[31];
    });
}
static uint64_t ballot(bool b) {
    return together(b, [] {
        uint64_t m = 0;
        for (int l = 0; l < 64; ++l) m |= (uint64_t)(g_lane_value[l] != 0) << l;
        return m;
    });
}
#define __builtin_amdgcn_readfirstlane(x) lane_read(x, 0)
#define __builtin_amdgcn_readlane(x, l) lane_read(x, l)
#define __builtin_amdgcn_update_dpp(old, x, ctrl, rows, banks, bound) dpp(old, x, ctrl, rows)
#define __ballot(x) ballot(x)
#define address_space(n) unused
using std::max;
using std::min;

#include "paged/walk.hpp"

using namespace kvr;

template <int K>
struct Op {
    static constexpr int KEYS = K, PARTS = K / 16;
};
struct At {
    int wg, r, hd, u;
};

// One workgroup's walk of a wave; `change` runs behind the first unit
template <class OP, int WAVES, class F>
static void walk(const DecodeParams &p, int wg, int wave, F change, std::vector<At> &units) {
    run_wave([&](int lane) {
        Walk<OP, WAVES> w(p, wave);
        Unit b;
        Cut cut;
        int at;
        if (!w.first(p, b, at, wg, cut, wave, lane)) return;
        for (;;) {
            meet();
            if (lane == 0) {
                if (b.r < 0 || b.r >= p.n || b.hd < 0 || b.hd >= w.heads || b.rows < 0 || b.rows > p.max_len || b.u < 0 || b.u >= b.units)
                    BAD("workgroup %d: unit %d of sequence %d of %d (%d rows), head %d", wg, b.u, b.r, p.n, b.rows, b.hd);
                const int part = (b.u * WAVES + wave) * OP::PARTS;
                if (b.page != part / (p.page_size / 16) || b.part != part % (p.page_size / 16)) BAD("page of a unit");
                units.push_back({wg, b.r, b.hd, b.u});
                if (units.size() == 1 || units[units.size() - 2].wg != wg) change();
            }
            meet();
            if (!w.next(p, b, lane)) return;
        }
    });
}

static uint64_t g_state = 88172645463325252ull;
static int rnd(int n) {
    g_state ^= g_state << 13; g_state ^= g_state >> 7; g_state ^= g_state << 17;
    return (int)(g_state % (uint64_t)n);
}

template <class OP, int WAVES>
static void one(int n, int longest, int ps, bool alone, bool changes) {
    std::vector<int32_t> len(n);
    for (auto &x : len) x = rnd(5) == 0 ? -1 - rnd(3) : rnd(4) == 0 ? 0 : rnd(longest + 1);
    if (rnd(2)) len[n - 1] = longest;
    DecodeParams p;
    memset(&p, 0, sizeof p);
    p.len = len.data();
    p.n = n;
    p.max_len = longest;
    p.page_size = ps;
    p.n_kv_heads = n > 100 ? 1 : 1 + rnd(3);
    p.tiles = n > 1000 ? 1 : 1 + rnd(2);
    p.alone = alone;
    const int heads = p.n_kv_heads * p.tiles;
    p.grid = alone ? n * heads : 1 + rnd(12);
    const uint64_t parts = ps / 16;
    int bits = 0;
    while (((uint64_t)1 << bits) < parts) ++bits;
    p.part_shift = 32 + bits;
    p.part_mul = (((uint64_t)1 << p.part_shift) + parts - 1) / parts;
    std::vector<At> want, got;
    const int unit = OP::KEYS * WAVES;
    for (int r = 0; r < n; ++r)
        for (int h = 0; h < heads; ++h)
            for (int u = 0; len[r] >= 0 && u < std::max(1, (len[r] + unit - 1) / unit); ++u) want.push_back({0, r, h, u});
    const std::vector<int32_t> was = len;
    for (int wg = 0; wg < p.grid; ++wg) {
        if (changes) len = was;
        walk<OP, WAVES>(p, wg, rnd(WAVES), [&] {
            if (!changes) return;
            const int how = rnd(4);
            for (auto &x : len) x = how == 0 ? -1 : how == 1 ? 0 : how == 2 ? x / 2 : rnd(longest + 1) - 5;
        }, got);
    }
    if (changes) return;
    bool same = got.size() == want.size();
    for (size_t i = 0; same && i < got.size(); ++i) same = got[i].r == want[i].r && got[i].hd == want[i].hd && got[i].u == want[i].u;
    if (!same) BAD("%d sequences, %d workgroups: %zu units of %zu", n, p.grid, got.size(), want.size());
}

int main() {
    for (int n : {1, 3, 63, 64, 65, 130, 200, 4200})
        for (int changes = 0; changes < 2; ++changes)
            for (int it = 0; it < (n > 1000 ? 1 : n > 100 ? 2 : 4); ++it) {
                const int longest = n > 1000 ? 40 : 600 / (1 + n / 40), ps = 16 * (1 + rnd(4));
                one<Op<32>, 4>(n, longest, ps, false, changes);
                if (n > 1000) continue;
                one<Op<32>, 1>(n, longest, ps, false, changes);
                one<Op<16>, 4>(n, longest, ps, false, changes);
                if (n < 60) one<Op<32>, 4>(n, longest, ps, true, changes);
            }
    if (g_bad) return 1;
    puts("all checks passed");
    return 0;
}
