// How norms share out their rows: teams of threads, and the items and workspace
// of a gradient call.  Host only; everything follows from the sizes.
#pragma once
#include <algorithm>
#include <cstddef>

namespace oc {

constexpr int NORM_CUS = 256;   // compute units

// Threads of a row (16, 32, 64 or the block of 256) and chunks of 8 channels of
// each; chunks 0: rows too long for registers.
struct NormTeam { int threads, chunks; };

// Forward: the fewest lanes that hold a row in three chunks (four from 1537
// channels) where there are rows for all units, so that fewer lanes idle and
// sums take fewer steps (230400 x 64: 29 us by 16 lanes, 94 by 64); else the
// block, whose threads have less to do one after another.
inline NormTeam norm_team(int rows, int C) {
    const int c = (C + 7) / 8;
    if (c <= 256 && rows >= 4 * NORM_CUS) {
        if (c <= 48) return {16, (c + 15) / 16};
        if (c <= 96) return {32, (c + 31) / 32};
        return {64, (c + 63) / 64};
    }
    if (c <= 256) return {256, 1};
    return {256, c <= 512 ? 2 : c <= 1024 ? 4 : 0};
}

// Gradients: 16 lanes up to 384 channels (in up to three chunks), 32 in two up to
// 512, 64 in two up to 1024 and in three up to 1536, then the block (a row's
// values, gradients and sums take over 12 registers a channel; 230400 x 320 with
// both norms' weights: 198 us by 16 lanes of three chunks, 200 by 32 of two).
inline NormTeam grad_team(int rows, int C) {
    const int c = (C + 7) / 8;
    if (c <= 192 && rows >= 4 * NORM_CUS) {
        if (c <= 48) return {16, (c + 15) / 16};
        if (c <= 64) return {32, 2};
        return {64, c <= 128 ? 2 : 3};
    }
    if (c <= 256) return {256, 1};
    return {256, c <= 512 ? 2 : c <= 1024 ? 4 : 0};
}

// Most blocks of a gradient call: about those that run at once (another round
// would pay again for a block's products and sums: 8192 x 1152 with both norms'
// weights 42 us by 256 blocks, 52 by 512).  One on a unit where a thread's chunks
// take its registers (from three, from two of fp32 of the block: 4000 x 2496 in
// fp32, likewise, 67 us by 256, 78 by 512) and where the block has few rows (300 x
// 1704 with all vectors 17 us by 150 blocks of two rows, 22 by 300), three where
// it has many of one bf16 chunk (16000 x 1704 without y 64 us by 768, 74 by 512,
// with y 80 and 86, with both norms' weights 94 and 102; 8192 rows with y 46 and
// 49, 4000 with both norms' weights 40 and 37; in fp32 16000 rows 154 and 148),
// else two.  (Teams that take a modulation row alone in two chunks hold one
// block's registers a unit where vectors' sums are wanted, so that their 512
// blocks take two rounds: a modulation row a token, both norms' weights, 20000 x
// 200 55 us and 51 by 256, x 512 125 and 124, x 704 222 and 221.  In fp32 with
// three chunks they spill 11 to 21 registers, the block with four 10.)
constexpr int GRAD_BLOCKS = 3 * NORM_CUS;
inline int grad_most_blocks(NormTeam t, int rows, bool bf16) {
    const bool block = t.threads == 256;
    if (t.chunks > 2 || (block && (rows <= 4 * NORM_CUS || (t.chunks == 2 && !bf16)))) return NORM_CUS;
    return block && t.chunks == 1 && bf16 && rows >= 32 * NORM_CUS ? GRAD_BLOCKS : 2 * NORM_CUS;
}

// Item i of n_items: rows [start, start + part) of modulation row i / per_group,
// part i % per_group of it.  alone: a team takes an item by itself, else the
// block's teams share it.  Rows too long for registers: n_items parts of all
// rows instead.  Workspace: the rows' statistics (long rows), modulation sums
// of the items (3 each; 6 for long rows' parts, which may cross two modulation
// rows), sums of the blocks (4 each).
struct GradPlan {
    NormTeam team;
    bool alone;
    int part, per_group, n_items, blocks;
    size_t stats, slots, sums;   // bytes, multiples of 256
    size_t bytes() const { return stats + slots + sums; }
};
constexpr size_t GRAD_ROW_STATS = 24;   // bytes of a long row's statistics

inline GradPlan grad_plan(int rows, int C, int rows_per_mod, bool mods, bool vecs, bool bf16 = true) {
    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    auto div = [](int a, int b) { return (a + b - 1) / b; };
    GradPlan g{};
    g.team = grad_team(rows, C);
    if (g.team.chunks == 0) {
        g.part = div(rows, 2 * NORM_CUS);
        g.per_group = 1;
        g.n_items = g.blocks = div(rows, g.part);
        g.stats = up((size_t)rows * GRAD_ROW_STATS);
        g.slots = mods ? up(6 * (size_t)g.n_items * C * 4) : 0;
    } else {
        const int most = grad_most_blocks(g.team, rows, bf16);
        const int teams = 256 / g.team.threads, per = std::min(rows_per_mod, rows), n_mod = div(rows, per);
        g.alone = teams > 1 && per < std::max(2 * teams, 16);
        // (an item's sums cost its share of LDS and of the join: four rows a team where that leaves no unit idle)
        const int least = std::min(std::max(rows / (NORM_CUS * teams), 1), 4) * teams;
        g.per_group = g.alone ? 1 : std::min(std::max(1, most / n_mod), div(per, least));
        g.part = div(per, g.per_group);
        g.per_group = div(per, g.part);
        g.n_items = n_mod * g.per_group;
        g.blocks = std::min(g.alone ? div(g.n_items, teams) : g.n_items, most);
        g.slots = mods && g.per_group > 1 ? up(3 * (size_t)g.n_items * C * 4) : 0;
    }
    g.sums = vecs ? up(4 * (size_t)g.blocks * C * 4) : 0;
    return g;
}

}  // namespace oc
