// Checks on the host, over a grid of sizes, that the items of a norm gradient
// cover every row once and that its workspace holds what its kernels index
// (the rules of oc_norm_plan.h).
#include "oc_norm_plan.h"
#include "oc.h"
#include <cstdio>
#include <cstring>
#include <vector>

using namespace oc;

static int check(int rows, int C, int per, bool mods, bool vecs, bool bf16) {
    const GradPlan g = grad_plan(rows, C, per, mods, vecs, bf16);
    const int T = 256 / g.team.threads;
    auto bad = [&](const char *what) {
        std::printf("%s: rows %d C %d per %d mods %d vecs %d: part %d per_group %d items %d blocks %d\n", what, rows, C,
                    per, mods, vecs, g.part, g.per_group, g.n_items, g.blocks);
        return 1;
    };
    if (g.part < 1 || g.per_group < 1 || g.n_items < 1 || g.blocks < 1 || g.blocks > GRAD_BLOCKS) return bad("range");
    if (g.team.chunks > 0 && g.team.threads * g.team.chunks * 8 < C) return bad("team");
    if (g.blocks > g.n_items && !g.alone) return bad("a block without an item");
    std::vector<char> seen(rows, 0);
    for (int i = 0; i < g.n_items; ++i) {
        long start, stop;
        if (g.team.chunks == 0) {
            start = (long)i * g.part;
            stop = std::min(start + g.part, (long)rows);
        } else {
            // as k_norm_grad
            const int group = i / g.per_group;
            start = (long)group * per + (long)(i - group * g.per_group) * g.part;
            stop = std::min(std::min(start + g.part, (long)(group + 1) * per), (long)rows);
            if (g.alone && g.per_group != 1) return bad("alone in parts");
        }
        for (long r = start; r < stop; ++r) {
            if (seen[r]) return bad("a row twice");
            seen[r] = 1;
        }
    }
    for (char s : seen)
        if (!s) return bad("a row without an item");
    // modulation rows and slots
    const long n_mod = (rows + per - 1) / per;
    if (g.team.chunks > 0 && (long)g.n_items != n_mod * g.per_group) return bad("items");
    const size_t slot = (g.team.chunks == 0 ? 6 : 3) * (size_t)g.n_items * C * 4;
    if (mods && (g.team.chunks == 0 || g.per_group > 1) && g.slots < slot) return bad("slots");
    if (vecs && g.sums < 4 * (size_t)g.blocks * C * 4) return bad("sums");
    if (g.team.chunks == 0 && (g.stats < (size_t)rows * GRAD_ROW_STATS || g.blocks != g.n_items)) return bad("stats");
    if (T > 1 && g.alone && (long)g.blocks * T < std::min<long>(g.n_items, (long)grad_most_blocks(g.team, rows, bf16) * T)) return bad("teams");
    // the size that callers are told covers every choice of gradients
    oc_shape sh;
    std::memset(&sh, 0, sizeof(sh));
    sh.F = sh.H = sh.W = sh.heads = 1;
    sh.head_dim = 16;
    sh.C = C;
    sh.dtype = bf16 ? OC_BF16 : OC_F32;
    if (mods && oc_norm_gate_grad_workspace_bytes(&sh, rows, per) < g.bytes()) return bad("workspace");
    if (!mods && per >= rows && oc_norm_gate_grad_workspace_bytes(&sh, rows, 0) < g.bytes()) return bad("workspace (no modulation)");
    return 0;
}

int main() {
    int rc = 0;
    for (int C : {8, 128, 136, 256, 384, 392, 512, 520, 1024, 1032, 1536, 1544, 2048, 2056, 4096, 4104, 8192, 8200, 16392})
        for (int rows : {1, 2, 3, 4, 5, 7, 15, 16, 17, 31, 100, 255, 256, 511, 512, 513, 1023, 1024, 1025, 1500, 2047, 4096,
                         4429, 20000})
            for (int per : {1, 2, 3, 4, 5, 7, 8, 15, 16, 17, 31, 32, 33, 40, 100, 256, 511, 513, 1024, 4096, 9216, 1 << 30})
                for (int w = 0; w < 8; ++w) rc |= check(rows, C, per, w & 1, w & 2, w & 4);
    return rc;
}
