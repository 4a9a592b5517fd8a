// norm_items ROWS C ROWS_PER_MOD BF16: "threads chunks alone items blocks" of a
// gradient call with every vector (the rules of oc_norm_plan.h).
#include "oc_norm_plan.h"
#include <cstdio>
#include <cstdlib>

int main(int argc, char **argv) {
    if (argc != 5) return 2;
    const oc::GradPlan g =
        oc::grad_plan(std::atoi(argv[1]), std::atoi(argv[2]), std::atoi(argv[3]), true, true, std::atoi(argv[4]) != 0);
    std::printf("%d %d %d %d %d\n", g.team.threads, g.team.chunks, (int)g.alone, g.n_items, g.blocks);
    return 0;
}
