// i8_pick ROWS K N ...: the ring tile (its number) of each 8-bit product.
#include "oc_i8_pick.h"
#include <cstdio>
#include <cstdlib>

int main(int argc, char **argv) {
    if (argc < 4 || argc % 3 != 1) return 2;
    for (int i = 1; i < argc; i += 3)
        std::printf("%d ", oc::i8_pick(std::atoi(argv[i]), std::atoi(argv[i + 1]), std::atoi(argv[i + 2])));
    std::printf("\n");
    return 0;
}
