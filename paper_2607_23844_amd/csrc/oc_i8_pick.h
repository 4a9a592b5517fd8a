// Which ring tile the 8-bit product of many rows takes (k_i8.hip).
#pragma once
#include "oc_attn_common.h"
#include "oc_ops.h"
#include "oc_ring_tile.h"

namespace oc {

// The tile shapes' costs for this product (as RING_SHAPES; its epilogue is
// longer, in 8 bits a step is 128 elements).  Least squares over 64 products of
// 33 to 230400 rows, K and N of 64 to 6144, with and without GELU in bf16: the
// shape picked is 0.9% slower than the fastest on the average (20% at worst), in
// fp32 0.9 (27%); with the figures of the 16-bit projections 2.6, with GELU 3.6
// and in fp32 4.2% (40%).
constexpr RingShapeCost I8_SHAPES[N_RING_SHAPES] = {
    {256, 256, 1, 6.09f, {1.252f}},         {256, 192, 1, 4.95f, {0.997f}},
    {256, 128, 1, 3.91f, {0.772f}},         {128, 192, 1, 3.92f, {0.638f}},
    {96, 128, 1, 2.65f, {0.434f}},          {128, 128, 2, 2.79f, {0.494f, 1.146f}},
    {128, 192, 2, 3.76f, {0.599f, 1.451f}}, {160, 128, 2, 3.12f, {0.575f, 1.326f}},
    {64, 64, 3, 1.63f, {0.267f, 0.462f, 0.625f}}, {128, 64, 2, 2.11f, {0.356f, 0.689f}},
};

inline int i8_pick(int rows, int K, int N) {
    return ring_pick((int)(i8_row(K) / 2), [&](int BA, int BB) { return (long)cdiv(N, BA) * cdiv(rows, BB); }, I8_SHAPES);
}

}  // namespace oc
