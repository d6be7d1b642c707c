// Sizes that the layers' kernels and their plan share.
#pragma once

namespace occ {

constexpr int kRowBytes = 128;   // of a row of K in a tile: 64 bf16 or 32 fp32

// fp32 as bf16 planes: planes of an operand, and pairs of planes whose products are summed
constexpr int kPlanes = 3, kPairs = 6;

// blocks that make dZ
constexpr int DZ_LANES = 32;   // threads along a row, 4 columns each
constexpr int DZ_ROWS = 8;     // rows at a time

}  // namespace occ
