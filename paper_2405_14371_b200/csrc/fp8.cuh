// What the calls with block-scaled e4m3 operands share.
#pragma once

namespace es {

constexpr int FP8_BLOCK = 128;                           // columns (and rows of a weight) that share a scale
constexpr int fp8_blocks(int n) { return (n - 1) / FP8_BLOCK + 1; }                    // that n > 0 columns or rows take
static_assert(fp8_blocks(1) == 1 && fp8_blocks(128) == 1 && fp8_blocks(129) == 2 && fp8_blocks(0x7ffffff0) == 1 << 24, "up to the largest number of columns");
constexpr float FP8_MIN_SCALE = 7.888609052210118e-31f;  // 2^-100
constexpr int FP8_MAX_ROWS = 65535 * 4;                  // rows of activations of one call (a grid's second dimension)

}  // namespace es
