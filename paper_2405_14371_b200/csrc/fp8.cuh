// What the calls with block-scaled e4m3 operands share.
#pragma once

namespace es {

constexpr int FP8_BLOCK = 128;                           // columns (and rows of a weight) that share a scale
constexpr float FP8_MIN_SCALE = 7.888609052210118e-31f;  // 2^-100
constexpr int FP8_MAX_ROWS = 65535 * 4;                  // rows of activations of one call (a grid's second dimension)

}  // namespace es
