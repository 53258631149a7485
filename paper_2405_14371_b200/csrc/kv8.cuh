// Conversions between values and the codes of the 8-bit cache, shared by the kernels that write and read it.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "edgeshard.h"

namespace es {

enum Code : int { CODE_I8 = 0, CODE_E4M3 = 1 };

constexpr float KV8_MIN_SCALE = 7.888609052210118e-31f;      // 2^-100

__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
__device__ __forceinline__ __half2 bits_h2(uint32_t u) { return *reinterpret_cast<const __half2*>(&u); }

// Codes 0, 1 (lo) and 2, 3 (hi) of a word as fp16 pairs; every code of either type is an fp16 number.
// int8: with the sign bit flipped a byte is code + 128, and 0x64 in front makes it the fp16 number 1024 + that:
// one permute and one subtraction for two codes.
template <int CODE>
__device__ __forceinline__ void codes_to_h2(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (CODE == CODE_I8) {
    const __half2 bias = bits_h2(0x64806480u);               // 1152, 1152
    const uint32_t u = w ^ 0x80808080u;
    lo = h2_bits(__hsub2(bits_h2(__byte_perm(u, 0x64646464u, 0x4140)), bias));
    hi = h2_bits(__hsub2(bits_h2(__byte_perm(u, 0x64646464u, 0x4342)), bias));
  } else {
    const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffffu), __NV_E4M3);
    const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
    lo = (uint32_t)a.x | ((uint32_t)a.y << 16);
    hi = (uint32_t)b.x | ((uint32_t)b.y << 16);
  }
}

inline bool kv8_code_of(int32_t dtype, int* code) {
  if (dtype == ES_DTYPE_I8) { *code = CODE_I8; return true; }
  if (dtype == ES_DTYPE_F8E4M3) { *code = CODE_E4M3; return true; }
  return false;
}

}  // namespace es
