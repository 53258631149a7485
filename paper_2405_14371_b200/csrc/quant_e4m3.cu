// Values to e4m3 codes with one fp32 scale per block of 128 columns and 1 or 128 rows.
//
//   s = max(largest magnitude of the block * fl(1 / 448), 2^-100),   code = e4m3(x / s), to nearest, ties to even
//
// The quotient is the correctly rounded fp32 one: with a product by 1 / s instead, values beside the border between two codes
// would fall to either side.  Magnitudes are compared as integers, in which infinities and NaN are the largest: a block that
// holds one gets the scale NaN and codes that are no numbers, so nothing hides it.
//
// Bound: reading x and writing a byte per value.  Activations of 8192 x 8192: fp32 51 us, the floor of the copy rate; bf16 and
// fp16 46 to 56 (floor 31): not memory then, by the code the correctly rounded division for every value.  One row of 4096: 1.6.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "es_internal.cuh"
#include "fp8.cuh"
#include "launch.cuh"

namespace es {
namespace {

struct QuantParams {
  const void* x;
  int64_t stride;          // elements from row to row
  uint8_t* codes;          // [M, K]
  float* scale;            // block_rows 1: [K blocks, M]; 128: [row blocks, K blocks]
  int M, K, kb;
};

// 8 consecutive values
__device__ __forceinline__ void load8(const __half* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    v[2 * i] = f.x; v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

__device__ __forceinline__ uint32_t magnitude(const float (&v)[8], uint32_t m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}

__device__ __forceinline__ float scale_of(uint32_t largest) {
  return largest >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : fmaxf(__uint_as_float(largest) * (1.0f / 448.0f), FP8_MIN_SCALE);
}

__device__ __forceinline__ void store8(uint8_t* p, const float (&v)[8], float s) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(v[4 * h], s), __fdiv_rn(v[4 * h + 1], s)), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(v[4 * h + 2], s), __fdiv_rn(v[4 * h + 3], s)), __NV_SATFINITE, __NV_E4M3);
    w[h] = lo | (hi << 16);
  }
  *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

// A scale per row: 8 lanes share a block, a warp holds the same block of 4 consecutive rows (so that their scales lie
// together), the 8 warps of a CTA 8 consecutive blocks.
template <typename T>
__global__ void __launch_bounds__(256) quant_rows_kernel(const QuantParams p) {
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, part = lane & 7;
  const int b = blockIdx.x * 8 + (threadIdx.x >> 5);
  const int64_t row = (int64_t)blockIdx.y * 4 + (lane >> 3);
  const bool here = b < p.kb && row < p.M;
  pdl_wait();
  const T* x = (const T*)p.x + row * p.stride;
  float v[2][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = b * FP8_BLOCK + (part + 8 * i) * 8;
    if (here && k < p.K) {
      load8(x + k, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
    m = magnitude(v[i], m);
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float s = scale_of(m);
  if (!here) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = b * FP8_BLOCK + (part + 8 * i) * 8;
    if (k < p.K) store8(p.codes + row * p.K + k, v[i], s);
  }
  if (part == 0) p.scale[(int64_t)b * p.M + row] = s;
}

// A scale per 128 x 128 block (weights, once): a CTA per block, every thread 8 pieces of 8 values.
template <typename T>
__global__ void __launch_bounds__(256) quant_blocks_kernel(const QuantParams p) {
  __shared__ uint32_t largest[8];
  const int tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.y * FP8_BLOCK;
  float v[8][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = tid + 256 * i, k = blockIdx.x * FP8_BLOCK + (at & 15) * 8;
    const int64_t row = row0 + (at >> 4);
    if (row < p.M && k < p.K) {
      load8((const T*)p.x + row * p.stride + k, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
    m = magnitude(v[i], m);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((tid & 31) == 0) largest[tid >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, largest[i]);
  const float s = scale_of(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = tid + 256 * i, k = blockIdx.x * FP8_BLOCK + (at & 15) * 8;
    const int64_t row = row0 + (at >> 4);
    if (row < p.M && k < p.K) store8(p.codes + row * p.K + k, v[i], s);
  }
  if (tid == 0) p.scale[(int64_t)blockIdx.y * p.kb + blockIdx.x] = s;
}

template <typename T>
es_status_t launch(const QuantParams& p, int block_rows, cudaStream_t s) {
  if (block_rows == 1)
    ES_CUDA_CHECK(launch_kernel(quant_rows_kernel<T>, dim3((p.kb + 7) / 8, (p.M + 3) / 4), dim3(256), 0, s, tunables().pdl != 0, p));
  else
    ES_CUDA_CHECK(launch_kernel(quant_blocks_kernel<T>, dim3(p.kb, (p.M + FP8_BLOCK - 1) / FP8_BLOCK), dim3(256), 0, s, false, p));
  return ES_OK;
}

}  // namespace
}  // namespace es

using namespace es;

extern "C" es_status_t es_op_quant_e4m3(const void* x, int32_t dtype, int64_t row_stride, int32_t M, int32_t K, int32_t block_rows, void* codes, float* scale,
                                        void* stream) {
  if (M < 0 || K <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (block_rows != 1 && block_rows != FP8_BLOCK) return fail(ES_ERR_INVALID_ARG, "block_rows must be 1 or 128");
  if (dtype != ES_DTYPE_F16 && dtype != ES_DTYPE_BF16 && dtype != ES_DTYPE_F32) return fail(ES_ERR_INVALID_ARG, "x must be fp16, bf16 or fp32");
  if (K % 16) return fail(ES_ERR_SHAPE, "K = %d is no multiple of 16", K);
  const int most = block_rows == 1 ? FP8_MAX_ROWS : 65535 * FP8_BLOCK;
  if (M > most) return fail(ES_ERR_RANGE, "M = %d exceeds %d rows", M, most);
  if (M == 0) return ES_OK;
  if (!x || !codes || !scale) return fail(ES_ERR_INVALID_ARG, "null argument");
  if (row_stride < K || row_stride % (dtype == ES_DTYPE_F32 ? 4 : 8)) return fail(ES_ERR_INVALID_ARG, "rows of x must start every multiple of 16 bytes, at least K elements apart");
  if (((uintptr_t)x | (uintptr_t)codes) % 16 || (uintptr_t)scale % 4) return fail(ES_ERR_INVALID_ARG, "x and codes must be 16-byte aligned, scale 4-byte aligned");
  if (M > 1 && row_stride > (1LL << 40)) return fail(ES_ERR_RANGE, "row_stride exceeds 2^40");
  // a warp may write codes while another has yet to read what they would lie on
  const int64_t x_bytes = ((int64_t)(M - 1) * (M > 1 ? row_stride : 0) + K) * (dtype == ES_DTYPE_F32 ? 4 : 2), code_bytes = (int64_t)M * K;
  const int64_t scale_bytes = (int64_t)fp8_blocks(K) * (block_rows == 1 ? M : fp8_blocks(M)) * 4;
  if (overlap(x, x_bytes, codes, code_bytes) || overlap(x, x_bytes, scale, scale_bytes) || overlap(codes, code_bytes, scale, scale_bytes))
    return fail(ES_ERR_INVALID_ARG, "codes, scale and x must lie apart");
  QuantParams p{x, row_stride, (uint8_t*)codes, scale, M, K, fp8_blocks(K)};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == ES_DTYPE_F16) return launch<__half>(p, block_rows, s);
  if (dtype == ES_DTYPE_BF16) return launch<__nv_bfloat16>(p, block_rows, s);
  return launch<float>(p, block_rows, s);
}
