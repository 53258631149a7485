// Norm of every query and key head, rotation by the position, and the way into the cache, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * gain          over the hd values of a head (left out where there is no gain)
//   (y_i, y_j) -> (y_i cos - y_j sin, y_j cos + y_i sin)   for the pairs (2i, 2i + 1) or (i, i + rot / 2) of the first rot values
//
// A head's hd values are 8 to a thread: 8, 16 or 32 lanes share a head, the squares are added by shuffles in fp32, and a
// partner of the second pairing lies in another lane of the group.  A warp keeps to one token and one kind of head, asks for
// all it reads at once, and holds the products of gains, cosines and sines in registers while it walks over its heads: a
// value then costs a square, two multiply-adds and a product.  All arithmetic is fp32, rounded once when it is stored.
//
// Bound: reading every element once and writing it once.
#include <cuda_bf16.h>

#include "es_internal.cuh"
#include "launch.cuh"
#include "sm100.cuh"

namespace es {
namespace {

struct HeadsParams {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;      // elements from token to token
  const void *q_gain, *k_gain;               // [hd] or nullptr
  const float *cosines, *sines;              // [max_pos, rot / 2]
  const int *positions, *slots;
  void *q_out, *k_out, *v_out;               // dense rows, or pages
  float eps;
  int n, Hq, Hkv, rot, max_pos;
  int paged, P, n_pages;
  int gain;                                  // ES_DTYPE_* of the gains
};

template <typename T> struct Pair;
template <> struct Pair<__half> {
  static __device__ __forceinline__ float2 get(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
  static __device__ __forceinline__ uint32_t put(float a, float b) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
};
template <> struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ float2 get(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
  static __device__ __forceinline__ uint32_t put(float a, float b) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = Pair<T>::get(w[i]);
    v[2 * i] = f.x; v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void load4(const float* p, float (&v)[8], int at) {
  const float4 f = *reinterpret_cast<const float4*>(p);
  v[at] = f.x; v[at + 1] = f.y; v[at + 2] = f.z; v[at + 3] = f.w;
}
__device__ __forceinline__ void load_gain(const void* g, int dtype, int at, float (&v)[8]) {
  if (dtype == ES_DTYPE_F16) load8((const __half*)g + at, v);
  else if (dtype == ES_DTYPE_BF16) load8((const __nv_bfloat16*)g + at, v);
  else { load4((const float*)g + at, v, 0); load4((const float*)g + at + 4, v, 4); }
}

constexpr int WARPS = 8;

// A warp has one token and PER_WARP groups of heads of one kind (query, key or value); the warps of a CTA have consecutive tokens.
// FULL: every value of a head is rotated.
template <typename T, int HD, bool HALVES, bool FULL, int PER_WARP>
__global__ void __launch_bounds__(WARPS * 32) qk_norm_rope_kernel(const HeadsParams p) {
  constexpr int LANES = HD / 8, PER = 32 / LANES, CHUNK = PER * PER_WARP;      // lanes of a head, heads at a time, heads of a warp
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, part = lane % LANES, sub = lane / LANES;
  const int q_tasks = (p.Hq + CHUNK - 1) / CHUNK, k_tasks = (p.Hkv + CHUNK - 1) / CHUNK;
  const int64_t token = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
  int task = blockIdx.y;
  const int kind = task < q_tasks ? 0 : task < q_tasks + k_tasks ? 1 : 2;
  task -= kind == 0 ? 0 : kind == 1 ? q_tasks : q_tasks + k_tasks;
  const int heads = kind == 0 ? p.Hq : p.Hkv, h0 = task * CHUNK + sub, d0 = part * 8;
  pdl_wait();
  if (token >= p.n) return;

  // everything that this warp reads is asked for at once
  const T* row = (const T*)(kind == 0 ? p.q : kind == 1 ? p.k : p.v) + token * (kind == 0 ? p.q_stride : kind == 1 ? p.k_stride : p.v_stride) + d0;
  uint4 raw[PER_WARP];
#pragma unroll
  for (int i = 0; i < PER_WARP; ++i) {
    const int h = h0 + i * PER;
    raw[i] = h < heads ? *reinterpret_cast<const uint4*>(row + (int64_t)h * HD) : make_uint4(0, 0, 0, 0);
  }
  const int pos = p.positions[token];
  const bool there = (unsigned)pos < (unsigned)p.max_pos;    // else a padded row: its queries are zeros, nothing is cached
  // where the first of the heads goes, and how far apart they are there
  T* out;
  int64_t step;
  if (kind == 0 || !p.paged) {
    out = (T*)(kind == 0 ? p.q_out : kind == 1 ? p.k_out : p.v_out) + token * heads * HD;
    step = HD;
  } else {
    const int slot = there ? p.slots[token] : -1, page = slot / p.P;
    if (slot < 0 || page >= p.n_pages) return;               // the whole warp: one token
    out = (T*)(kind == 1 ? p.k_out : p.v_out) + ((int64_t)page * p.Hkv * p.P + slot % p.P) * HD;
    step = (int64_t)p.P * HD;
  }
  out += d0;
  if (kind == 2 || !there) {
#pragma unroll
    for (int i = 0; i < PER_WARP; ++i) {
      const int h = h0 + i * PER;
      if (h < heads) *reinterpret_cast<uint4*>(out + h * step) = there ? raw[i] : make_uint4(0, 0, 0, 0);
    }
    return;
  }

  // factors of this lane's values: y' = r * (x * own + partner's x * other), gains and rotation in one
  const void* gain = kind == 0 ? p.q_gain : p.k_gain;
  const int half = p.rot >> 1;
  const bool turned = FULL || d0 < p.rot, first = d0 < half;
  float own[8], other[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) { own[j] = 1.f; other[j] = 0.f; }
  if (gain) load_gain(gain, p.gain, d0, own);
  int from = lane;                                           // HALVES: the partner's lane
  if (HALVES) {
    if (turned) {
      const int shift = first ? half : -half;
      from = lane + shift / 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) other[j] = 1.f;
      if (gain) load_gain(gain, p.gain, d0 + shift, other);
      const int64_t at = (int64_t)pos * half + (first ? d0 : d0 - half);
      float c[8], s[8];
      load4(p.cosines + at, c, 0); load4(p.cosines + at + 4, c, 4);
      load4(p.sines + at, s, 0); load4(p.sines + at + 4, s, 4);
#pragma unroll
      for (int j = 0; j < 8; ++j) { own[j] *= c[j]; other[j] *= first ? -s[j] : s[j]; }
    }
  } else if (turned) {
    const int64_t at = (int64_t)pos * half + (d0 >> 1);
    float c[8], s[8];
    load4(p.cosines + at, c, 0);
    load4(p.sines + at, s, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      other[2 * j] = -s[j] * own[2 * j + 1];
      other[2 * j + 1] = s[j] * own[2 * j];
      own[2 * j] *= c[j];
      own[2 * j + 1] *= c[j];
    }
  }

  uint64_t own2[4], other2[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) { own2[j] = pack_f32x2(own[2 * j], own[2 * j + 1]); other2[j] = pack_f32x2(other[2 * j], other[2 * j + 1]); }
#pragma unroll
  for (int i = 0; i < PER_WARP; ++i) {
    const int h = h0 + i * PER;
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    float2 y[4];
    uint64_t y2[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) { y[j] = Pair<T>::get(w[j]); y2[j] = pack_f32x2(y[j].x, y[j].y); }
    float r = 1.f;
    if (gain) {
      uint64_t sum2 = mul_f32x2(y2[0], y2[0]);
#pragma unroll
      for (int j = 1; j < 4; ++j) sum2 = fma_f32x2(y2[j], y2[j], sum2);
      const float2 both = unpack_f32x2(sum2);
      float sum = both.x + both.y;
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      r = rsqrtf(sum * (1.0f / HD) + p.eps);
    }
    const uint64_t r2 = pack_f32x2(r, r);
    uint32_t z[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float2 m = make_float2(y[j].y, y[j].x);
      if (HALVES) m = Pair<T>::get(__shfl_sync(0xffffffffu, w[j], from));
      // a value without a partner takes nothing of the one that stands there, whatever it is
      uint64_t v = mul_f32x2(y2[j], own2[j]);
      if (FULL) v = fma_f32x2(pack_f32x2(m.x, m.y), other2[j], v);
      else if (turned) v = fma_f32x2(pack_f32x2(m.x, m.y), other2[j], v);
      const float2 t = unpack_f32x2(mul_f32x2(v, r2));
      z[j] = Pair<T>::put(t.x, t.y);
    }
    if (h < heads) *reinterpret_cast<uint4*>(out + h * step) = make_uint4(z[0], z[1], z[2], z[3]);
  }
}

template <typename T, int HD, bool HALVES, int PER_WARP>
es_status_t launch_per(const HeadsParams& p, cudaStream_t s) {
  constexpr int CHUNK = 32 / (HD / 8) * PER_WARP;
  const int tasks = (p.Hq + CHUNK - 1) / CHUNK + (p.Hkv + CHUNK - 1) / CHUNK * (p.v ? 2 : 1);
  const dim3 grid((unsigned)((p.n - 1) / WARPS + 1), (unsigned)tasks);
  const bool pdl = tunables().pdl != 0;
  if (p.rot == HD) ES_CUDA_CHECK(launch_kernel(qk_norm_rope_kernel<T, HD, HALVES, true, PER_WARP>, grid, dim3(WARPS * 32), 0, s, pdl, p));
  else ES_CUDA_CHECK(launch_kernel(qk_norm_rope_kernel<T, HD, HALVES, false, PER_WARP>, grid, dim3(WARPS * 32), 0, s, pdl, p));
  return ES_OK;
}

template <typename T, int HD>
es_status_t launch(const HeadsParams& p, bool halves, cudaStream_t s) {
  // A warp walks over four groups of heads once that leaves enough warps (about 16 for each of an SM's schedulers), which
  // spares it the token's factors.
  constexpr int CHUNK = 32 / (HD / 8) * 4;
  const bool many = (long long)p.n * (p.Hq + p.Hkv) >= 64LL * sm_count() * CHUNK;
  if (halves) return many ? launch_per<T, HD, true, 4>(p, s) : launch_per<T, HD, true, 1>(p, s);
  return many ? launch_per<T, HD, false, 4>(p, s) : launch_per<T, HD, false, 1>(p, s);
}

template <typename T>
es_status_t launch_hd(const HeadsParams& p, int hd, bool halves, cudaStream_t s) {
  if (hd == 64) return launch<T, 64>(p, halves, s);
  if (hd == 128) return launch<T, 128>(p, halves, s);
  return launch<T, 256>(p, halves, s);
}

bool stride_ok(int64_t stride, int64_t least, int64_t n) { return stride % 8 == 0 && (n <= 1 || stride >= least); }

}  // namespace
}  // namespace es

using namespace es;

extern "C" es_status_t es_op_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int32_t dtype,
                                          const void* q_gain, const void* k_gain, int32_t gain_dtype, float eps, const float* cosines, const float* sines,
                                          int32_t max_pos, int32_t rot, int32_t halves, const int32_t* positions, void* q_out, void* k_out, void* v_out, int32_t n,
                                          int32_t Hq, int32_t Hkv, int32_t hd, const int32_t* slot_map, int32_t page_tokens, int32_t n_pages, void* stream) {
  if (n < 0 || Hq <= 0 || Hkv <= 0 || max_pos <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (hd != 64 && hd != 128 && hd != 256) return fail(ES_ERR_SHAPE, "head_dim must be 64, 128 or 256");
  if (rot < 0 || rot > hd || rot % 16) return fail(ES_ERR_SHAPE, "rot must be a multiple of 16, at most the head dimension");
  if (dtype != ES_DTYPE_F16 && dtype != ES_DTYPE_BF16) return fail(ES_ERR_INVALID_ARG, "q, k and v must be fp16 or bf16");
  if (gain_dtype != ES_DTYPE_F16 && gain_dtype != ES_DTYPE_BF16 && gain_dtype != ES_DTYPE_F32) return fail(ES_ERR_INVALID_ARG, "gains must be fp16, bf16 or fp32");
  if (!(eps >= 0.f)) return fail(ES_ERR_INVALID_ARG, "eps must not be negative");
  if (Hq > (1 << 14) || Hkv > (1 << 14)) return fail(ES_ERR_RANGE, "more than 2^14 heads");
  if (slot_map) {
    if (page_tokens < 16 || (page_tokens & (page_tokens - 1))) return fail(ES_ERR_SHAPE, "page_tokens must be a power of two, at least 16");
    if (n_pages <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
    if ((long long)n_pages * page_tokens > INT32_MAX) return fail(ES_ERR_RANGE, "the pool exceeds 2^31 - 1 slots");
  }
  if (n == 0) return ES_OK;
  if (!q || !k || !q_out || !k_out || !positions || (rot && (!cosines || !sines))) return fail(ES_ERR_INVALID_ARG, "null argument");
  if (!v != !v_out) return fail(ES_ERR_INVALID_ARG, "v and its destination go together");
  if (!stride_ok(q_stride, (int64_t)Hq * hd, n) || !stride_ok(k_stride, (int64_t)Hkv * hd, n) || (v && !stride_ok(v_stride, (int64_t)Hkv * hd, n)))
    return fail(ES_ERR_INVALID_ARG, "token strides must be multiples of 8, at least a token's heads");
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)k_out | (uintptr_t)v_out | (uintptr_t)q_gain | (uintptr_t)k_gain | (uintptr_t)cosines |
       (uintptr_t)sines) % 16)
    return fail(ES_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  // a warp may write a head while another has yet to read its own: results lie apart from what is read, and from one another
  const int64_t qs = (int64_t)(n - 1) * q_stride + (int64_t)Hq * hd, ks = (int64_t)(n - 1) * k_stride + (int64_t)Hkv * hd,
                vs = (int64_t)(n - 1) * v_stride + (int64_t)Hkv * hd, qo = (int64_t)n * Hq * hd,
                ko = slot_map ? (int64_t)n_pages * Hkv * page_tokens * hd : (int64_t)n * Hkv * hd;
  const struct { const void* p; int64_t n; } in[3] = {{q, qs}, {k, ks}, {v, vs}}, out[3] = {{q_out, qo}, {k_out, ko}, {v_out, ko}};
  for (auto& i : in)
    for (auto& o : out)
      if (overlap(i.p, 2 * i.n, o.p, 2 * o.n)) return fail(ES_ERR_INVALID_ARG, "a result overlaps what is read");
  for (int i = 0; i < 3; ++i)
    if (overlap(out[i].p, 2 * out[i].n, out[(i + 1) % 3].p, 2 * out[(i + 1) % 3].n)) return fail(ES_ERR_INVALID_ARG, "two results overlap");
  HeadsParams p{};
  p.q = q; p.k = k; p.v = v;
  p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
  p.q_gain = q_gain; p.k_gain = k_gain; p.gain = gain_dtype;
  p.cosines = cosines; p.sines = sines;
  p.positions = positions; p.slots = slot_map;
  p.q_out = q_out; p.k_out = k_out; p.v_out = v_out;
  p.eps = eps;
  p.n = n; p.Hq = Hq; p.Hkv = Hkv; p.rot = rot; p.max_pos = max_pos;
  p.paged = slot_map != nullptr; p.P = page_tokens > 0 ? page_tokens : 1; p.n_pages = n_pages;
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == ES_DTYPE_F16 ? launch_hd<__half>(p, hd, halves != 0, s) : launch_hd<__nv_bfloat16>(p, hd, halves != 0, s);
}
