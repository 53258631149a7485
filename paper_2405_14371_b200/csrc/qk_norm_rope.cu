// Norm of every query and key head, rotation by the position, and the way into the cache, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * gain          over the hd values of a head (left out where there is no gain)
//   (y_i, y_j) -> (y_i cos - y_j sin, y_j cos + y_i sin)   for the pairs (2i, 2i + 1) or (i, i + rot / 2) of the first rot values
//
// A head's hd values are 8 to a thread: 8, 16 or 32 lanes share a head, the squares are added by shuffles in fp32, and a
// partner of the second pairing lies in another lane of the group.  A warp keeps to one token, whose cosines and sines it
// holds in registers while it walks over the token's heads.  All arithmetic is fp32, rounded once when it is stored.
//
// Bound: reading every element once and writing it once.
#include <cuda_bf16.h>

#include "es_internal.cuh"
#include "launch.cuh"

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
  int heads;                                 // Hq + Hkv (+ Hkv with v)
  int paged, P, n_pages;
  int gain;                                  // ES_DTYPE_* of the gains
  int per_warp;                              // groups of heads a warp walks over
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
  if (!g) return;
  if (dtype == ES_DTYPE_F16) load8((const __half*)g + at, v);
  else if (dtype == ES_DTYPE_BF16) load8((const __nv_bfloat16*)g + at, v);
  else { load4((const float*)g + at, v, 0); load4((const float*)g + at + 4, v, 4); }
}

constexpr int WARPS = 8;

template <typename T, int HD, bool HALVES>
__global__ void __launch_bounds__(WARPS * 32) qk_norm_rope_kernel(const HeadsParams p) {
  constexpr int LANES = HD / 8, PER = 32 / LANES;          // lanes of a head, heads a warp holds at a time
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, part = lane % LANES, sub = lane / LANES;
  const int chunk = PER * p.per_warp;                      // heads of a warp
  const int tasks = (p.heads + chunk - 1) / chunk;         // warps of a token
  const int64_t task = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
  const int64_t token = task / tasks;
  const int h0 = (int)(task % tasks) * chunk;
  pdl_wait();
  if (token >= p.n) return;

  const int pos = p.positions[token];
  const bool there = (unsigned)pos < (unsigned)p.max_pos;  // else a padded row: its queries are zeros, nothing is cached
  int64_t page = -1;
  int off = 0;
  if (p.paged && there) {
    const int slot = p.slots[token];
    if (slot >= 0 && slot / p.P < p.n_pages) { page = slot / p.P; off = slot % p.P; }
  }
  // factors of this lane's values
  const int d0 = part * 8, half = p.rot >> 1;
  const bool turned = d0 < p.rot;
  float c[8], s[8];
  if (turned && there) {
    if (HALVES) {
      const int64_t at = (int64_t)pos * half + (d0 < half ? d0 : d0 - half);
      load4(p.cosines + at, c, 0); load4(p.cosines + at + 4, c, 4);
      load4(p.sines + at, s, 0); load4(p.sines + at + 4, s, 4);
    } else {
      const int64_t at = (int64_t)pos * half + (d0 >> 1);
      load4(p.cosines + at, c, 0);
      load4(p.sines + at, s, 0);
    }
  }
  float qg[8], kg[8];
  load_gain(p.q_gain, p.gain, d0, qg);
  load_gain(p.k_gain, p.gain, d0, kg);

#pragma unroll 2
  for (int i = 0; i < p.per_warp; ++i) {
    const int h = h0 + i * PER + sub;
    const bool real = h < p.heads;
    const int kind = h < p.Hq ? 0 : h < p.Hq + p.Hkv ? 1 : 2;           // query, key, value
    const int hh = kind == 0 ? h : kind == 1 ? h - p.Hq : h - p.Hq - p.Hkv;
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = 0.f;
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (real && there) {
      const T* row = kind == 0 ? (const T*)p.q + token * p.q_stride : kind == 1 ? (const T*)p.k + token * p.k_stride : (const T*)p.v + token * p.v_stride;
      raw = *reinterpret_cast<const uint4*>(row + (int64_t)hh * HD + d0);
    }
    {
      const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) { const float2 f = Pair<T>::get(w[j]); y[2 * j] = f.x; y[2 * j + 1] = f.y; }
    }
    const void* gain = kind == 0 ? p.q_gain : p.k_gain;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fmaf(y[j], y[j], sum);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (gain && kind < 2) {
      const float r = rsqrtf(sum * (1.0f / HD) + p.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = y[j] * r * (kind == 0 ? qg[j] : kg[j]);
    }
    float z[8];
    if (HALVES) {
      const bool first = d0 < half;
      const int from = first ? lane + half / 8 : lane - half / 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float other = __shfl_sync(0xffffffffu, y[j], from);
        z[j] = first ? y[j] * c[j] - other * s[j] : y[j] * c[j] + other * s[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        z[2 * j] = y[2 * j] * c[j] - y[2 * j + 1] * s[j];
        z[2 * j + 1] = y[2 * j + 1] * c[j] + y[2 * j] * s[j];
      }
    }
    if (!real) continue;
    uint4 u = raw;
    if (kind < 2 && there) {
#pragma unroll
      for (int j = 0; j < 8; ++j) if (turned) y[j] = z[j];
      u = make_uint4(Pair<T>::put(y[0], y[1]), Pair<T>::put(y[2], y[3]), Pair<T>::put(y[4], y[5]), Pair<T>::put(y[6], y[7]));
    }
    T* out;
    if (kind == 0) {
      out = (T*)p.q_out + (token * p.Hq + hh) * HD;
    } else {
      T* base = (T*)(kind == 1 ? p.k_out : p.v_out);
      if (p.paged) {
        if (page < 0) continue;
        out = base + ((page * p.Hkv + hh) * p.P + off) * HD;
      } else {
        out = base + (token * p.Hkv + hh) * HD;
      }
    }
    *reinterpret_cast<uint4*>(out + d0) = u;
  }
}

template <typename T, int HD>
es_status_t launch(const HeadsParams& p0, bool halves, cudaStream_t s) {
  HeadsParams p = p0;
  constexpr int PER = 32 / (HD / 8);
  // A warp walks over several groups of heads once there are enough warps without it (about 16 for each of an SM's
  // schedulers), which spares it the token's factors.
  const int groups = (p.heads + PER - 1) / PER;
  int per = 1;
  while (per < 4 && (long long)p.n * ((groups + 2 * per - 1) / (2 * per)) >= 64LL * sm_count()) per *= 2;
  p.per_warp = per;
  const long long warps = (long long)p.n * ((groups + per - 1) / per), ctas = (warps + WARPS - 1) / WARPS;
  if (ctas > INT32_MAX) return fail(ES_ERR_RANGE, "n * heads exceeds one launch");
  if (halves) ES_CUDA_CHECK(launch_kernel(qk_norm_rope_kernel<T, HD, true>, dim3((unsigned)ctas), dim3(WARPS * 32), 0, s, tunables().pdl != 0, p));
  else ES_CUDA_CHECK(launch_kernel(qk_norm_rope_kernel<T, HD, false>, dim3((unsigned)ctas), dim3(WARPS * 32), 0, s, tunables().pdl != 0, p));
  return ES_OK;
}

template <typename T>
es_status_t launch_hd(const HeadsParams& p, int hd, bool halves, cudaStream_t s) {
  if (hd == 64) return launch<T, 64>(p, halves, s);
  if (hd == 128) return launch<T, 128>(p, halves, s);
  return launch<T, 256>(p, halves, s);
}

bool stride_ok(int64_t stride, int64_t least, int64_t n) { return stride % 8 == 0 && (n <= 1 || stride >= least); }

bool overlap(const void* a, int64_t a_elems, const void* b, int64_t b_elems) {
  const char *x = (const char*)a, *y = (const char*)b;
  return a && b && x < y + 2 * b_elems && y < x + 2 * a_elems;
}

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
  if (Hq > (1 << 16) || Hkv > (1 << 16)) return fail(ES_ERR_RANGE, "more than 2^16 heads");
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
  // a warp may write a head while another has yet to read its own: results lie apart from what is read
  const int64_t qs = (int64_t)(n - 1) * q_stride + (int64_t)Hq * hd, ks = (int64_t)(n - 1) * k_stride + (int64_t)Hkv * hd,
                vs = (int64_t)(n - 1) * v_stride + (int64_t)Hkv * hd, qo = (int64_t)n * Hq * hd,
                ko = slot_map ? (int64_t)n_pages * Hkv * page_tokens * hd : (int64_t)n * Hkv * hd;
  const struct { const void* p; int64_t n; } in[3] = {{q, qs}, {k, ks}, {v, vs}}, out[3] = {{q_out, qo}, {k_out, ko}, {v_out, ko}};
  for (auto& i : in)
    for (auto& o : out)
      if (overlap(i.p, i.n, o.p, o.n)) return fail(ES_ERR_INVALID_ARG, "a result overlaps what is read");
  HeadsParams p{};
  p.q = q; p.k = k; p.v = v;
  p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
  p.q_gain = q_gain; p.k_gain = k_gain; p.gain = gain_dtype;
  p.cosines = cosines; p.sines = sines;
  p.positions = positions; p.slots = slot_map;
  p.q_out = q_out; p.k_out = k_out; p.v_out = v_out;
  p.eps = eps;
  p.n = n; p.Hq = Hq; p.Hkv = Hkv; p.rot = rot; p.max_pos = max_pos;
  p.heads = Hq + Hkv * (v ? 2 : 1);
  p.paged = slot_map != nullptr; p.P = page_tokens > 0 ? page_tokens : 1; p.n_pages = n_pages;
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == ES_DTYPE_F16 ? launch_hd<__half>(p, hd, halves != 0, s) : launch_hd<__nv_bfloat16>(p, hd, halves != 0, s);
}
