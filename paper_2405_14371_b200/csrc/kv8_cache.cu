// Writing K and V rows into the paged 8-bit cache, and reading them back.
//
// append: an item is one stretch of consecutive rows in one page, for one KV head and one of K / V.  A group of warps
// takes an item: it finds the stretch's length in the slot map, takes the largest magnitude of its rows (as integers:
// the bits of |x| order like the numbers, infinities and NaN above all), settles the page's scale, brings the codes in
// front to it if it grew, and writes the new codes.  One group owns the page and head for the whole call, so nothing is
// atomic and the result does not depend on scheduling.
//
// Bound: append reads two bytes and writes one per value, gather the reverse.  8 prompts of up to 2600 tokens behind up to 300,
// 32 heads of 128 (256 MB for append, 285 MB for gather), take 103 us together, 5.2 TB/s; append fills 60 % of the issue
// slots beside that (two conversions, the scaling and the rounding of every value).  The newest token of 64 sequences of 8
// heads, and all 3900 of theirs read back (24 MB), take 9.0 us: two launches and a chain of slot, scale and codes each.
#include "es_internal.cuh"
#include "kv8.cuh"
#include "launch.cuh"

namespace es {
namespace {

constexpr int APPEND_THREADS = 256;

struct AppendParams {
  const uint16_t *k, *v;
  int64_t row_stride;
  const int *slots, *runs;
  int n_rows, n_items;             // n_items: runs, or rows where there are none
  uint8_t *k_pages, *v_pages;
  float *k_scale, *v_scale;
  int Hkv, P, log2P, n_pages;
};

template <bool BF16>
__device__ __forceinline__ float2 to_float2(uint32_t w) {
  if (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  return __half22float2(bits_h2(w));
}

// larger magnitudes of two pairs; NaN wins
template <bool BF16>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  if (BF16) {
    const __nv_bfloat162 r = __hmax2_nan(__habs2(*reinterpret_cast<const __nv_bfloat162*>(&a)), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  return h2_bits(__hmax2_nan(__habs2(bits_h2(a)), __habs2(bits_h2(b))));
}

// round(x / s) to nearest, ties to even, exactly: x * (1 / s) is within one of it, and the remainder x - q s is a
// multiple of the last place of s no larger than s, so one fused multiply-add gives it without rounding.
__device__ __forceinline__ int quotient_code(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float r = fmaf(-q, s, x), twice = 2.f * fabsf(r);
  if (twice > s || (twice == s && (((int)q) & 1))) q += r > 0.f ? 1.f : -1.f;
  return (int)q;
}

// 8 values at scale s -> 8 codes.  int8: x * inv is within 127 * 2^-24 < 1e-5 of x / s (the product is not rounded
// before it meets 1.5 * 2^23, which leaves the nearest integer in the low bits), so only where it comes that close to the
// middle between two codes does the exact form decide: 6 instructions a value instead of 14.
template <int CODE, bool BF16>
__device__ __forceinline__ uint2 encode(const uint4& x, float s, float inv) {
  const uint32_t in[4] = {x.x, x.y, x.z, x.w};
  uint32_t out[2];
  float off = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 a = to_float2<BF16>(in[2 * i]), b = to_float2<BF16>(in[2 * i + 1]);
    if (CODE == CODE_I8) {
      const float v[4] = {a.x, a.y, b.x, b.y};
      uint32_t t[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float m = fmaf(v[j], inv, 12582912.f);
        t[j] = __float_as_uint(m);
        off = fmaxf(off, fabsf(fmaf(v[j], inv, 12582912.f - m)));
      }
      out[i] = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
    } else {
      const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a.x * inv, a.y * inv), __NV_SATFINITE, __NV_E4M3);
      const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(b.x * inv, b.y * inv), __NV_SATFINITE, __NV_E4M3);
      out[i] = (uint32_t)lo | ((uint32_t)hi << 16);
    }
  }
  if (CODE == CODE_I8 && off > 0.49998f) {
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      const float2 a = to_float2<BF16>(i ? x.z : x.x), b = to_float2<BF16>(i ? x.w : x.y);
      const int c0 = quotient_code(a.x, s, inv), c1 = quotient_code(a.y, s, inv), c2 = quotient_code(b.x, s, inv),
                c3 = quotient_code(b.y, s, inv);
      const uint32_t w = (c0 & 255) | ((c1 & 255) << 8) | ((c2 & 255) << 16) | ((uint32_t)c3 << 24);
      if (i) out[1] = w; else out[0] = w;
    }
  }
  return make_uint2(out[0], out[1]);
}

// 8 values at an e4m3 scale that is no power of two (append makes none; a page another program filled may hold one): 1 / s
// is not exact then.  A quotient of 11 and 24 bits that is not the middle between two codes lies more than 2^-30 of itself
// from it, so the 64-bit one lies on its side, and is rounded once.  A division a value: only pages with such a scale come here.
template <bool BF16>
__device__ __forceinline__ uint2 encode_divided(const uint4& x, float s) {
  uint2 out = make_uint2(0, 0);
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    const uint32_t w = i < 2 ? x.x : i < 4 ? x.y : i < 6 ? x.z : x.w;
    const float2 v = to_float2<BF16>(w);
    const uint32_t c = __nv_cvt_double_to_fp8((double)(i & 1 ? v.y : v.x) / (double)s, __NV_SATFINITE, __NV_E4M3);
    if (i < 4) out.x |= c << (8 * i); else out.y |= c << (8 * (i - 4));
  }
  return out;
}

// Four codes at the old scale -> four codes at the new one, round(code * old / new) to nearest, ties to even.  int8: with
// `ratio` rounded to 53 bits the product misses the middle between two codes by at most 2^-45, and what is not the middle
// itself lies at least 2^-34 from it (32 bits over 24); so only there the remainder decides, which two 32-bit products give exactly.
// e4m3: the new scale is a power of two, so the product of 4 and 24 bits is exact in 64 bits, and in 32 where the old one is too.
template <int CODE>
__device__ __forceinline__ uint32_t rescale(uint32_t w, double ratio, float s_old, float s) {
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t c = (w >> (8 * i)) & 255u;
    uint32_t n;
    if (CODE == CODE_I8) {
      const double code = (double)(int)(int8_t)c, to = code * ratio;
      int q = __double2int_rn(to);
      if (fabs(to - (double)q) > 0.4999999999) {
        const double r = fma(code, (double)s_old, -(double)q * (double)s), twice = 2.0 * fabs(r);
        if (twice > (double)s || (twice == (double)s && (q & 1))) q += r > 0.0 ? 1 : -1;
      }
      n = (uint32_t)q & 255u;
    } else {
      const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)c, __NV_E4M3);
      const float number = __half2float(__half(h));
      n = __float_as_uint(s_old) & 0x7fffffu ? __nv_cvt_double_to_fp8((double)number * ratio, __NV_SATFINITE, __NV_E4M3)
                                             : __nv_cvt_float_to_fp8(number * (float)ratio, __NV_SATFINITE, __NV_E4M3);
    }
    out |= n << (8 * i);
  }
  return out;
}

// the scale that a largest magnitude asks for
template <int CODE>
__device__ __forceinline__ float wanted_scale(float amax) {
  if (CODE == CODE_I8) return fmaxf(__fdiv_rn(amax, 127.f), KV8_MIN_SCALE);
  // smallest power of two s with amax <= 448 s = 1.75 * 2^8 s
  const uint32_t bits = __float_as_uint(amax);
  int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
  e = e < -100 ? -100 : e;         // zero and subnormal magnitudes end here too
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// barrier of the WARPS warps that share an item (groups of a CTA may leave early, so each has a barrier of its own)
template <int WARPS>
__device__ __forceinline__ void group_sync() {
  if (WARPS == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / (32 * WARPS)), "n"(32 * WARPS) : "memory");
}

template <int HD, int CODE, bool BF16, int WARPS>
__global__ void __launch_bounds__(APPEND_THREADS, 4) kv8_append_kernel(const AppendParams p) {
  constexpr int GROUP = 32 * WARPS;                // threads of an item
  constexpr int CPR = HD / 8;                      // 16-byte pieces of a row
  constexpr int KEEP = 8;                          // pieces a thread holds in registers between the two uses
  __shared__ uint32_t s_max[APPEND_THREADS / 32];
  __shared__ int s_len[APPEND_THREADS / 32];
  const int tid = threadIdx.x % GROUP, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // heads change fastest: the groups of a CTA share rows of the slot map and read one row's heads side by side
  const unsigned item = blockIdx.x * (APPEND_THREADS / GROUP) + threadIdx.x / GROUP;
  const int which = item / (unsigned)p.Hkv, h = item - which * p.Hkv;
  pdl_launch_dependents();
  if (which >= p.n_items) return;                  // uniform over the group
  const int r0 = p.runs ? p.runs[which] : which;
  if (r0 < 0 || r0 >= p.n_rows) return;
  const int slot = p.slots[r0];
  if (slot < 0 || slot >= p.n_pages * p.P) return;
  const int page = slot >> p.log2P, off = slot & (p.P - 1);
  if (!p.runs && r0 > 0 && off > 0 && p.slots[r0 - 1] == slot - 1) return;      // inside a stretch

  const uint16_t* src = (blockIdx.y ? p.v : p.k) + (int64_t)r0 * p.row_stride + (int64_t)h * HD;
  uint8_t* dst = (blockIdx.y ? p.v_pages : p.k_pages) + ((int64_t)page * p.Hkv + h) * ((int64_t)p.P * HD);
  float* scale = (blockIdx.y ? p.v_scale : p.k_scale) + (int64_t)page * p.Hkv + h;
  const float s_old = off > 0 ? *scale : 0.f;
  // this thread's pieces: tid, tid + GROUP, ... of the stretch, row after row
  const uint16_t* at = src + (int64_t)(tid / CPR) * p.row_stride + (tid % CPR) * 8;
  const int64_t step = (int64_t)(GROUP / CPR) * p.row_stride;
  auto piece = [&](int j) { return *reinterpret_cast<const uint4*>(at + j * step); };

  // ---- the first rows are on their way while the length of the stretch is found: the first row that does not follow on ----
  const int most = min(p.P - off, p.n_rows - r0);
  uint4 keep[KEEP];
#pragma unroll
  for (int j = 0; j < KEEP; ++j) {
    keep[j] = make_uint4(0, 0, 0, 0);
    if (tid + j * GROUP < most * CPR) keep[j] = piece(j);
  }
  int len = most;
  if (WARPS == 1) {
    for (int i = 1; i < most; i += 32) {
      const bool stop = i + lane < most && p.slots[r0 + i + lane] != slot + i + lane;
      const unsigned m = __ballot_sync(~0u, stop);
      if (m) { len = i + __ffs(m) - 1; break; }
    }
  } else {
    int stop = most;
    for (int i = tid; i < most; i += GROUP)
      if (p.slots[r0 + i] != slot + i) { stop = i; break; }
    stop = __reduce_min_sync(~0u, stop);
    if (lane == 0) s_len[warp] = stop;
    group_sync<WARPS>();
    len = __reduce_min_sync(~0u, s_len[warp / WARPS * WARPS + lane % WARPS]);
  }
  const int pieces = len * CPR;

  // ---- largest magnitude ----
  uint32_t pair = 0;                               // two magnitudes
  auto take = [&](const uint4& x) { pair = larger<BF16>(larger<BF16>(larger<BF16>(pair, x.x), larger<BF16>(x.y, x.z)), x.w); };
#pragma unroll
  for (int j = 0; j < KEEP; ++j)
    if (tid + j * GROUP < pieces) take(keep[j]);
  for (int j = KEEP; tid + j * GROUP < pieces; ++j) take(piece(j));
  // as integers the bits of magnitudes order like the numbers, infinities and NaN above all
  uint32_t mx = max(pair & 0x7fffu, (pair >> 16) & 0x7fffu);
  mx = __reduce_max_sync(~0u, mx);
  if (WARPS > 1) {
    if (lane == 0) s_max[warp] = mx;
    group_sync<WARPS>();
    mx = __reduce_max_sync(~0u, s_max[warp / WARPS * WARPS + lane % WARPS]);
  }

  // ---- the page's scale ----
  const bool finite = mx < (BF16 ? 0x7f80u : 0x7c00u);
  const float amax = BF16 ? __uint_as_float(mx << 16) : __half2float(__ushort_as_half((unsigned short)mx));
  const float want = wanted_scale<CODE>(amax);
  float s = off > 0 ? (s_old >= want || isnan(s_old) ? s_old : want) : want;
  if (!finite) s = __int_as_float(0x7fffffff);
  const bool bad = isnan(s);
  const float inv = bad ? 0.f : 1.f / s;

  // ---- codes in front ----
  if (off > 0 && !bad && s != s_old) {
    const double ratio = (double)s_old / (double)s;
    uint4* front = reinterpret_cast<uint4*>(dst);
    for (int i = tid; i < off * HD / 16; i += GROUP) {
      uint4 w = front[i];
      w.x = rescale<CODE>(w.x, ratio, s_old, s); w.y = rescale<CODE>(w.y, ratio, s_old, s);
      w.z = rescale<CODE>(w.z, ratio, s_old, s); w.w = rescale<CODE>(w.w, ratio, s_old, s);
      front[i] = w;
    }
  }

  // ---- new codes ----
  uint2* to = reinterpret_cast<uint2*>(dst + (int64_t)off * HD);
  if (CODE == CODE_E4M3 && !bad && (__float_as_uint(s) & 0x7fffffu)) {
    for (int j = 0; tid + j * GROUP < pieces; ++j) to[tid + j * GROUP] = encode_divided<BF16>(piece(j), s);
  } else {
#pragma unroll
    for (int j = 0; j < KEEP; ++j)
      if (tid + j * GROUP < pieces) to[tid + j * GROUP] = bad ? make_uint2(0, 0) : encode<CODE, BF16>(keep[j], s, inv);
    for (int j = KEEP; tid + j * GROUP < pieces; ++j) to[tid + j * GROUP] = bad ? make_uint2(0, 0) : encode<CODE, BF16>(piece(j), s, inv);
  }
  if (WARPS == 1) __syncwarp();                    // every thread has read the old scale (several warps have met since)
  if (tid == 0) *scale = s;
}

template <int HD, int CODE, bool BF16, int WARPS>
es_status_t launch_append_warps(const AppendParams& p, cudaStream_t s) {
  constexpr int per = APPEND_THREADS / (32 * WARPS);
  const int64_t blocks = ((int64_t)p.n_items * p.Hkv + per - 1) / per;
  if ((int64_t)p.n_items * p.Hkv > INT32_MAX) return fail(ES_ERR_RANGE, "too many (run, head) items for one launch");
  // not before the kernel in front has ended: CTAs of this one that wait early cost the 64 sequences and the gather in front of
  // them 1.2 us (9.6 and 8.4 us for both; the gather itself begins early, which saves 0.6 us)
  ES_CUDA_CHECK(launch_kernel(kv8_append_kernel<HD, CODE, BF16, WARPS>, dim3((unsigned)blocks, 2), dim3(APPEND_THREADS), 0, s, false, p));
  return ES_OK;
}

// A warp per item where stretches are short on average (a decode step: one row each); else as many as give a thread eight
// 16-byte pieces of a whole page, up to eight.  Pages of 64 tokens, 1 / 2 / 4 / 8 warps: 8 prompts of up to 2600 tokens, 32 heads,
// 139 / 118 / 103 / 118 us; a decode step of 64 sequences 8.9 / 9.3 / 10.0 / 11.3 us (with the gather that follows).  The
// border is 8 rows an entry of `runs`, padding included, since the host knows no more.  64 sequences of 16 / 24 / 64 / 128 new
// rows in pages of 64 (7 / 10 / 21 / 32 rows an entry), append alone: 8 heads 6.4 / 8.6 / 14.1 / 29.3 us with one warp, 5.9 / 6.5 /
// 10.1 / 16.7 with four; 32 heads 9.6 / 15.5 / 36.4 / 66.0 and 16.1 / 19.1 / 33.6 / 51.4.  Without `runs` nothing tells prompts
// from decode steps, and a prompt takes one warp an item.
template <int HD, int CODE, bool BF16>
es_status_t launch_append(const AppendParams& p, bool whole_pages, cudaStream_t s) {
  const int warps = whole_pages ? p.P * (HD / 8) / 256 : 1;
  if (warps >= 8) return launch_append_warps<HD, CODE, BF16, 8>(p, s);
  if (warps >= 4) return launch_append_warps<HD, CODE, BF16, 4>(p, s);
  if (warps >= 2) return launch_append_warps<HD, CODE, BF16, 2>(p, s);
  return launch_append_warps<HD, CODE, BF16, 1>(p, s);
}

// ---- reading back ----------------------------------------------------------------------------------------------

constexpr int GATHER_THREADS = 256;

struct GatherParams {
  const int* slots;
  const uint8_t *k_pages, *v_pages;
  const float *k_scale, *v_scale;
  void *k, *v;
  int64_t n_items;                 // rows * Hkv * hd / 8
  int Hkv, P, log2P, n_pages;
};


// 8 codes -> 8 values of the output type at dst + 8 * item
template <int CODE, int OUT>
__device__ __forceinline__ void store_values(void* dst, int64_t item, const uint2& w, float s) {
  const uint32_t in[2] = {w.x, w.y};
  float f[8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t lo, hi;
    codes_to_h2<CODE>(in[i], lo, hi);
    const float2 a = __half22float2(bits_h2(lo)), b = __half22float2(bits_h2(hi));
    f[4 * i] = a.x * s; f[4 * i + 1] = a.y * s; f[4 * i + 2] = b.x * s; f[4 * i + 3] = b.y * s;
  }
  if (OUT == ES_DTYPE_F32) {
    float4* o = reinterpret_cast<float4*>(dst) + item * 2;
    __stcs(o, make_float4(f[0], f[1], f[2], f[3]));
    __stcs(o + 1, make_float4(f[4], f[5], f[6], f[7]));
  } else {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (OUT == ES_DTYPE_F16) {
        r[i] = h2_bits(__floats2half2_rn(f[2 * i], f[2 * i + 1]));
      } else {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        r[i] = *reinterpret_cast<const uint32_t*>(&b);
      }
    }
    __stcs(reinterpret_cast<uint4*>(dst) + item, make_uint4(r[0], r[1], r[2], r[3]));
  }
}

// A thread takes 8 values of K and of V at ROUNDS places a block apart, all loads under way together: 8 bytes in, 16 out,
// neighbouring threads side by side in the output and, within a row of a head, in the page.
template <int HD, int CODE, int OUT>
__global__ void __launch_bounds__(GATHER_THREADS) kv8_gather_kernel(const GatherParams p) {
  constexpr int PPR = HD / 8, ROUNDS = 2;
  uint2 a[ROUNDS], b[ROUNDS];
  float sa[ROUNDS], sb[ROUNDS];
  int slot[ROUNDS];
  const int64_t first = (int64_t)blockIdx.x * (ROUNDS * GATHER_THREADS) + threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int64_t item = first + i * GATHER_THREADS;
    slot[i] = item < p.n_items ? p.slots[(unsigned)(item / PPR) / (unsigned)p.Hkv] : -1;
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int64_t item = first + i * GATHER_THREADS;
    const unsigned rh = (unsigned)(item / PPR);             // rows * heads fit 32 bits
    const int part = (int)(item % PPR), h = (int)(rh % (unsigned)p.Hkv);
    a[i] = b[i] = make_uint2(0, 0);
    sa[i] = sb[i] = 0.f;
    if (slot[i] >= 0 && slot[i] < p.n_pages * p.P) {
      const int page = slot[i] >> p.log2P, off = slot[i] & (p.P - 1);
      const int64_t ph = (int64_t)page * p.Hkv + h;
      const int64_t at = (ph * p.P + off) * HD + part * 8;
      a[i] = __ldcs(reinterpret_cast<const uint2*>(p.k_pages + at));
      b[i] = __ldcs(reinterpret_cast<const uint2*>(p.v_pages + at));
      sa[i] = p.k_scale[ph];
      sb[i] = p.v_scale[ph];
    }
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int64_t item = first + i * GATHER_THREADS;
    if (item >= p.n_items) break;
    store_values<CODE, OUT>(p.k, item, a[i], sa[i]);
    store_values<CODE, OUT>(p.v, item, b[i], sb[i]);
  }
}

template <int HD, int CODE>
es_status_t launch_gather(const GatherParams& p, int out, cudaStream_t s) {
  const int64_t blocks = (p.n_items + 2 * GATHER_THREADS - 1) / (2 * GATHER_THREADS);
  if (blocks > INT32_MAX || p.n_items / (HD / 8) > UINT32_MAX) return fail(ES_ERR_RANGE, "too many rows for one launch");
  const dim3 grid((unsigned)blocks);
  switch (out) {
    case ES_DTYPE_F16: ES_CUDA_CHECK(launch_kernel(kv8_gather_kernel<HD, CODE, ES_DTYPE_F16>, grid, dim3(GATHER_THREADS), 0, s, tunables().pdl != 0, p)); break;
    case ES_DTYPE_BF16: ES_CUDA_CHECK(launch_kernel(kv8_gather_kernel<HD, CODE, ES_DTYPE_BF16>, grid, dim3(GATHER_THREADS), 0, s, tunables().pdl != 0, p)); break;
    default: ES_CUDA_CHECK(launch_kernel(kv8_gather_kernel<HD, CODE, ES_DTYPE_F32>, grid, dim3(GATHER_THREADS), 0, s, tunables().pdl != 0, p));
  }
  ES_CUDA_CHECK(cudaGetLastError());
  return ES_OK;
}

}  // namespace

es_status_t kv8_check_pool(int32_t code_dtype, int32_t Hkv, int32_t hd, int32_t page_tokens, int32_t n_pages, int* code) {
  if (!kv8_code_of(code_dtype, code)) return fail(ES_ERR_INVALID_ARG, "code_dtype must be ES_DTYPE_I8 or ES_DTYPE_F8E4M3");
  if (Hkv <= 0 || hd <= 0 || page_tokens <= 0 || n_pages <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (hd != 64 && hd != 128) return fail(ES_ERR_SHAPE, "head_dim must be 64 or 128");
  if (page_tokens < 16 || (page_tokens & (page_tokens - 1))) return fail(ES_ERR_SHAPE, "page_tokens must be a power of two >= 16");
  if ((long long)n_pages * page_tokens > INT32_MAX) return fail(ES_ERR_RANGE, "n_pages * page_tokens exceeds 2^31 - 1");
  return ES_OK;
}

}  // namespace es

extern "C" {

es_status_t es_op_kv8_append(const void* k, const void* v, int32_t dtype, int64_t row_stride, int32_t n_rows,
                             const int32_t* slot_map, const int32_t* runs, int32_t n_runs, void* k_pages, void* v_pages,
                             int32_t code_dtype, float* k_scale, float* v_scale, int32_t Hkv, int32_t hd,
                             int32_t page_tokens, int32_t n_pages, void* stream) {
  using namespace es;
  int code = 0;
  if (n_rows < 0 || n_runs < 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (dtype != ES_DTYPE_F16 && dtype != ES_DTYPE_BF16) return fail(ES_ERR_INVALID_ARG, "k and v must be fp16 or bf16");
  ES_TRY(kv8_check_pool(code_dtype, Hkv, hd, page_tokens, n_pages, &code));
  if (n_rows == 0 || (runs && n_runs == 0)) return ES_OK;
  if (!k || !v || !slot_map || !k_pages || !v_pages || !k_scale || !v_scale) return fail(ES_ERR_INVALID_ARG, "null argument");
  if (row_stride < (int64_t)Hkv * hd || row_stride % 8) return fail(ES_ERR_INVALID_ARG, "row_stride must be a multiple of 8, at least Hkv * hd");
  if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_pages | (uintptr_t)v_pages) % 16) return fail(ES_ERR_INVALID_ARG, "rows and pages must be 16-byte aligned");
  AppendParams p{(const uint16_t*)k, (const uint16_t*)v, row_stride, slot_map, runs, n_rows, runs ? n_runs : n_rows,
                 (uint8_t*)k_pages, (uint8_t*)v_pages, k_scale, v_scale, Hkv, page_tokens, 0, n_pages};
  while ((1 << p.log2P) < page_tokens) ++p.log2P;
  const bool wide = runs ? n_rows >= 8 * (int64_t)n_runs : false;
  const bool bf16 = dtype == ES_DTYPE_BF16;
  cudaStream_t s = (cudaStream_t)stream;
  if (hd == 128) {
    if (code == CODE_I8) return bf16 ? launch_append<128, CODE_I8, true>(p, wide, s) : launch_append<128, CODE_I8, false>(p, wide, s);
    return bf16 ? launch_append<128, CODE_E4M3, true>(p, wide, s) : launch_append<128, CODE_E4M3, false>(p, wide, s);
  }
  if (code == CODE_I8) return bf16 ? launch_append<64, CODE_I8, true>(p, wide, s) : launch_append<64, CODE_I8, false>(p, wide, s);
  return bf16 ? launch_append<64, CODE_E4M3, true>(p, wide, s) : launch_append<64, CODE_E4M3, false>(p, wide, s);
}

es_status_t es_op_kv8_gather(const int32_t* slot_map, int32_t n_rows, const void* k_pages, const void* v_pages,
                             int32_t code_dtype, const float* k_scale, const float* v_scale, int32_t Hkv, int32_t hd,
                             int32_t page_tokens, int32_t n_pages, void* k, void* v, int32_t dtype, void* stream) {
  using namespace es;
  int code = 0;
  if (n_rows < 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (dtype != ES_DTYPE_F16 && dtype != ES_DTYPE_BF16 && dtype != ES_DTYPE_F32)
    return fail(ES_ERR_INVALID_ARG, "k and v must be fp16, bf16 or fp32");
  ES_TRY(kv8_check_pool(code_dtype, Hkv, hd, page_tokens, n_pages, &code));
  if (n_rows == 0) return ES_OK;
  if (!slot_map || !k_pages || !v_pages || !k_scale || !v_scale || !k || !v) return fail(ES_ERR_INVALID_ARG, "null argument");
  if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_pages | (uintptr_t)v_pages) % 16) return fail(ES_ERR_INVALID_ARG, "rows and pages must be 16-byte aligned");
  GatherParams p{slot_map, (const uint8_t*)k_pages, (const uint8_t*)v_pages, k_scale, v_scale, k, v,
                 (int64_t)n_rows * Hkv * (hd / 8), Hkv, page_tokens, 0, n_pages};
  while ((1 << p.log2P) < page_tokens) ++p.log2P;
  cudaStream_t s = (cudaStream_t)stream;
  if (hd == 128) return code == CODE_I8 ? launch_gather<128, CODE_I8>(p, dtype, s) : launch_gather<128, CODE_E4M3>(p, dtype, s);
  return code == CODE_I8 ? launch_gather<64, CODE_I8>(p, dtype, s) : launch_gather<64, CODE_E4M3>(p, dtype, s);
}

}  // extern "C"
