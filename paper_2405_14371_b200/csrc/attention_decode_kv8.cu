// Split-KV decode attention over the paged 8-bit cache (mma.sync m16n8k16), for one or a few query tokens per sequence.
//
// The bound is reading every code of K and V once.  A KV head's query rows (T tokens x G heads of the group) form row
// tiles of 8 (NT = 1) or 16 (NT = 2); a CTA takes one split of one sequence's keys for one row tile, its four warps
// every fourth block of 16 tokens each:
//
//   * codes go from global memory to registers with 16-byte loads and become fp16 there, which holds every code of both
//     types exactly; the contraction visits the head's dimensions in whatever order the bytes arrive in, and the query
//     fragments are gathered with the same permutation, so nothing passes through shared memory;
//   * scores S[row, token]: A = query rows, B = K.  The scale of K's page, 1/sqrt(hd) and the query's own exponent are
//     factors of the finished score;
//   * softmax per block against the block's own maximum, in fp32: the probabilities lie in [0, 1] whatever the other
//     pages hold, and enter the next product as two fp16 halves (hi + lo, together 22 bits), so that rounding them costs
//     the output nothing next to its own;
//   * O^T[dim, row] = V^T P^T into a block accumulator, which joins the running sum with the factor
//     (scale of V's page) * exp(block maximum - new maximum): pages of very different scales cannot wash each other out.
//
// bf16 queries are brought to fp16 by a power of two per row (largest magnitude to [1, 2)): 11 bits hold bf16's 8, and
// what underflows is below 2^-24 of the row's largest.
//
// A block lies in one page (P >= 16).  Codes behind the context are zeroed in V and masked by selection in the scores, so
// that garbage (NaN codes among it) never meets a product; a page whose scale is NaN makes the rows that see it NaN.
// Splits are merged in order by a second kernel.
#include "es_internal.cuh"
#include "kv8.cuh"
#include "launch.cuh"

namespace es {
namespace {

constexpr int AW = 4;                    // warps of a CTA

struct Kv8AttnParams {
  const void* q;
  int64_t q_stride;
  const uint8_t *k, *v;
  const float *ks, *vs;
  const int *table, *ctx_len;
  void* out;
  float *part_o, *part_ml;               // [B * T * Hq][n_splits][hd], [..][n_splits][2]
  int B, T, Hq, Hkv, G, P, log2P, pps, n_pages, max_ctx;
  int row_tiles, n_splits, tokens_per_split;
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint4 ld16(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.cg.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ld8(const uint8_t* p) {
  uint2 v;
  asm volatile("ld.global.cg.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

template <bool BF16>
__device__ __forceinline__ float2 pair_of(uint32_t w) {
  if (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  return __half22float2(bits_h2(w));
}

template <bool BF16>
__device__ __forceinline__ void store_out(void* out, int64_t i, float x) {
  if (BF16) reinterpret_cast<__nv_bfloat16*>(out)[i] = __float2bfloat16_rn(x);
  else reinterpret_cast<__half*>(out)[i] = __float2half_rn(x);
}

template <int HD, int CODE, bool BF16, int NT>
__global__ void __launch_bounds__(AW * 32, NT == 1 ? 3 : 2) kv8_attn_kernel(const Kv8AttnParams p) {
  pdl_launch_dependents();
  constexpr int J = HD / 64;             // 16-byte pieces of a K row per thread
  constexpr int D = HD / 8;              // dimensions of V per thread
  constexpr int NM = D / 2;              // output MMAs
  constexpr int ROWS = 8 * NT;
  constexpr float LOG2E = 1.4426950408889634f;
  __shared__ float sm_o[AW][ROWS][HD];
  __shared__ float sm_m[AW][ROWS], sm_l[AW][ROWS];

  const int split = blockIdx.x;
  const int kvh = blockIdx.y / p.row_tiles, tile = blockIdx.y - kvh * p.row_tiles, b = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n_rows = p.T * p.G;
  const int ctx = max(0, min(p.ctx_len[b], p.max_ctx));
  const int t_begin = split * p.tokens_per_split;
  if (t_begin >= ctx && split > 0) return;               // nothing to read and nobody reads its part (split 0 answers for empty contexts)
  const int t_end = (int)min((long long)ctx, (long long)t_begin + p.tokens_per_split);

  // row r of the tile: query token (r / G), head kvh * G + r % G; it sees keys below `limit`
  auto row_of = [&](int r, int& token, int& head) { const int i = tile * ROWS + r; token = i / p.G; head = kvh * p.G + i - token * p.G; return i < n_rows; };
  int limit[NT];
  float qscale[NT];
  uint32_t qa[NT][8 * J];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    int token, head;
    const bool real = row_of(8 * n + g, token, head);
    limit[n] = real ? ctx - p.T + token + 1 : 0;
    qscale[n] = 1.f;
    const uint16_t* row = reinterpret_cast<const uint16_t*>(p.q) + ((int64_t)b * p.T + token) * p.q_stride + (int64_t)head * HD;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      uint4 x = make_uint4(0, 0, 0, 0), y = x;
      if (real) { x = *reinterpret_cast<const uint4*>(row + (4 * j + t) * 16); y = *reinterpret_cast<const uint4*>(row + (4 * j + t) * 16 + 8); }
      qa[n][8 * j] = x.x; qa[n][8 * j + 1] = x.y; qa[n][8 * j + 2] = x.z; qa[n][8 * j + 3] = x.w;
      qa[n][8 * j + 4] = y.x; qa[n][8 * j + 5] = y.y; qa[n][8 * j + 6] = y.z; qa[n][8 * j + 7] = y.w;
    }
    if (BF16) {
      uint32_t mx = 0;
#pragma unroll
      for (int i = 0; i < 8 * J; ++i) mx = __vmaxu2(mx, qa[n][i] & 0x7fff7fffu);
      mx = max(mx & 0xffffu, mx >> 16);
      mx = max(mx, __shfl_xor_sync(~0u, mx, 1));
      mx = max(mx, __shfl_xor_sync(~0u, mx, 2));
      // 2^-e and 2^e with e the exponent of the largest magnitude, kept where both are normal numbers
      const int e = min(max((int)(mx >> 7) - 127, -126), 126);
      const float down = __uint_as_float((uint32_t)(127 - e) << 23);
      qscale[n] = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
      for (int i = 0; i < 8 * J; ++i) {
        const float2 f = pair_of<true>(qa[n][i]);
        qa[n][i] = h2_bits(__floats2half2_rn(f.x * down, f.y * down));
      }
    }
    qscale[n] *= rsqrtf((float)HD) * LOG2E;                // scores in units of log2
  }

  const int64_t head_bytes = (int64_t)p.P * HD;
  const int* table = p.table + (int64_t)b * p.pps;
  uint4 kreg[2][J];
  uint32_t vreg[4][D / 4];
  float k_s = 0.f, v_s = 0.f, k_n = 0.f, v_n = 0.f;        // scales of the block at hand and of the one being loaded
  bool ok = false, ok_n = false;                           // whether their pages exist

  auto page_of = [&](int T0) -> int { return T0 < t_end ? table[T0 >> p.log2P] : -1; };
  auto load_k = [&](int T0, int page) {
    ok_n = page >= 0 && page < p.n_pages;
    if (!ok_n) return;
    const int64_t ph = (int64_t)page * p.Hkv + kvh;
    const uint8_t* base = p.k + ph * head_bytes + (int64_t)(T0 & (p.P - 1)) * HD;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int j = 0; j < J; ++j) kreg[nt][j] = ld16(base + (8 * nt + g) * HD + (4 * j + t) * 16);
    k_n = p.ks[ph];
    v_n = p.vs[ph];
  };
  auto load_v = [&](int T0, int page) {
    if (page < 0 || page >= p.n_pages) return;
    const uint8_t* base = p.v + ((int64_t)page * p.Hkv + kvh) * head_bytes + (int64_t)(T0 & (p.P - 1)) * HD;
    const int left = ctx - T0;
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int r = 2 * t + (q4 & 1) + 8 * (q4 >> 1);
      if constexpr (HD == 128) {
        const uint4 x = r < left ? ld16(base + r * HD + g * 16) : make_uint4(0, 0, 0, 0);
        vreg[q4][0] = x.x; vreg[q4][1] = x.y; vreg[q4][2] = x.z; vreg[q4][3] = x.w;
      } else {
        const uint2 x = r < left ? ld8(base + r * HD + g * 8) : make_uint2(0, 0);
        vreg[q4][0] = x.x; vreg[q4][1] = x.y;
      }
    }
  };

  float o[NT][NM][4];
  float m_run[NT], l_run[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m_run[n] = -INFINITY; l_run[n] = 0.f;
#pragma unroll
    for (int i = 0; i < NM; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
  }

  constexpr int STEP = AW * 16;
  int T0 = t_begin + warp * 16;
  int page = page_of(T0), page_next = page_of(T0 + STEP);
  load_k(T0, page);
  load_v(T0, page);
  for (; T0 < t_end; T0 += STEP) {
    ok = ok_n; k_s = k_n; v_s = v_n;
    page = page_next;
    page_next = page_of(T0 + 2 * STEP);
    if (!ok) {                                             // a page nobody sees (uniform over the warp)
      load_k(T0 + STEP, page);
      load_v(T0 + STEP, page);
      continue;
    }
    // ---- scores: rows g (and 8 + g), tokens T0 + 8 nt + 2 t + {0, 1} ----
    float s[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t w[4] = {kreg[nt][j].x, kreg[nt][j].y, kreg[nt][j].z, kreg[nt][j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t lo, hi;
          codes_to_h2<CODE>(w[i], lo, hi);
          mma(s[nt], qa[0][8 * j + 2 * i], NT == 2 ? qa[NT - 1][8 * j + 2 * i] : 0u, qa[0][8 * j + 2 * i + 1],
              NT == 2 ? qa[NT - 1][8 * j + 2 * i + 1] : 0u, lo, hi);
        }
      }
    }
    load_k(T0 + STEP, page);
    // ---- softmax of the block ----
    uint32_t ph[NT][2], pl[NT][2];                         // probabilities, hi and lo halves: the B fragments of the output MMAs
    float alpha[NT], beta[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float x[4], mx = -INFINITY;
      const float f = qscale[n] * k_s;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int tok = T0 + 8 * (e >> 1) + 2 * t + (e & 1);
        x[e] = tok < limit[n] ? s[e >> 1][2 * n + (e & 1)] * f : -INFINITY;
        mx = fmaxf(mx, x[e]);
      }
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 2));
      const bool sees = T0 < limit[n];
      const float ref = mx == -INFINITY ? 0.f : mx;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[e] = ex2(x[e] - ref); sum += x[e]; }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
        const float2 back = __half22float2(h);
        ph[n][i] = h2_bits(h);
        pl[n][i] = h2_bits(__floats2half2_rn(x[2 * i] - back.x, x[2 * i + 1] - back.y));
      }
      sum += __shfl_xor_sync(~0u, sum, 1);
      sum += __shfl_xor_sync(~0u, sum, 2);
      const float mn = fmaxf(m_run[n], mx);
      const float to = mn == -INFINITY ? 0.f : mn;
      alpha[n] = ex2(m_run[n] - to);
      const float join = sees ? ex2(ref - to) : 0.f;       // NaN scores pass through: they are in `sum` and in the product
      beta[n] = sees ? join * v_s : 0.f;
      l_run[n] = sees ? l_run[n] * alpha[n] + sum * join : l_run[n];
      m_run[n] = mn;
    }
    // ---- output: MMA i gives dimensions D g + i (rows 0..7) and D g + D / 2 + i (rows 8..15) ----
    float al[NT][2], be[NT][2];                            // factors of rows 2 t and 2 t + 1
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        al[n][i] = __shfl_sync(~0u, alpha[n], (2 * t + i) * 4);
        be[n][i] = __shfl_sync(~0u, beta[n], (2 * t + i) * 4);
      }
    #pragma unroll
    for (int w = 0; w < D / 8; ++w) {
      uint32_t a[4][4];                                    // A registers 0..3 of four MMAs
#pragma unroll
      for (int q2 = 0; q2 < 2; ++q2)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t x = vreg[2 * q2][w + half * (D / 8)], y = vreg[2 * q2 + 1][w + half * (D / 8)];
          codes_to_h2<CODE>(__byte_perm(x, y, 0x5140), a[2 * q2 + half][0], a[2 * q2 + half][1]);
          codes_to_h2<CODE>(__byte_perm(x, y, 0x7362), a[2 * q2 + half][2], a[2 * q2 + half][3]);
        }
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float c[4] = {0.f, 0.f, 0.f, 0.f};
          mma(c, a[0][d], a[1][d], a[2][d], a[3][d], ph[n][0], ph[n][1]);
          mma(c, a[0][d], a[1][d], a[2][d], a[3][d], pl[n][0], pl[n][1]);
          float (&acc)[4] = o[n][4 * w + d];
          acc[0] = acc[0] * al[n][0] + c[0] * be[n][0];
          acc[1] = acc[1] * al[n][1] + c[1] * be[n][1];
          acc[2] = acc[2] * al[n][0] + c[2] * be[n][0];
          acc[3] = acc[3] * al[n][1] + c[3] * be[n][1];
        }
    }
    load_v(T0 + STEP, page);
  }

  // ---- the warps' parts join in warp order ----
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      sm_o[warp][8 * n + 2 * t][D * g + i] = o[n][i][0];
      sm_o[warp][8 * n + 2 * t + 1][D * g + i] = o[n][i][1];
      sm_o[warp][8 * n + 2 * t][D * g + D / 2 + i] = o[n][i][2];
      sm_o[warp][8 * n + 2 * t + 1][D * g + D / 2 + i] = o[n][i][3];
    }
    if (t == 0) { sm_m[warp][8 * n + g] = m_run[n]; sm_l[warp][8 * n + g] = l_run[n]; }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < ROWS * HD; i += AW * 32) {
    const int r = i / HD, c = i - r * HD;
    int token, head;
    if (!row_of(r, token, head)) break;
    float mm = sm_m[0][r];
#pragma unroll
    for (int w = 1; w < AW; ++w) mm = fmaxf(mm, sm_m[w][r]);
    const float ref = mm == -INFINITY ? 0.f : mm;
    float acc = 0.f, ll = 0.f;
#pragma unroll
    for (int w = 0; w < AW; ++w) {
      const float f = ex2(sm_m[w][r] - ref);
      acc += sm_o[w][r][c] * f;
      ll += sm_l[w][r] * f;
    }
    const int64_t row = ((int64_t)b * p.T + token) * p.Hq + head;
    if (p.n_splits == 1) {
      store_out<BF16>(p.out, row * HD + c, ll == 0.f ? 0.f : acc / ll);
    } else {
      p.part_o[(row * p.n_splits + split) * HD + c] = acc;
      if (c == 0) *reinterpret_cast<float2*>(p.part_ml + (row * p.n_splits + split) * 2) = make_float2(mm, ll);
    }
  }
}

// One warp per output row: the splits that hold keys, in ascending order.
template <int HD, bool BF16>
__global__ void __launch_bounds__(128) kv8_merge_kernel(const Kv8AttnParams p) {
  constexpr int V = HD / 32;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  pdl_wait();
  if (row >= (int64_t)p.B * p.T * p.Hq) return;
  const int b = (int)(row / ((int64_t)p.T * p.Hq));
  const int ctx = max(0, min(p.ctx_len[b], p.max_ctx));
  const int active = max(1, (ctx + p.tokens_per_split - 1) / p.tokens_per_split);
  const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + row * p.n_splits;
  const float* po = p.part_o + row * p.n_splits * HD + lane * V;
  float mm = -INFINITY;
  for (int i = lane; i < active; i += 32) mm = fmaxf(mm, __ldcg(&ml[i]).x);
#pragma unroll
  for (int d = 16; d; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(~0u, mm, d));
  const float ref = mm == -INFINITY ? 0.f : mm;
  float acc[V], ll = 0.f;
#pragma unroll
  for (int c = 0; c < V; ++c) acc[c] = 0.f;
#pragma unroll 4
  for (int i = 0; i < active; ++i) {
    const float2 x = __ldcg(&ml[i]);
    const float f = ex2(x.x - ref);
    ll += x.y * f;
#pragma unroll
    for (int c = 0; c < V; ++c) acc[c] += __ldcg(po + (int64_t)i * HD + c) * f;
  }
#pragma unroll
  for (int c = 0; c < V; ++c) store_out<BF16>(p.out, row * HD + lane * V + c, ll == 0.f ? 0.f : acc[c] / ll);
}

struct Split { int row_tiles, nt, n_splits, tokens; };

Split choose_kv8_split(int B, int T, int Hq, int Hkv, int max_ctx) {
  Split s;
  const int rows = T * (Hq / Hkv);
  s.nt = rows > 8 ? 2 : 1;
  s.row_tiles = (rows + 8 * s.nt - 1) / (8 * s.nt);
  const long long items = (long long)B * Hkv * s.row_tiles;
  long long n = (3LL * sm_count() + items - 1) / items;
  const int unit = AW * 16;
  long long tokens = (max_ctx + n - 1) / n;
  if (tokens < 256) tokens = 256;
  tokens = (tokens + unit - 1) / unit * unit;
  if (tokens > max_ctx) tokens = (max_ctx + unit - 1) / unit * unit;
  s.tokens = (int)tokens;
  s.n_splits = (int)((max_ctx + tokens - 1) / tokens);
  return s;
}

size_t part_bytes(const Split& s, int B, int T, int Hq, int hd) {
  return s.n_splits > 1 ? (size_t)B * T * Hq * s.n_splits * (hd + 2) * sizeof(float) : 0;
}

template <int HD, int CODE, bool BF16>
es_status_t launch(const Kv8AttnParams& p, int nt, cudaStream_t s) {
  const dim3 grid(p.n_splits, p.Hkv * p.row_tiles, p.B);
  if (nt == 1) ES_CUDA_CHECK(launch_kernel(kv8_attn_kernel<HD, CODE, BF16, 1>, grid, dim3(AW * 32), 0, s, false, p));
  else ES_CUDA_CHECK(launch_kernel(kv8_attn_kernel<HD, CODE, BF16, 2>, grid, dim3(AW * 32), 0, s, false, p));
  if (p.n_splits > 1) {
    const long long rows = (long long)p.B * p.T * p.Hq;
    ES_CUDA_CHECK(launch_kernel(kv8_merge_kernel<HD, BF16>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, s, true, p));
  }
  return ES_OK;
}

es_status_t check_heads(int B, int T, int Hq, int Hkv, int hd, int page_tokens, int max_ctx) {
  if (B <= 0 || T <= 0 || Hq <= 0 || Hkv <= 0 || hd <= 0 || page_tokens <= 0 || max_ctx <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (Hq % Hkv != 0) return fail(ES_ERR_SHAPE, "Hq must be a multiple of Hkv");
  if (hd != 64 && hd != 128) return fail(ES_ERR_SHAPE, "head_dim must be 64 or 128");
  const long long rows = (long long)T * (Hq / Hkv);
  if (max_ctx > (1 << 30)) return fail(ES_ERR_RANGE, "max_ctx exceeds 2^30");
  if (B > 65535 || rows > 65535 || (rows + 15) / 16 * Hkv > 32767 || (long long)B * T * Hq > (1LL << 30))
    return fail(ES_ERR_RANGE, "B, T or the head counts exceed one launch");
  return ES_OK;
}

}  // namespace
}  // namespace es

extern "C" {

size_t es_op_decode_attention_kv8_scratch_bytes(int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t hd,
                                                int32_t page_tokens, int32_t max_ctx) {
  using namespace es;
  if (check_heads(B, T, Hq, Hkv, hd, page_tokens, max_ctx) != ES_OK) return 0;
  return part_bytes(choose_kv8_split(B, T, Hq, Hkv, max_ctx), B, T, Hq, hd);
}

es_status_t es_op_decode_attention_kv8(const void* q, int32_t dtype, int64_t q_stride, const void* k_pages,
                                       const void* v_pages, int32_t code_dtype, const float* k_scale,
                                       const float* v_scale, const int32_t* block_table, const int32_t* ctx_len,
                                       void* out, int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t hd,
                                       int32_t page_tokens, int32_t pages_per_seq, int32_t n_pages, int32_t max_ctx,
                                       void* scratch, size_t scratch_bytes, void* stream) {
  using namespace es;
  int code = 0;
  if (!q || !k_pages || !v_pages || !k_scale || !v_scale || !block_table || !ctx_len || !out) return fail(ES_ERR_INVALID_ARG, "null argument");
  if (dtype != ES_DTYPE_F16 && dtype != ES_DTYPE_BF16) return fail(ES_ERR_INVALID_ARG, "q must be fp16 or bf16");
  ES_TRY(check_heads(B, T, Hq, Hkv, hd, page_tokens, max_ctx));
  ES_TRY(kv8_check_pool(code_dtype, Hkv, hd, page_tokens, n_pages, &code));
  if (pages_per_seq <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if ((long long)max_ctx > (long long)page_tokens * pages_per_seq) return fail(ES_ERR_RANGE, "max_ctx exceeds the block table");
  if (q_stride < (int64_t)Hq * hd || q_stride % 8) return fail(ES_ERR_INVALID_ARG, "q_stride must be a multiple of 8, at least Hq * hd");
  if (((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)scratch) % 16)
    return fail(ES_ERR_INVALID_ARG, "q, pages and scratch must be 16-byte aligned");
  const Split sp = choose_kv8_split(B, T, Hq, Hkv, max_ctx);
  const size_t need = part_bytes(sp, B, T, Hq, hd);
  if (scratch_bytes < need || (need && !scratch)) return fail(ES_ERR_WORKSPACE, "scratch: %zu bytes given, %zu needed", scratch ? scratch_bytes : (size_t)0, need);
  int log2P = 0;
  while ((1 << log2P) < page_tokens) ++log2P;
  const size_t rows = (size_t)B * T * Hq;
  Kv8AttnParams p{q, q_stride, (const uint8_t*)k_pages, (const uint8_t*)v_pages, k_scale, v_scale, block_table, ctx_len, out,
                  (float*)scratch, (float*)scratch + rows * sp.n_splits * hd, B, T, Hq, Hkv, Hq / Hkv, page_tokens, log2P,
                  pages_per_seq, n_pages, max_ctx, sp.row_tiles, sp.n_splits, sp.tokens};
  const bool bf16 = dtype == ES_DTYPE_BF16;
  cudaStream_t s = (cudaStream_t)stream;
  if (hd == 128) {
    if (code == CODE_I8) return bf16 ? launch<128, CODE_I8, true>(p, sp.nt, s) : launch<128, CODE_I8, false>(p, sp.nt, s);
    return bf16 ? launch<128, CODE_E4M3, true>(p, sp.nt, s) : launch<128, CODE_E4M3, false>(p, sp.nt, s);
  }
  if (code == CODE_I8) return bf16 ? launch<64, CODE_I8, true>(p, sp.nt, s) : launch<64, CODE_I8, false>(p, sp.nt, s);
  return bf16 ? launch<64, CODE_E4M3, true>(p, sp.nt, s) : launch<64, CODE_E4M3, false>(p, sp.nt, s);
}

}  // extern "C"
