// Products with block-scaled e4m3 operands on the tensor cores (tcgen05 kind::f8f6f4, TMA, TMEM).
//
//   C[m, n] = sum over blocks b of 128 columns:  sa[b, m] * sw[n / 128, b] * sum over k in b:  A[m, k] * W[n, k]     (+ R[m, n])
//
// The codes of a block are multiplied and added by one accumulation of 4 MMAs in TMEM (K = 32 each); the scales differ from
// block to block, so each block's sums are read back and join the running fp32 sums of the result in registers,
// acc = fma(sums, sa * sw, acc), while the tensor cores work on the next block into another TMEM buffer.
//
// Two kernels:
//
//   * tiles of 128 weight rows (few tokens).  The weights are the M side of the MMA, 16 to 128 tokens its N side, so a decode
//     batch wastes no tensor-core rows on absent tokens and a block costs a thread 16 to 64 multiply-adds.  Bound: reading
//     the weights once.  The K range of a tile is shared by a cluster of 1 to 8 CTAs so that the machine is full in one wave;
//     their sums meet in distributed shared memory and are added in rank order, so the result depends on the sizes and the
//     device (how many clusters it holds) alone.
//   * 256 x 256 tiles on CTA pairs (many tokens): cta_group::2, each CTA stages 128 rows of A and 128 of W per block and
//     keeps 128 x 256 running sums in the registers of 8 warps (128 each).  Where tiles are few, two or four pairs share a
//     tile's K range and join their sums the same way.  Bound: the tensor cores' e4m3 rate, and the power it draws.
//
// Every wait is bounded by a second; the tiles of a CTA whose wait ran out become NaN.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>

#include "es_internal.cuh"
#include "fp8.cuh"
#include "launch.cuh"
#include "sm100.cuh"

namespace cg = cooperative_groups;

namespace es {
namespace {

struct alignas(64) Fp8Maps { CUtensorMap a, w; };

struct Fp8Params {
  const float *as, *ws;      // [K blocks, M], [N blocks, K blocks]
  const float* R;            // [M, N] or nullptr
  void* C;
  int M, N, nkb;
  int out;                   // ES_DTYPE_*
  int ready;                 // the weights may be read before the kernel in front has ended
  int vec;                   // rows of C (and R) start on multiples of 16 bytes
};

constexpr int BKB = 128;                         // bytes (= codes) of a row per block
constexpr int W_TILE = 128 * BKB;

// Results of one weight row, of tokens m, m + step, ... < m1.  The residual of all is asked for before the first is stored (it may
// be where the result goes, so the compiler keeps the order: token by token, 113 of them waited 8 us).
template <int MANY>
__device__ __forceinline__ void store_many(const Fp8Params& p, int n, int m, int step, int m1, const float* v) {
  const int64_t at = (int64_t)m * p.N + n, far = (int64_t)step * p.N;
  if (p.out == ES_DTYPE_F32) {
    float r[MANY];
#pragma unroll
    for (int q = 0; q < MANY; ++q) r[q] = p.R && m + q * step < m1 ? p.R[at + q * far] : 0.f;
#pragma unroll
    for (int q = 0; q < MANY; ++q)
      if (m + q * step < m1) ((float*)p.C)[at + q * far] = p.R ? v[q] + r[q] : v[q];
  } else if (p.out == ES_DTYPE_F16) {
#pragma unroll
    for (int q = 0; q < MANY; ++q)
      if (m + q * step < m1) ((__half*)p.C)[at + q * far] = __float2half_rn(v[q]);
  } else {
#pragma unroll
    for (int q = 0; q < MANY; ++q)
      if (m + q * step < m1) ((__nv_bfloat16*)p.C)[at + q * far] = __float2bfloat16_rn(v[q]);
  }
}

// ---- tiles of 128 weight rows x NT tokens ----------------------------------------------------------

template <int NT> struct RowsCfg {
  static constexpr int OCC = NT <= 64 ? 2 : 1;                       // CTAs per SM
  static constexpr int SUMS = NT <= 32 ? 4 : 8;                      // warps of sums; a thread has one weight row
  static constexpr int MINE = NT * 4 / SUMS;                         // and so many tokens
  static constexpr int THREADS = 128 + 32 * SUMS;                    // TMA, MMA, factors, an idle warp
  static constexpr int X_TILE = NT * BKB;
  static constexpr int STAGE = W_TILE + X_TILE;
  static constexpr int STAGES = (OCC == 2 ? 108 * 1024 : 200 * 1024) / STAGE;
  static constexpr int BUFS = 4;                                     // TMEM buffers
  static constexpr int COLS = BUFS * NT;                             // 64 to 512, a power of two
  static constexpr int FACTORS = 8;                                  // blocks whose factors are in shared memory
  static constexpr int BARS = 2 * STAGES + 2 * BUFS + 2 * FACTORS;
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + FACTORS * NT * 4 + BARS * 8 + 16;
  static_assert(STAGES * STAGE >= 128 * NT * 4, "the running sums of a CTA go where the ring was");
};

template <int NT>
__global__ void __launch_bounds__(RowsCfg<NT>::THREADS, RowsCfg<NT>::OCC) linear_fp8_rows_kernel(const __grid_constant__ Fp8Maps maps, const Fp8Params p, const int split) {
  using L = RowsCfg<NT>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char* ring = smem;                                          // stage: weight tile, token tile
  float* factor = (float*)(smem + L::STAGES * L::STAGE);               // [FACTORS][NT] sa * sw of a block
  uint64_t* bars = (uint64_t*)(factor + L::FACTORS * NT);
  uint64_t *full = bars, *empty = full + L::STAGES, *acc_full = empty + L::STAGES, *acc_empty = acc_full + L::BUFS, *fac_full = acc_empty + L::BUFS,
           *fac_empty = fac_full + L::FACTORS;
  uint32_t* tmem_slot = (uint32_t*)(bars + L::BARS);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)blockIdx.x % split, n0 = ((int)blockIdx.x / split) * 128, m0 = (int)blockIdx.y * NT;
  const int b0 = (int)((long long)p.nkb * rank / split), blocks = (int)((long long)p.nkb * (rank + 1) / split) - b0;

  if (threadIdx.x == 0) {
    prefetch_tmap(&maps.a);
    prefetch_tmap(&maps.w);
    for (int s = 0; s < L::STAGES; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), 1); }
    for (int s = 0; s < L::BUFS; ++s) { mbar_init(smem_u32(&acc_full[s]), 1); mbar_init(smem_u32(&acc_empty[s]), L::SUMS); }
    for (int s = 0; s < L::FACTORS; ++s) { mbar_init(smem_u32(&fac_full[s]), 1); mbar_init(smem_u32(&fac_empty[s]), L::SUMS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), L::COLS);
  tc_fence_before();
  __syncthreads();
  pdl_launch_dependents();          // every CTA has its TMEM before a kernel behind this one can take any and then wait for this one's end
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  const int col0 = warp >= 4 ? ((warp - 4) >> 2) * L::MINE : 0;         // first token of a thread of sums
  float acc[L::MINE];
  if (warp == 0) {
    if (lane == 0) {
      // ---- TMA: weights of the first stages ahead of the wait for the kernel in front, if they are known to be complete ----
      const int early = min(blocks, L::STAGES);
      for (int i = 0; i < early; ++i) {
        mbar_expect_tx(smem_u32(&full[i]), L::STAGE);
        if (p.ready) tma_load_2d(smem_u32(ring + i * L::STAGE), &maps.w, (b0 + i) * (BKB / 2), n0, smem_u32(&full[i]));
      }
      pdl_wait();
      for (int i = 0; i < early; ++i) {
        if (!p.ready) tma_load_2d(smem_u32(ring + i * L::STAGE), &maps.w, (b0 + i) * (BKB / 2), n0, smem_u32(&full[i]));
        tma_load_2d(smem_u32(ring + i * L::STAGE + W_TILE), &maps.a, (b0 + i) * (BKB / 2), m0, smem_u32(&full[i]));
      }
      for (int i = early; i < blocks; ++i) {
        const int s = i % L::STAGES;
        if (!mbar_wait_soon(smem_u32(&empty[s]), ((i / L::STAGES) & 1) ^ 1, abort_flag)) break;
        const uint32_t fb = smem_u32(&full[s]);
        mbar_expect_tx(fb, L::STAGE);
        tma_load_2d(smem_u32(ring + s * L::STAGE), &maps.w, (b0 + i) * (BKB / 2), n0, fb);
        tma_load_2d(smem_u32(ring + s * L::STAGE + W_TILE), &maps.a, (b0 + i) * (BKB / 2), m0, fb);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      // ---- MMA ----
      constexpr uint32_t idesc = umma_idesc_f16(128, NT);
      const uint64_t w0 = umma_desc_sw128(smem_u32(ring)), x0 = umma_desc_sw128(smem_u32(ring) + W_TILE);
      const uint32_t full0 = smem_u32(full), empty0 = smem_u32(empty), acc_full0 = smem_u32(acc_full), acc_empty0 = smem_u32(acc_empty);
      uint32_t s = 0, ring_phase = 0, buf = 0, buf_phase = 1;
      pdl_wait();                                                       // the second that a wait may last is this kernel's alone
      for (int left = blocks; left > 0; --left) {
        if (!mbar_wait_soon(full0 + s * 8, ring_phase, abort_flag) || !mbar_wait_soon(acc_empty0 + buf * 8, buf_phase, abort_flag)) break;
        tc_fence_after();
        umma_f8_block(tmem + buf * NT, w0 + s * (L::STAGE >> 4), x0 + s * (L::STAGE >> 4), idesc);
        umma_commit(acc_full0 + buf * 8);
        umma_commit(empty0 + s * 8);
        if (++s == L::STAGES) { s = 0; ring_phase ^= 1; }
        if (++buf == L::BUFS) { buf = 0; buf_phase ^= 1; }
      }
    }
  } else if (warp == 2) {
    // ---- factors: fetched four blocks at a time, the next four on their way while these are handed on (with the loads in the
    // loop of the sums, every block waited for memory: 113 x 5120 x 13824 70 us) ----
    constexpr int PER = (NT + 31) / 32, BATCH = 4;
    const float* ws = p.ws + (int64_t)(n0 / FP8_BLOCK) * p.nkb + b0;
    const float* as = p.as + (int64_t)b0 * p.M + m0;
    pdl_wait();
    float sa[2][BATCH][PER], sw[2][BATCH];
    auto fetch = [&](int i0, float (&a)[BATCH][PER], float (&w)[BATCH]) {
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int i = i0 + q;
        w[q] = i < blocks ? ws[i] : 0.f;
#pragma unroll
        for (int t = 0; t < PER; ++t) {
          const int token = lane + 32 * t;
          a[q][t] = (i < blocks && token < NT && m0 + token < p.M) ? as[(int64_t)i * p.M + token] : 0.f;
        }
      }
    };
    auto hand_on = [&](int i0, const float (&a)[BATCH][PER], const float (&w)[BATCH]) {
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int i = i0 + q, slot = i % L::FACTORS;
        if (i >= blocks) break;
        if (!mbar_wait_soon(smem_u32(&fac_empty[slot]), ((i / L::FACTORS) & 1) ^ 1, abort_flag)) return;
#pragma unroll
        for (int t = 0; t < PER; ++t)
          if (lane + 32 * t < NT) factor[slot * NT + lane + 32 * t] = a[q][t] * w[q];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&fac_full[slot]));
      }
    };
    fetch(0, sa[0], sw[0]);
    for (int i = 0; i < blocks; i += 2 * BATCH) {
      fetch(i + BATCH, sa[1], sw[1]);
      hand_on(i, sa[0], sw[0]);
      fetch(i + 2 * BATCH, sa[0], sw[0]);
      hand_on(i + BATCH, sa[1], sw[1]);
    }
  } else if (warp >= 4) {
    // ---- sums ----
    const uint32_t taddr = tmem + col0 + ((uint32_t)((warp & 3) * 32) << 16);
    bool ok = true;
    pdl_wait();
#pragma unroll
    for (int j = 0; j < L::MINE; ++j) acc[j] = 0.f;
    for (int i = 0; i < blocks; ++i) {
      const int buf = i % L::BUFS, slot = i % L::FACTORS;
      ok = mbar_wait_soon(smem_u32(&fac_full[slot]), (i / L::FACTORS) & 1, abort_flag) &&
           mbar_wait_soon(smem_u32(&acc_full[buf]), (i / L::BUFS) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      constexpr int CH = L::MINE < 32 ? 16 : 32;
      const float* f = factor + slot * NT + col0;
#pragma unroll
      for (int c = 0; c < L::MINE; c += CH) {
        uint32_t v[CH];
        tmem_ld_issue(taddr + buf * NT + c, v);
        tmem_ld_wait(v);
        if (c + CH == L::MINE) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&acc_empty[buf]));
        }
#pragma unroll
        for (int j = 0; j < CH; j += 4) {
          const float4 q = *reinterpret_cast<const float4*>(f + c + j);
          acc[c + j] = fmaf(__uint_as_float(v[j]), q.x, acc[c + j]);
          acc[c + j + 1] = fmaf(__uint_as_float(v[j + 1]), q.y, acc[c + j + 1]);
          acc[c + j + 2] = fmaf(__uint_as_float(v[j + 2]), q.z, acc[c + j + 2]);
          acc[c + j + 3] = fmaf(__uint_as_float(v[j + 3]), q.w, acc[c + j + 3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&fac_empty[slot]));
    }
    if (!ok) {
#pragma unroll
      for (int j = 0; j < L::MINE; ++j) acc[j] = __uint_as_float(0x7fffffffu);
    }
  }

  // ---- teardown, and the sums of the cluster's CTAs ----
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    if (*abort_flag) settle();
    tmem_dealloc(tmem, L::COLS);
  }
  const int tokens = min(NT, p.M - m0);
  const int at = (warp & 3) * 32 + lane, n = n0 + at;                   // of the warps of sums: the weight row
  if (split == 1) {
    if (warp >= 4 && n < p.N) {
#pragma unroll
      for (int j = 0; j < L::MINE; j += 16) store_many<16>(p, n, m0 + col0 + j, 1, m0 + tokens, acc + j);
    }
    return;
  }
  float* sums = (float*)ring;                                           // [NT][128]
  if (warp >= 4) {
#pragma unroll
    for (int j = 0; j < L::MINE; ++j) sums[(col0 + j) * 128 + at] = acc[j];
  }
  cg::cluster_group cl = cg::this_cluster();
  cl.sync();
  // this CTA's share of the tokens, eight at a time: their sums of all ranks are under way together (one by one, the reads of
  // 113 tokens took 15 us; the whole product takes 33)
  constexpr int TEAMS = L::SUMS / 4, MANY = 8;
  const int j1 = min(tokens, NT * (rank + 1) / split);
  if (warp >= 4) {
    // sums of a CTA whose wait ran out are not read: copies that were under way may have landed on them
    const bool lost = lane < split && *cl.map_shared_rank((int*)abort_flag, lane) != 0;
    for (int j0 = NT * rank / split + (warp - 4) / 4; j0 < j1; j0 += TEAMS * MANY) {
      float v[MANY];
#pragma unroll
      for (int q = 0; q < MANY; ++q) v[q] = 0.f;
#pragma unroll 4
      for (int r = 0; r < split; ++r) {
        const float* from = cl.map_shared_rank(sums, r) + at;
#pragma unroll
        for (int q = 0; q < MANY; ++q) v[q] += from[min(j0 + q * TEAMS, NT - 1) * 128];
      }
      if (__any_sync(0xffffffffu, lost)) {
#pragma unroll
        for (int q = 0; q < MANY; ++q) v[q] = __uint_as_float(0x7fffffffu);
      }
      if (n < p.N) store_many<MANY>(p, n, m0 + j0, TEAMS, m0 + j1, v);
    }
  }
  cl.sync();                                                            // nobody leaves while its sums are being read
}

template <int NT>
es_status_t launch_rows(const Fp8Maps& maps, const Fp8Params& p, int split, cudaStream_t s) {
  using L = RowsCfg<NT>;
  auto kern = linear_fp8_rows_kernel<NT>;
  const dim3 grid((unsigned)((p.N + 127) / 128 * split), (unsigned)((p.M + NT - 1) / NT));
  ES_CUDA_CHECK(launch_clusters(kern, split > 1 ? split : 0, grid, dim3(L::THREADS), L::SMEM, s, tunables().pdl != 0, maps, p, split));
  return ES_OK;
}

// ---- 256 x 256 tiles on CTA pairs ------------------------------------------------------------------

constexpr int P_STAGES = 6, P_STAGE = 2 * W_TILE;                       // 128 rows of A, 128 of W
constexpr int P_EPI = 8, P_THREADS = 128 + 32 * P_EPI;                  // TMA, MMA and two idle warps; eight warps of sums
// Registers: 168 a thread at launch (64512 in all); the first four warps give theirs up, 128 * 72 + 256 * 216 = 64512.
constexpr int P_REGS_FEW = 72, P_REGS_SUMS = 216;
static_assert(128 * P_REGS_FEW + 32 * P_EPI * P_REGS_SUMS <= 168 * P_THREADS, "the register split must fit what the launch gets");
constexpr int P_TURN = 32 * 128;                                        // a warp's store tile: 32 rows of 128 bytes
constexpr size_t P_SMEM = 1024 + (size_t)P_STAGES * P_STAGE + P_EPI * P_TURN + (2 * P_STAGES + 4) * 8 + 16;

__device__ __forceinline__ uint32_t two(float a, float b, int out) {
  if (out == ES_DTYPE_F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// A warp's 32 rows x 128 columns of sums, 128 bytes of every row at a time through its store tile (16-byte pieces at place
// piece ^ (row & 7): no bank conflicts either way), so that global stores cover whole row segments.
template <bool WIDE>                                                    // fp32 results
__device__ __forceinline__ void store_tile(const Fp8Params& p, unsigned char* turn, const uint64_t (&acc)[64], int row0, int n, int lane) {
  constexpr int CH = WIDE ? 32 : 64;                                    // columns in 128 bytes
#pragma unroll
  for (int c = 0; c < 128; c += CH) {
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      uint4 u;
      if (WIDE) {
        const float2 a = unpack_f32x2(acc[(c + 4 * q) / 2]), b = unpack_f32x2(acc[(c + 4 * q) / 2 + 1]);
        u = make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
      } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 a = unpack_f32x2(acc[(c + 8 * q) / 2 + i]);
          w[i] = two(a.x, a.y, p.out);
        }
        u = make_uint4(w[0], w[1], w[2], w[3]);
      }
      *reinterpret_cast<uint4*>(turn + lane * 128 + ((q ^ (lane & 7)) << 4)) = u;
    }
    __syncwarp();
    if (n + c >= p.N) continue;
    if (p.vec && n + c + CH <= p.N) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3), q = lane & 7;
        if (row0 + r >= p.M) continue;
        uint4 u = *reinterpret_cast<const uint4*>(turn + r * 128 + ((q ^ (r & 7)) << 4));
        const int64_t at = (int64_t)(row0 + r) * p.N + n + c + q * (WIDE ? 4 : 8);
        if (WIDE) {
          if (p.R) {
            const float4 x = *reinterpret_cast<const float4*>(p.R + at);
            u.x = __float_as_uint(__uint_as_float(u.x) + x.x); u.y = __float_as_uint(__uint_as_float(u.y) + x.y);
            u.z = __float_as_uint(__uint_as_float(u.z) + x.z); u.w = __float_as_uint(__uint_as_float(u.w) + x.w);
          }
          *reinterpret_cast<uint4*>((float*)p.C + at) = u;
        } else {
          *reinterpret_cast<uint4*>((uint16_t*)p.C + at) = u;
        }
      }
    } else {
      // ragged or unaligned rows: a column a lane, eight rows under way at a time
#pragma unroll 8
      for (int r = 0; r < 32; ++r) {
#pragma unroll
        for (int i = 0; i < CH / 32; ++i) {
          const int col = lane + 32 * i;
          const int64_t at = (int64_t)(row0 + r) * p.N + n + c + col;
          const bool here = row0 + r < p.M && n + c + col < p.N;
          if (WIDE) {
            float v = *reinterpret_cast<const float*>(turn + r * 128 + (((col >> 2) ^ (r & 7)) << 4) + (col & 3) * 4);
            if (here && p.R) v += p.R[at];
            if (here) ((float*)p.C)[at] = v;
          } else {
            const uint16_t v = *reinterpret_cast<const uint16_t*>(turn + r * 128 + (((col >> 3) ^ (r & 7)) << 4) + (col & 7) * 2);
            if (here) ((uint16_t*)p.C)[at] = v;
          }
        }
      }
    }
  }
}

// split > 1: a cluster of 2 or 4 pairs shares one tile's K range; their sums meet in distributed shared memory, where each pair
// adds up and stores its share of the columns, in order of the ranges.
constexpr int P_PITCH = 260;                                            // floats of a row of sums: 16-byte writes of 32 rows without bank conflicts
static_assert(128 * P_PITCH * 4 <= P_STAGES * P_STAGE, "the sums go where the ring was");

template <bool SPLIT>
__global__ void __launch_bounds__(P_THREADS, 1) linear_fp8_pair_kernel(const __grid_constant__ Fp8Maps maps, const Fp8Params p, const int m_tiles, const int n_tiles,
                                                                       const int pairs_of_tile) {
  const int split = SPLIT ? pairs_of_tile : 1;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char* ring = smem;
  unsigned char* turn = smem + P_STAGES * P_STAGE;
  uint64_t* bars = (uint64_t*)(turn + P_EPI * P_TURN);
  uint64_t *full = bars, *empty = full + P_STAGES, *acc_full = empty + P_STAGES, *acc_empty = acc_full + 2;   // full, acc_empty: rank 0's are used
  uint32_t* tmem_slot = (uint32_t*)(bars + 2 * P_STAGES + 4);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank() & 1;
  const int ks = SPLIT ? (int)(cluster_ctarank() >> 1) : 0;             // range of K
  const uint16_t both = (uint16_t)(3u << (2 * ks));                     // this pair in the cluster
  const int pair = (int)blockIdx.x / (2 * split), n_pairs = (int)gridDim.x / (2 * split);
  const int tiles = m_tiles * n_tiles;
  const int b0 = (int)((long long)p.nkb * ks / split), b1 = (int)((long long)p.nkb * (ks + 1) / split);

  // 16 row tiles share a column tile: what a wave of pairs reads then fits in L2
  auto origin = [&](int tile, int& m0, int& n0) {
    constexpr int GM = 16;
    const int per_group = GM * n_tiles;
    const int first_m = (tile / per_group) * GM;
    const int gsz = min(GM, m_tiles - first_m);
    m0 = (first_m + (tile % per_group) % gsz) * 256;
    n0 = ((tile % per_group) / gsz) * 256;
  };

  if (threadIdx.x == 0) {
    prefetch_tmap(&maps.a);
    prefetch_tmap(&maps.w);
    for (int s = 0; s < P_STAGES; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&acc_full[s]), 1); mbar_init(smem_u32(&acc_empty[s]), 2 * P_EPI); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  pdl_launch_dependents();          // behind the allocation, as above
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P_REGS_FEW));
    if (warp == 0 && lane == 0) {
      int it = 0;
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += n_pairs) {
        int m0, n0;
        origin(tile, m0, n0);
        for (int b = b0; b < b1; ++b, ++it) {
          const int s = it % P_STAGES;
          if (!mbar_wait_soon(smem_u32(&empty[s]), ((it / P_STAGES) & 1) ^ 1, abort_flag)) { ok = false; break; }
          const uint32_t fb = smem_u32(&full[s]), dst = smem_u32(ring + s * P_STAGE);
          if (rank == 0) mbar_expect_tx(fb, 2 * P_STAGE);               // both CTAs' bytes land on this barrier
          tma_load_2d_pair(dst, &maps.a, b * (BKB / 2), m0 + (int)rank * 128, fb);
          tma_load_2d_pair(dst + W_TILE, &maps.w, b * (BKB / 2), n0 + (int)rank * 128, fb);
        }
      }
    }
    if (warp == 1 && lane == 0 && rank == 0) {
      // This thread's own instructions are on the path of every block: they are kept few.
      constexpr uint32_t idesc = umma_idesc_f16(256, 256);
      const uint64_t a0 = umma_desc_sw128(smem_u32(ring)), w0 = umma_desc_sw128(smem_u32(ring) + W_TILE);
      const uint32_t full0 = smem_u32(full), empty0 = smem_u32(empty), acc_full0 = smem_u32(acc_full), acc_empty0 = smem_u32(acc_empty);
      int left = pair < tiles ? ((tiles - 1 - pair) / n_pairs + 1) * (b1 - b0) : 0;
      uint32_t s = 0, ring_phase = 0, buf = 0, buf_phase = 1;
      for (; left > 0; --left) {
        if (!mbar_wait_soon(full0 + s * 8, ring_phase, abort_flag) || !mbar_wait_soon(acc_empty0 + buf * 8, buf_phase, abort_flag)) break;
        tc_fence_after();
        umma_f8_block_pair(tmem + buf * 256, a0 + s * (P_STAGE >> 4), w0 + s * (P_STAGE >> 4), idesc);
        umma_commit_pair(acc_full0 + buf * 8, both);
        umma_commit_pair(empty0 + s * 8, both);
        if (++s == P_STAGES) { s = 0; ring_phase ^= 1; }
        buf ^= 1;
        if (buf == 0) buf_phase ^= 1;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(P_REGS_SUMS));
    const int quarter = warp & 3, half = (warp - 4) >> 2;               // 32 rows, 128 columns
    unsigned char* my_turn = turn + (warp - 4) * P_TURN;
    int it = 0;
    bool ok = true;
    for (int tile = pair; tile < tiles; tile += n_pairs) {
      int m0, n0;
      origin(tile, m0, n0);
      const int row0 = m0 + (int)rank * 128 + quarter * 32, n = n0 + half * 128;
      const bool in = row0 + lane < p.M && n < p.N;
      const float* as = p.as + row0 + lane;
      const float* ws = p.ws + (int64_t)(n / FP8_BLOCK) * p.nkb;
      uint64_t acc[64];
#pragma unroll
      for (int j = 0; j < 64; ++j) acc[j] = 0;
      // Factors are fetched four blocks at a time, the next four while these are used, so that no block waits for its load.
      float sa[4], sw[4], fac[4];
      auto fetch = [&](int b) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bool have = in && b + q < b1;
          sa[q] = have ? as[(int64_t)(b + q) * p.M] : 0.f;
          sw[q] = have ? ws[b + q] : 0.f;
        }
      };
      fetch(b0);
      for (int b = b0; b < b1; ++b, ++it) {
        const int buf = it & 1;
        if (((b - b0) & 3) == 0) {
#pragma unroll
          for (int q = 0; q < 4; ++q) fac[q] = sa[q] * sw[q];
          fetch(b + 4);
        }
        const float f = fac[0];
        fac[0] = fac[1]; fac[1] = fac[2]; fac[2] = fac[3];
        if (ok) ok = mbar_wait_soon(smem_u32(&acc_full[buf]), (it >> 1) & 1, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after();
        const uint64_t ff = pack_f32x2(f, f);
        const uint32_t t = tmem + buf * 256 + half * 128 + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t v[64];
          tmem_ld_issue(t + c * 64, v);
          tmem_ld_wait(v);
          if (c == 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_rank0(smem_u32(&acc_empty[buf]));
          }
#pragma unroll
          for (int j = 0; j < 32; ++j)
            acc[c * 32 + j] = fma_f32x2(pack_f32x2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), ff, acc[c * 32 + j]);
        }
      }
      if (!ok) {
#pragma unroll
        for (int j = 0; j < 64; ++j) acc[j] = 0x7fffffff7fffffffull;
      }
      if (SPLIT) {
        float* mine = (float*)ring + (quarter * 32 + lane) * P_PITCH + half * 128;
#pragma unroll
        for (int j = 0; j < 64; j += 2) {
          const float2 u = unpack_f32x2(acc[j]), w = unpack_f32x2(acc[j + 1]);
          *reinterpret_cast<float4*>(mine + 2 * j) = make_float4(u.x, u.y, w.x, w.y);
        }
      } else if (p.out == ES_DTYPE_F32) {
        store_tile<true>(p, my_turn, acc, row0, n, lane);
      } else {
        store_tile<false>(p, my_turn, acc, row0, n, lane);
      }
    }
  }
  if (SPLIT) {
    __syncwarp();
    cluster_sync_all();
    if (warp >= 4) {
      cg::cluster_group cl = cg::this_cluster();
      int m0, n0;
      origin(pair, m0, n0);
      int lost = 0;                                                     // as above
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s < split) lost |= *cl.map_shared_rank((int*)abort_flag, 2 * s + (int)rank);
      const int lanes = 64 / split, e = (int)threadIdx.x - 128, c = ks * (256 / split) + e % lanes * 4, n = n0 + c;      // lanes of a row, first of four columns
#pragma unroll 4
      for (int r = e / lanes; r < 128; r += 32 * P_EPI / lanes) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          if (s >= split) break;
          const float4 x = *reinterpret_cast<const float4*>(cl.map_shared_rank((float*)ring, 2 * s + (int)rank) + r * P_PITCH + c);
          v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        }
        if (lost) v.x = v.y = v.z = v.w = __uint_as_float(0x7fffffffu);
        const int m = m0 + (int)rank * 128 + r;
        if (m >= p.M || n >= p.N) continue;
        const int64_t at = (int64_t)m * p.N + n;
        if (p.vec) {                                                    // then n + 4 <= N
          if (p.out == ES_DTYPE_F32) {
            if (p.R) {
              const float4 x = *reinterpret_cast<const float4*>(p.R + at);
              v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            *reinterpret_cast<float4*>((float*)p.C + at) = v;
          } else {
            *reinterpret_cast<uint2*>((uint16_t*)p.C + at) = make_uint2(two(v.x, v.y, p.out), two(v.z, v.w, p.out));
          }
        } else {
          const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (n + i >= p.N) break;
            if (p.out == ES_DTYPE_F32) ((float*)p.C)[at + i] = p.R ? x[i] + p.R[at + i] : x[i];
            else ((uint16_t*)p.C)[at + i] = (uint16_t)two(x[i], 0.f, p.out);
          }
        }
      }
    }
  }

  // neither CTA leaves while its partner may still signal or read it
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    if (*abort_flag) settle();
    tmem_dealloc_pair(tmem, 512);
  }
}

template <bool SPLIT>
es_status_t launch_pair_form(const Fp8Maps& maps, const Fp8Params& p, int split, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  auto kern = linear_fp8_pair_kernel<SPLIT>;
  ES_CUDA_CHECK(allow_shared_memory(kern, (int)P_SMEM, &allowed));
  const int m_tiles = (p.M + 255) / 256, n_tiles = (p.N + 255) / 256;
  const long long tiles = (long long)m_tiles * n_tiles;
  long long pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
  if (SPLIT || pairs > tiles) pairs = tiles;
  ES_CUDA_CHECK(launch_clusters(kern, 2 * split, dim3((unsigned)(2 * split * pairs)), dim3(P_THREADS), P_SMEM, s, tunables().pdl != 0, maps, p, m_tiles, n_tiles, split));
  return ES_OK;
}

es_status_t launch_pair(const Fp8Maps& maps, const Fp8Params& p, int split, cudaStream_t s) {
  return split > 1 ? launch_pair_form<true>(maps, p, split, s) : launch_pair_form<false>(maps, p, 1, s);
}

// Clusters of `split` CTAs that the device holds with a CTA on each SM, asked of the form that fits an SM once.  (Fewer than the
// SMs divided by the size: a cluster lies in one part of the device, and the parts differ.  0: it holds none of this size.)
es_status_t places_of(int split, int* places) {
  using L = RowsCfg<128>;
  static_assert(L::OCC == 1, "one CTA an SM");
  static std::atomic<int> known[64][9];                                 // one more than the answer; 0: not asked yet
  static std::atomic<uint64_t> allowed{0};
  int dev = 0;
  ES_CUDA_CHECK(cudaGetDevice(&dev));
  std::atomic<int>* at = dev < 64 ? &known[dev][split] : nullptr;
  if (at && (*places = at->load(std::memory_order_relaxed) - 1) >= 0) return ES_OK;
  ES_CUDA_CHECK(allow_shared_memory(linear_fp8_rows_kernel<128>, (int)L::SMEM, &allowed));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(split);
  cfg.blockDim = dim3(L::THREADS);
  cfg.dynamicSmemBytes = L::SMEM;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  ES_CUDA_CHECK(cudaOccupancyMaxActiveClusters(&n, linear_fp8_rows_kernel<128>, &cfg));
  *places = n;
  if (at) at->store(n + 1, std::memory_order_relaxed);
  return ES_OK;
}

// CTAs that share a tile's K range: as many as make the time of the waves shortest, counted in blocks; starting and joining
// cost about 4 of them (8 with 128 tokens: their sums take longer to join).  Measured for 1, 2, 3, 4 CTAs: 1 x 12288 x 4096
// 15.2 / 12.7 / 17.9 / 16.1 us (2 taken: 3 no longer fit in one wave), 16 x 10240 x 8192 28.5 / 18.7 / 18.0 / 25.6 (3),
// 113 x 5120 x 13824 74.6 / 43.4 / 32.5 / 49.7 (3).
struct Split { int n; long long cost; };
constexpr Split rows_split_of(long long tiles, int nkb, const int (&places)[9], int occ, int start) {
  Split best{1, 0};
  for (int s = 1; s <= 8 && s <= nkb; ++s) {
    const long long at_once = (long long)(s == 1 && places[1] < 1 ? 1 : places[s]) * occ;       // a single CTA remains, whatever was answered
    if (at_once == 0) continue;
    const long long cost = ((tiles + at_once - 1) / at_once) * ((nkb + s - 1) / s + start);
    if (s == 1 || cost < best.cost) best = Split{s, cost};
  }
  return best;
}
constexpr int EVEN[9] = {0, 148, 74, 48, 36, 26, 24, 20, 16}, SMALL_PARTS[9] = {0, 148, 74, 48, 0, 0, 0, 0, 0}, NOTHING[9] = {};
static_assert(rows_split_of(1, 512, EVEN, 1, 8).n == 8 && rows_split_of(1, 512, SMALL_PARTS, 1, 8).n == 3 && rows_split_of(1, 512, NOTHING, 1, 8).n == 1,
              "one tile is shared by the most CTAs that the device holds as a cluster");

template <int NT>
es_status_t rows_split(const Fp8Params& p, int* split, long long* blocks) {
  int places[9] = {};
  for (int s = 1; s <= 8 && s <= p.nkb; ++s) ES_TRY(places_of(s, &places[s]));
  const Split best = rows_split_of((long long)((p.N + 127) / 128) * ((p.M + NT - 1) / NT), p.nkb, places, RowsCfg<NT>::OCC, RowsCfg<NT>::OCC == 1 ? 8 : 4);
  *split = best.n;
  *blocks = best.cost;
  return ES_OK;
}

template <int NT>
es_status_t rows_auto(const Fp8Maps& maps, const Fp8Params& p, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  ES_CUDA_CHECK(allow_shared_memory(linear_fp8_rows_kernel<NT>, (int)RowsCfg<NT>::SMEM, &allowed));
  int split = 1;
  long long blocks = 0;
  ES_TRY(rows_split<NT>(p, &split, &blocks));
  return launch_rows<NT>(maps, p, split, s);
}

// Pairs that share a tile's K range, and eighths of the blocks (of a single CTA's) that the rounds take: a block of a pair's tile
// costs 7 / 8 of one of a single CTA's (0.55 and 0.62 us), start and stores 5, joining SPLIT_JOIN.
constexpr int SPLIT_JOIN = 5;          // measured with two pairs a tile: 320 x 4096 x 4096 21.2 -> 19.1 us, 129 x 5003 x 2064 16.3 -> 16.5
constexpr Split pairs_split_of(long long tiles, int nkb, long long n_pairs, int places4, int places8) {
  Split best{1, (tiles + n_pairs - 1) / n_pairs * nkb * 7 + 5 * 8};
  for (int s = 2; s <= 4 && s <= nkb && tiles * s <= n_pairs; s *= 2) {
    const int places = s == 2 ? places4 : places8;
    if (places < 1) continue;
    const long long cost = (tiles + places - 1) / places * ((nkb + s - 1) / s) * 7 + (5 + SPLIT_JOIN) * 8;
    if (cost < best.cost) best = Split{s, cost};
  }
  return best;
}
static_assert(pairs_split_of(4, 64, 74, 36, 16).n == 4 && pairs_split_of(4, 64, 74, 36, 0).n == 2 && pairs_split_of(4, 64, 74, 0, 0).n == 1,
              "pairs share a tile only in clusters that the device holds");

es_status_t pairs_split(const Fp8Params& p, int* split, long long* eighths) {
  int places4 = 0, places8 = 0;
  ES_TRY(places_of(4, &places4));
  ES_TRY(places_of(8, &places8));
  const Split best = pairs_split_of((long long)((p.M + 255) / 256) * ((p.N + 255) / 256), p.nkb, sm_count() / 2 > 0 ? sm_count() / 2 : 1, places4, places8);
  *split = best.n;
  *eighths = best.cost;
  return ES_OK;
}

// The kernel for more than 64 tokens: the one whose waves take fewer blocks.  Measured, us with tiles of 128 weight rows / on
// pairs: 320 x 4096 x 4096 24.8 / 21.4, 100 x 11008 x 4096 29.0 / 22.3, 512 x 5003 x 2064 37.9 / 18.1, 1024 x 4096 x 4096
// 48.9 / 22.1, 256 x 28672 x 8192 187 / 79; up to 64 tokens the first is ahead everywhere (64 x 28672 x 8192 65 / 78).
es_status_t pairs_better(const Fp8Params& p, bool* pairs) {
  *pairs = false;
  if (p.M <= 64) return ES_OK;
  int split = 1;
  long long blocks = 0, eighths = 0;
  ES_TRY(rows_split<128>(p, &split, &blocks));
  ES_TRY(pairs_split(p, &split, &eighths));
  *pairs = eighths < blocks * 8;
  return ES_OK;
}

}  // namespace
}  // namespace es

using namespace es;

extern "C" es_status_t es_op_linear_fp8(const void* a, const float* a_scale, const void* w, const float* w_scale, const float* R, void* C, int32_t out_dtype, int32_t M,
                                        int32_t N, int32_t K, int32_t path, int32_t weights_ready, void* stream) {
  if (M < 0 || N <= 0 || K <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (out_dtype != ES_DTYPE_F16 && out_dtype != ES_DTYPE_BF16 && out_dtype != ES_DTYPE_F32) return fail(ES_ERR_INVALID_ARG, "the result must be fp16, bf16 or fp32");
  if (R && out_dtype != ES_DTYPE_F32) return fail(ES_ERR_INVALID_ARG, "a residual needs an fp32 result");
  if (path < 0 || path > 2) return fail(ES_ERR_INVALID_ARG, "unknown path %d", path);
  if (K % 16) return fail(ES_ERR_SHAPE, "K = %d is no multiple of 16", K);
  if (M > FP8_MAX_ROWS || N > (1 << 24)) return fail(ES_ERR_RANGE, "more than %d rows or 2^24 columns", FP8_MAX_ROWS);
  if (M == 0) return ES_OK;
  if (!a || !a_scale || !w || !w_scale || !C) return fail(ES_ERR_INVALID_ARG, "null argument");
  const size_t esize = out_dtype == ES_DTYPE_F32 ? 4 : 2;
  if (((uintptr_t)a | (uintptr_t)w) % 16 || ((uintptr_t)a_scale | (uintptr_t)w_scale | (uintptr_t)R) % 4 || (uintptr_t)C % esize)
    return fail(ES_ERR_INVALID_ARG, "a and w must be 16-byte aligned, the others by their elements");
  // a tile may be stored while another has yet to read what its results would lie on; the residual is read where its result goes
  const int64_t c_bytes = (int64_t)M * N * esize, kb = fp8_blocks(K);
  if (overlap(C, c_bytes, a, (int64_t)M * K) || overlap(C, c_bytes, w, (int64_t)N * K) || overlap(C, c_bytes, a_scale, kb * M * 4) ||
      overlap(C, c_bytes, w_scale, kb * fp8_blocks(N) * 4) || (R != C && overlap(C, c_bytes, R, c_bytes)))
    return fail(ES_ERR_INVALID_ARG, "the result overlaps what is read");
  if (!tma_available()) return fail(ES_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const int NT = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128;
  Fp8Params p{a_scale, w_scale, R, C, M, N, fp8_blocks(K), out_dtype, weights_ready != 0, 0};
  bool pairs = path == 2;
  if (path == 0) ES_TRY(pairs_better(p, &pairs));
  p.vec = ((size_t)N * esize) % 16 == 0 && ((uintptr_t)C | (uintptr_t)R) % 16 == 0;
  Fp8Maps maps;
  // two codes make one 16-bit element of the map: boxes of 64 elements are 128 bytes
  ES_TRY(tma_encode_2d_f16(&maps.a, a, M, K / 2, K / 2, pairs ? 128 : NT));
  ES_TRY(tma_encode_2d_f16(&maps.w, w, N, K / 2, K / 2, 128));
  cudaStream_t s = (cudaStream_t)stream;
  if (pairs) {
    int split = 1;
    long long eighths = 0;
    ES_TRY(pairs_split(p, &split, &eighths));
    return launch_pair(maps, p, split, s);
  }
  if (NT == 16) return rows_auto<16>(maps, p, s);
  if (NT == 32) return rows_auto<32>(maps, p, s);
  if (NT == 64) return rows_auto<64>(maps, p, s);
  return rows_auto<128>(maps, p, s);
}
