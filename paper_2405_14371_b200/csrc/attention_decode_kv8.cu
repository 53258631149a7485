// Decode attention over the paged 8-bit cache (TMA + mma.sync m16n8k16), for one or a few query tokens per sequence.
//
// The bound is reading every code of K and V once, so the work is cut for an even and unbroken stream of bytes.  An item is
// one sequence and KV head (and row tile, below); its keys come in tiles of 64 or 32 tokens.  A warp feeds itself: it asks
// for a tile's K and V through TMA into a ring of its own, so that up to 192 KB per SM are on their way while it computes,
// and no warp waits for another.  Two ways of handing out the tiles:
//
//   * stretches: the tiles of all items form one line, and every warp of the machine (8 or 12 in a CTA, one CTA per SM)
//     takes an equal stretch of it, whatever the lengths.  An item that lies in one stretch is finished by its warp; the
//     others leave (o, max, sum), which a second kernel merges in order of the stretches;
//   * groups: where there are no more items than SMs and little to read for each, an item belongs to a CTA or a cluster of
//     2 to 8, whose warps share its tiles and join through (distributed) shared memory.  That saves the second kernel,
//     which is what such calls spend most of their time on.
//
// For a tile and a tile of 8 (NT = 1) or 16 (NT = 2) query rows (T tokens x G heads of the KV head's group):
//   * codes become fp16, which holds every code of both types exactly, on their way from shared memory into the
//     fragments.  The contraction visits the head's dimensions in the order in which a thread's 16-byte pieces hold them;
//     the query fragments are gathered with the same permutation.  The 128-byte swizzle keeps both the K reads (8 rows,
//     4 pieces) and the V reads (4 rows, 8 pieces) free of bank conflicts;
//   * scores S[row, token]: A = query rows, B = K.  The scale of K's page, 1/sqrt(hd) and the query's own exponent are
//     factors of the finished score;
//   * softmax in sub-tiles (SUB tokens of one page) against the sub-tile's own maximum, in fp32: the probabilities lie in
//     [0, 2^15] whatever the other pages hold, and enter the next product as two fp16 halves (hi + lo: 22 bits, and nothing
//     lost above 2^-40 of the largest), so that rounding them costs the output nothing next to its own;
//   * O^T[dim, row] = V^T P^T into a sub-tile accumulator, which joins the running sum with the factor
//     (scale of V's page) * exp(sub-tile maximum - new maximum): pages of very different scales cannot wash each other out.
//
// bf16 queries are brought to fp16 by a power of two per row, largest magnitude to [2^15, 2^16) (bf16's largest mantissa stays
// below 65504): elements down to 2^-32 of the row's largest are exact, smaller ones are off by 2^-40 of it at most.
//
// Measured: 32 sequences of 500 to 8191 tokens, 64 / 8 heads of 128 (286 MB): 59.1 us = 4.8 TB/s, of which the merge kernel
// 6.4 us; in the loop an SM takes in 23.4 bytes a clock, the rate at which memory feeds it (with the multiplications of the
// low halves and the conversions left out it took no less).  8 sequences of 3 to 2500 with 4 draft tokens, 40 heads (103 MB):
// 30.3 us.  16 of 1025 to 1152 (36 MB): 13.7 us.  One of 1000, 32 heads (8 MB): 6.0 us, of which about 3 us are the launch
// and the chain from length to table to the first tile.
//
// Codes behind the context are zeroed in V and masked by selection in the scores, so that garbage (NaN codes among it)
// never meets a product; a page whose scale is NaN makes the rows that see it NaN, a V code that is no number its dimension
// of them.
#include <cooperative_groups.h>
#include <cuda.h>

#include "es_internal.cuh"
#include "kv8.cuh"
#include "launch.cuh"
#include "sm100.cuh"

namespace cg = cooperative_groups;

namespace es {
namespace {

// Warps of a CTA and half tiles of a warp's ring.  8 query rows leave registers for 12 warps, whose latencies hide one
// another's better than 8 warps' do; two half tiles each are then what 192 KB hold (32 sequences of 64/8 heads, 500 to 8191
// tokens: 59.6 us, with 8 warps 65 us).
template <int HD, int NT> constexpr int WARPS = NT == 1 ? 12 : 8;
template <int HD, int NT, int TILE> constexpr int SLOTS = HD == 128 && NT == 1 && TILE == 64 ? 2 : 3;
constexpr int MAX_GROUP = 8;             // CTAs of an item (groups)
constexpr int KV8_MAX_B = 4096;          // sequences whose tile sums fit beside the rings

struct Kv8AttnParams {
  const void* q;
  int64_t q_stride;
  const float *ks, *vs;
  const int *table, *ctx_len;
  void* out;
  float *part_o, *part_ml;               // [2 * warps][rows][hd], [..][rows][2]
  int B, T, Hq, Hkv, G, P, log2P, pps, n_pages, max_ctx;
  int row_tiles, rows;                   // rows = rows of a row tile that are stored
  int16_t bf16;
  int16_t give_up;                       // every warp's first wait counts as run out
  int group;                             // CTAs of an item (groups)
};

// With the maps 384 bytes of parameters; with 8 more every call took 0.1 to 0.2 us longer (drafts 30.5 and 30.3 us).
static_assert(sizeof(Kv8AttnParams) <= 128, "parameters of the attention kernel");

struct alignas(64) Kv8Maps { CUtensorMap k, v; };

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// the same with nothing to add to
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint4 lds16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}

__device__ __forceinline__ uint32_t two_outputs(float a, float b, int bf16) {
  if (bf16) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  return h2_bits(__floats2half2_rn(a, b));
}

// A place on the line of tiles: sequence b, KV head and row tile in it, tile of that item.
struct Cursor {
  int b, kvh, rt, tile, tiles;
  __device__ __forceinline__ void seek(int at, const int* pre, int B, int Hkv, int row_tiles) {
    const int items = Hkv * row_tiles;
    int lo = 0, hi = B;                  // pre[lo] * items <= at < pre[hi] * items
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] * items <= at) lo = mid; else hi = mid;
    }
    b = lo;
    tiles = pre[b + 1] - pre[b];
    const int r = at - pre[b] * items, item = r / tiles;
    tile = r - item * tiles;
    kvh = item / row_tiles;
    rt = item - kvh * row_tiles;
  }
  __device__ __forceinline__ void next(const int* pre, int B, int Hkv, int row_tiles) {
    if (++tile < tiles) return;
    tile = 0;
    if (++rt < row_tiles) return;
    rt = 0;
    if (++kvh < Hkv) return;
    kvh = 0;
    if (++b < B) tiles = pre[b + 1] - pre[b];
  }
};

// Tiles of a warp's stretch.
__device__ __forceinline__ int stretch_of(int total, int warps) { return (total + warps - 1) / warps; }

// Tiles of a sequence; an empty one has a tile without keys, so that somebody writes its rows.
template <int TILE>
__device__ __forceinline__ int tiles_of(int ctx, int max_ctx) { return (min(max(ctx, 1), max_ctx) + TILE - 1) / TILE; }

template <int HD, int CODE, int NT, int TILE, int SUB, bool GROUPED>
__global__ void __launch_bounds__(WARPS<HD, NT> * 32, 1) kv8_attn_kernel(const __grid_constant__ Kv8Maps maps, const Kv8AttnParams p) {
  constexpr int AW = WARPS<HD, NT>, SL = SLOTS<HD, NT, TILE>;
  constexpr int J = HD / 64;             // 16-byte pieces of a K row per thread
  constexpr int D = HD / 8;              // dimensions of V per thread
  constexpr int NM = D / 2;              // output MMAs of 16 tokens
  constexpr int ROWS = 8 * NT;
  constexpr int HALF = TILE * HD;        // bytes of a half tile
  constexpr int NSUB = TILE / SUB, KK = SUB / 16;
  constexpr float LOG2E = 1.4426950408889634f;
  extern __shared__ __align__(1024) unsigned char dyn[];
  unsigned char* ring = dyn + ((1024 - (smem_u32(dyn) & 1023)) & 1023);  // the swizzle goes by address bits 7 to 9
  __shared__ __align__(8) uint64_t bars[AW * SL];
  __shared__ int s_warp[AW];
  __shared__ float2 s_ml[GROUPED ? AW : 1][ROWS];          // groups: maximum and sum of every warp, its factor, the CTAs'
  __shared__ float s_f[GROUPED ? AW : 1][ROWS];
  __shared__ float2 s_all[GROUPED ? MAX_GROUP : 1][ROWS];
  __shared__ int s_abort;
  int* pre = reinterpret_cast<int*>(ring + AW * SL * HALF);          // [B + 1] tiles before each sequence

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int items = p.Hkv * p.row_tiles, n_rows = p.T * p.G;
  const uint32_t my_ring = smem_u32(ring) + warp * SL * HALF, my_bars = smem_u32(bars) + warp * SL * 8;

  if (GROUPED && p.group > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // "this CTA runs"
  if (lane < SL) {                       // a warp's barriers are its own
    mbar_init(my_bars + lane * 8, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 0) {
    s_abort = 0;
    prefetch_tmap(&maps.k);
    prefetch_tmap(&maps.v);
  }
  Cursor c, ahead;
  int begin, end, me = 0;                // tiles of this warp, and its place among the warps
  if constexpr (GROUPED) {
    const int item = blockIdx.x / p.group, in_b = item % items;
    c.b = item / items;
    c.kvh = in_b / p.row_tiles;
    c.rt = in_b - c.kvh * p.row_tiles;
    pdl_wait();
    pdl_launch_dependents();
    c.tiles = tiles_of<TILE>(p.ctx_len[c.b], p.max_ctx);
    const int workers = p.group * AW, per_warp = stretch_of(c.tiles, workers);
    begin = min((warp * p.group + (int)blockIdx.x % p.group) * per_warp, c.tiles);
    end = min(begin + per_warp, c.tiles);
    c.tile = begin;
    __syncthreads();
  } else {
    pdl_wait();
    pdl_launch_dependents();             // only now: the merge kernel reads the lengths before it waits
    int before = 0;
    if (p.B <= 32) {                     // every warp for itself, all writing the same
      const int v = lane < p.B ? tiles_of<TILE>(p.ctx_len[lane], p.max_ctx) : 0;
      int inc = v;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(~0u, inc, d); if (lane >= d) inc += o; }
      if (lane < p.B) pre[lane + 1] = inc;
      if (lane == 0) pre[0] = 0;
      __syncthreads();                   // also: s_abort is set
    }
    for (int base = 0; p.B > 32 && base < p.B; base += AW * 32) {
      const int b = base + tid;
      const int v = b < p.B ? tiles_of<TILE>(p.ctx_len[b], p.max_ctx) : 0;
      int inc = v;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(~0u, inc, d); if (lane >= d) inc += o; }
      if (lane == 31) s_warp[warp] = inc;
      __syncthreads();
      int sum = 0, off = 0;
#pragma unroll
      for (int w = 0; w < AW; ++w) { if (w < warp) off += s_warp[w]; sum += s_warp[w]; }
      if (b < p.B) pre[b + 1] = before + off + inc;
      before += sum;
      __syncthreads();
    }
    if (p.B > 32) {
      if (tid == 0) pre[0] = 0;
      __syncthreads();
    }
    const int total = pre[p.B] * items;
    // stretches go round the SMs first: few tiles spread over all of them
    me = warp * gridDim.x + blockIdx.x;
    const int per_warp = stretch_of(total, AW * gridDim.x);
    begin = min((int64_t)me * per_warp, (int64_t)total);
    end = min(begin + per_warp, total);
    if (begin >= end) return;
    c.seek(begin, pre, p.B, p.Hkv, p.row_tiles);
  }

  const int log2box = min(p.log2P, TILE == 64 ? 6 : 5), boxes = TILE >> log2box;             // tokens that lie together
  ahead = c;
  const int n_half = 2 * (end - begin);
  int asked = 0, ask_slot = 0;           // half tiles asked for: K, V, K, V, ...
  float ks_a = 0.f, vs_a = 0.f;          // lane i: scales of box i of the tile asked for last, and its first 128-byte line
  int row_a = -1;                        // (-1: nothing there)
  float ks_c = 0.f, vs_c = 0.f;
  unsigned ok_a = 0, ok_c = 0;
  auto ask = [&](float& ks_to, float& vs_to) {
    const bool is_v = asked & 1;
    if (!is_v) {
      row_a = -1;
      const int tok = ahead.tile * TILE + (lane << log2box);
      if (lane < boxes && tok < min(p.ctx_len[ahead.b], p.max_ctx)) {
        const int page = p.table[(int64_t)ahead.b * p.pps + (tok >> p.log2P)];
        if ((unsigned)page < (unsigned)p.n_pages) {
          const int ph = page * p.Hkv + ahead.kvh;         // the pool has less than 2^31 lines, so this fits
          ks_to = p.ks[ph];
          vs_to = p.vs[ph];
          row_a = (int)((((unsigned)ph << p.log2P) + (tok & (p.P - 1))) / (128 / HD));
        }
      }
      ok_a = __ballot_sync(~0u, row_a >= 0);
    }
    const uint32_t bar = my_bars + ask_slot * 8;
    if (lane == 0) mbar_expect_tx(bar, __popc(ok_a) * (HD << log2box));
    __syncwarp();
    if (row_a >= 0) tma_load_2d(my_ring + ask_slot * HALF + lane * (HD << log2box), is_v ? &maps.v : &maps.k, 0, row_a, bar);
    if (is_v) {
      if (GROUPED) ++ahead.tile; else ahead.next(pre, p.B, p.Hkv, p.row_tiles);
    }
    ++asked;
    if (++ask_slot == SL) ask_slot = 0;
  };
  int used = 0, slot = 0, parity = 0;    // half tiles used, the place of the next and the phase that it completes
  auto arrived = [&]() -> bool { return __all_sync(~0u, mbar_wait(my_bars + slot * 8, parity, &s_abort, nullptr, 1)); };
  auto release = [&]() {
    __syncwarp();
    ++used;
    if (++slot == SL) { slot = 0; parity ^= 1; }
    if (asked < n_half) ask(ks_a, vs_a);
  };

  int limit[NT];
  float qscale[NT];
  uint32_t qa[NT][8 * J];
  float o[NT][NM][4], m_run[NT], l_run[NT];
  int ctx = 0, item_begin = 0;
  bool fresh = false, running = !p.give_up;
  // query rows of the item at hand; row r of the row tile is token r / G, head kv_head * G + r % G
  auto load_q = [&]() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int i = c.rt * ROWS + 8 * n + g, token = i / p.G;
      const uint16_t* row = reinterpret_cast<const uint16_t*>(p.q) + ((int64_t)c.b * p.T + token) * p.q_stride + (int64_t)(c.kvh * p.G + i - token * p.G) * HD + t * (HD / 4);
#pragma unroll
      for (int j = 0; j < 2 * J; ++j) {
        const uint4 x = i < n_rows ? *reinterpret_cast<const uint4*>(row + 8 * j) : make_uint4(0, 0, 0, 0);
        qa[n][4 * j] = x.x; qa[n][4 * j + 1] = x.y; qa[n][4 * j + 2] = x.z; qa[n][4 * j + 3] = x.w;
      }
    }
  };
  auto start_item = [&](int at) {
    ctx = max(0, min(p.ctx_len[c.b], p.max_ctx));
    item_begin = at - c.tile;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int i = c.rt * ROWS + 8 * n + g;
      limit[n] = i < n_rows ? ctx - p.T + i / p.G + 1 : ctx;         // rows that do not exist have zero queries and are not stored
      qscale[n] = 1.f;
      if (p.bf16) {
        uint32_t mx = 0;
#pragma unroll
        for (int k = 0; k < 8 * J; ++k) mx = __vmaxu2(mx, qa[n][k] & 0x7fff7fffu);
        mx = max(mx & 0xffffu, mx >> 16);
        mx = max(mx, __shfl_xor_sync(~0u, mx, 1));
        mx = max(mx, __shfl_xor_sync(~0u, mx, 2));
        // 2^(15 - e) and its reciprocal, e the exponent of the largest magnitude; from 2^-100 down the row is exact as it is
        const int e = min(max((int)(mx >> 7) - 127, -100), 127);
        const float down = __uint_as_float((uint32_t)(127 + 15 - e) << 23);
        qscale[n] = __uint_as_float((uint32_t)(127 - 15 + e) << 23);
#pragma unroll
        for (int k = 0; k < 8 * J; ++k)
          qa[n][k] = h2_bits(__floats2half2_rn(__uint_as_float(qa[n][k] << 16) * down, __uint_as_float(qa[n][k] & 0xffff0000u) * down));
      }
      qscale[n] *= rsqrtf((float)HD) * LOG2E;              // scores in units of log2
      m_run[n] = -INFINITY;
      l_run[n] = 0.f;
#pragma unroll
      for (int k = 0; k < NM; ++k) o[n][k][0] = o[n][k][1] = o[n][k][2] = o[n][k][3] = 0.f;
    }
  };

  load_q();                              // before the first tiles are asked for: behind them it would wait for their bytes
  if (asked < n_half) {
    ask(ks_c, vs_c);                     // the first tile's K
    ok_c = ok_a;
    ask(ks_c, vs_c);                     // its V
  }
  if (SL == 3 && asked < n_half) ask(ks_a, vs_a);          // the second tile's K, whose scales wait in ks_a, vs_a
  start_item(begin);

  for (int at = begin; at < end && running; ++at) {
    if (fresh) {
      fresh = false;
      load_q();
      start_item(at);
    }
    // ---- scores: rows g (and 8 + g), tokens 8 nt + 2 t + {0, 1} of the tile ----
    if (!arrived()) { running = false; break; }
    float s[TILE / 8][4];
    {
      const uint32_t base = my_ring + slot * HALF;
#pragma unroll
      for (int nt = 0; nt < TILE / 8; ++nt) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          // the 16-byte pieces of token 8 nt + g: J t + j of its row, moved by the swizzle of its 128-byte line
          const uint32_t line = HD == 128 ? 8 * nt + g : 4 * nt + (g >> 1);
          const uint32_t piece = HD == 128 ? 2 * t + j : 4 * (g & 1) + t;
          const uint4 k = lds16(base + line * 128 + ((piece ^ (line & 7)) << 4));
          const uint32_t w[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t lo, hi;
            codes_to_h2<CODE>(w[i], lo, hi);
            const uint32_t a1 = NT == 2 ? qa[NT - 1][8 * j + 2 * i] : 0u, a3 = NT == 2 ? qa[NT - 1][8 * j + 2 * i + 1] : 0u;
            if (j == 0 && i == 0) mma_first(s[nt], qa[0][0], a1, qa[0][1], a3, lo, hi);
            else mma(s[nt], qa[0][8 * j + 2 * i], a1, qa[0][8 * j + 2 * i + 1], a3, lo, hi);
          }
        }
      }
    }
    release();                           // a ring of two takes this tile's successor only now; a longer one has it already

    const uint32_t vbase = my_ring + slot * HALF;
    bool v_here = false;
#pragma unroll
    for (int sub = 0; sub < NSUB; ++sub) {
      const int T0 = c.tile * TILE + sub * SUB;
      const int bx = (sub * SUB) >> log2box;
      if (T0 >= ctx || !((ok_c >> bx) & 1)) continue;      // nothing there, or a page nobody sees
      const float k_s = __shfl_sync(~0u, ks_c, bx), v_s = __shfl_sync(~0u, vs_c, bx);
      // ---- softmax of the sub-tile ----
      uint32_t ph[NT][KK][2], pl[NT][KK][2];               // probabilities, hi and lo halves: B fragments of the output MMAs
      float al[NT][2], be[NT][2];                          // factors of rows 2 t and 2 t + 1
      const bool inner = T0 + SUB <= ctx - p.T + 1;        // every row sees all of it
      bool same = true;                                    // no row's maximum changes
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float x[2 * KK][2], mx = -INFINITY;
        const float f = qscale[n] * k_s;
#pragma unroll
        for (int nt = 0; nt < 2 * KK; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            x[nt][e] = s[sub * 2 * KK + nt][2 * n + e] * f;
            if (!inner && T0 + 8 * nt + 2 * t + e >= limit[n]) x[nt][e] = -INFINITY;
            mx = fmaxf(mx, x[nt][e]);
          }
        mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 2));
        const bool sees = T0 < limit[n];
        // the reference is a whole number, so that taking it off 15 is exact and factors between references are powers of two
        const float ref = mx == -INFINITY ? 0.f : ceilf(mx), shift = 15.f - ref;
        float sum = 0.f;
#pragma unroll
        for (int nt = 0; nt < 2 * KK; ++nt) {
          x[nt][0] = ex2(x[nt][0] + shift);
          x[nt][1] = ex2(x[nt][1] + shift);
          sum += x[nt][0] + x[nt][1];
          const __half2 h = __floats2half2_rn(x[nt][0], x[nt][1]);
          const float2 back = __half22float2(h);
          ph[n][nt >> 1][nt & 1] = h2_bits(h);
          pl[n][nt >> 1][nt & 1] = h2_bits(__floats2half2_rn(x[nt][0] - back.x, x[nt][1] - back.y));
        }
        sum += __shfl_xor_sync(~0u, sum, 1);
        sum += __shfl_xor_sync(~0u, sum, 2);
        const float mn = fmaxf(m_run[n], mx == -INFINITY ? mx : ref);
        const float to = mn == -INFINITY ? 0.f : mn;
        const float alpha = ex2(m_run[n] - to);
        const float join = sees ? ex2(ref - to - 15.f) : 0.f;        // NaN scores pass through: they are in `sum` and in the product
        const float beta = sees ? join * v_s : 0.f;
        l_run[n] = sees ? l_run[n] * alpha + sum * join : l_run[n];
        m_run[n] = mn;
        same = same && alpha == 1.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          al[n][i] = __shfl_sync(~0u, alpha, (2 * t + i) * 4);
          be[n][i] = __shfl_sync(~0u, beta, (2 * t + i) * 4);
        }
      }
      if (!v_here) {
        v_here = true;
        if (!arrived()) { running = false; break; }
      }
      if (!__all_sync(~0u, same)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < NM; ++i) { o[n][i][0] *= al[n][0]; o[n][i][1] *= al[n][1]; o[n][i][2] *= al[n][0]; o[n][i][3] *= al[n][1]; }
      }
      // ---- a V code that is no number shows in the rows that see its token, and in no others (0 * NaN would be NaN there):
      // where rows differ in what they see, it is written into their sums and taken out of the tile ----
      if constexpr (CODE == CODE_E4M3) {
        if (!inner && p.T > 1) {
          const int n_tok = min(SUB, ctx - T0);
          auto place = [&](int j) -> uint32_t {            // dimensions D g .. of token j of the sub-tile
            const uint32_t line = HD == 128 ? sub * SUB + j : sub * (SUB / 2) + (j >> 1);
            const uint32_t piece = HD == 128 ? g : 4 * (j & 1) + (g >> 1);
            return vbase + line * 128 + ((piece ^ (line & 7)) << 4) + (HD == 128 ? 0 : 8 * (g & 1));
          };
          auto no_number = [](uint32_t w) { return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu); };
          uint32_t any = 0;
          for (int j = t; j < n_tok; j += 4) {
            const uint2 a = lds8(place(j)), b = HD == 128 ? lds8(place(j) + 8) : a;
            any |= no_number(a.x) | no_number(a.y) | no_number(b.x) | no_number(b.y);
          }
          if (__any_sync(~0u, any != 0)) {
            int lim[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) lim[n][e] = __shfl_sync(~0u, limit[n], (2 * t + e) * 4);
#pragma unroll 1
            for (int j = 0; j < n_tok; ++j) {
              uint32_t w[D / 4];
#pragma unroll
              for (int i = 0; i < D / 4; i += 2) { const uint2 x = lds8(place(j) + 4 * i); w[i] = x.x; w[i + 1] = x.y; }
              __syncwarp();
#pragma unroll
              for (int i = 0; i < D / 4; ++i) {
                const uint32_t bad = no_number(w[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                  for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                      if (((bad >> (8 * k)) & 1) && T0 + j < lim[n][e]) o[n][(4 * i + k) % NM][2 * ((4 * i + k) / NM) + e] = NAN;
                if (t == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(place(j) + 4 * i), "r"(w[i] & ~bad) : "memory");
              }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");              // before the next copy into this place
            __syncwarp();
          }
        }
      }
      // ---- output: MMA i gives dimensions D g + i (rows 0..7) and D g + D / 2 + i (rows 8..15) ----
      auto load_v = [&](int kk, uint32_t (&v)[4][D / 4]) {
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          // token 16 kk + 2 t + {0, 1} (+ 8) of the sub-tile: its dimensions D g ..
          const int e = q4 & 1, up = q4 >> 1;
          if constexpr (HD == 128) {
            const uint32_t line = sub * SUB + 16 * kk + 8 * up + 2 * t + e;
            const uint4 x = lds16(vbase + line * 128 + ((g ^ (line & 7)) << 4));
            v[q4][0] = x.x; v[q4][1] = x.y; v[q4][2] = x.z; v[q4][3] = x.w;
          } else {
            const uint32_t line = sub * (SUB / 2) + 8 * kk + 4 * up + t;
            const uint2 x = lds8(vbase + line * 128 + (((4 * e + (g >> 1)) ^ (line & 7)) << 4) + 8 * (g & 1));
            v[q4][0] = x.x; v[q4][1] = x.y;
          }
        }
        if (T0 + SUB > ctx) {            // the last tokens' sub-tile: nothing behind them enters a product
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4)
            if (T0 + 16 * kk + 8 * (q4 >> 1) + 2 * t + (q4 & 1) >= ctx)
#pragma unroll
              for (int w = 0; w < D / 4; ++w) v[q4][w] = 0;
        }
      };
      // A registers 0..3 of the four MMAs that words w and w + D / 8 of the four tokens make
      auto fragments = [&](const uint32_t (&v)[4][D / 4], int w, uint32_t (&a)[4][4]) {
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t x = v[2 * q2][w + half * (D / 8)], y = v[2 * q2 + 1][w + half * (D / 8)];
            codes_to_h2<CODE>(__byte_perm(x, y, 0x5140), a[2 * q2 + half][0], a[2 * q2 + half][1]);
            codes_to_h2<CODE>(__byte_perm(x, y, 0x7362), a[2 * q2 + half][2], a[2 * q2 + half][3]);
          }
      };
      if constexpr (NT == 1) {           // accumulators of the whole sub-tile, V as it is needed
        float acc[NM][4];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          uint32_t v[4][D / 4], a[4][4];
          load_v(kk, v);
#pragma unroll
          for (int w = 0; w < D / 8; ++w) {
            fragments(v, w, a);
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              if (kk == 0) mma_first(acc[4 * w + d], a[0][d], a[1][d], a[2][d], a[3][d], ph[0][kk][0], ph[0][kk][1]);
              else mma(acc[4 * w + d], a[0][d], a[1][d], a[2][d], a[3][d], ph[0][kk][0], ph[0][kk][1]);
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) mma(acc[4 * w + d], a[0][d], a[1][d], a[2][d], a[3][d], pl[0][kk][0], pl[0][kk][1]);
          }
        }
#pragma unroll
        for (int i = 0; i < NM; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[0][i][k] += acc[i][k] * be[0][k & 1];
      } else {                           // two row blocks: accumulators of four MMAs, all of V held
        uint32_t v[KK][4][D / 4];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) load_v(kk, v[kk]);
#pragma unroll
        for (int w = 0; w < D / 8; ++w) {
          float acc[4][NT][4];
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            uint32_t a[4][4];
            fragments(v[kk], w, a);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                if (kk == 0) mma_first(acc[d][n], a[0][d], a[1][d], a[2][d], a[3][d], ph[n][kk][0], ph[n][kk][1]);
                else mma(acc[d][n], a[0][d], a[1][d], a[2][d], a[3][d], ph[n][kk][0], ph[n][kk][1]);
                mma(acc[d][n], a[0][d], a[1][d], a[2][d], a[3][d], pl[n][kk][0], pl[n][kk][1]);
              }
          }
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int k = 0; k < 4; ++k) o[n][4 * w + d][k] += acc[d][n][k] * be[n][k & 1];
        }
      }
    }
    if (!running) break;
    if (!v_here && !arrived()) { running = false; break; }
    if (SL == 2) {                       // the next tile's K was asked for above or is asked for now: its scales come then
      release();
      ks_c = ks_a; vs_c = vs_a; ok_c = ok_a;
    } else {                             // they wait in ks_a, vs_a until the K after it is asked for
      ks_c = ks_a; vs_c = vs_a; ok_c = ok_a;
      release();
    }

    if constexpr (GROUPED) {
      ++c.tile;
      continue;
    }
    // ---- the item's end, or the stretch's ----
    const bool item_ends = c.tile + 1 == c.tiles;
    if (item_ends || at + 1 == end) {
      const bool whole = item_ends && item_begin >= begin;
      const int64_t part = 2 * (int64_t)me + (item_begin >= begin);       // a stretch has two split items at most
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {                      // this thread holds dimensions D g .. D g + D - 1 of row 8 n + 2 t + e
          const int r = 8 * n + 2 * t + e, i = c.rt * ROWS + r, token = i / p.G;
          const float m = __shfl_sync(~0u, m_run[n], (2 * t + e) * 4), l = __shfl_sync(~0u, l_run[n], (2 * t + e) * 4);
          if (i >= n_rows) continue;
          if (whole) {
            const int64_t row = ((int64_t)c.b * p.T + token) * p.Hq + c.kvh * p.G + (i - token * p.G);
            uint32_t* to = reinterpret_cast<uint32_t*>(p.out) + (row * HD + D * g) / 2;
            const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int k = 0; k < NM; k += 2) to[(h * NM + k) / 2] = two_outputs(o[n][k][2 * h + e] * inv, o[n][k + 1][2 * h + e] * inv, p.bf16);
          } else {
            float* to = p.part_o + (part * p.rows + r) * HD + D * g;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int k = 0; k < NM; k += 4)
                *reinterpret_cast<float4*>(to + h * NM + k) = make_float4(o[n][k][2 * h + e], o[n][k + 1][2 * h + e], o[n][k + 2][2 * h + e], o[n][k + 3][2 * h + e]);
            if (g == 0) *reinterpret_cast<float2*>(p.part_ml + (part * p.rows + r) * 2) = make_float2(m, l);
          }
        }
      fresh = true;
    }
    c.next(pre, p.B, p.Hkv, p.row_tiles);
  }
  // A wait ran out.  These calls have no status word: every row that this warp was to finish or to hand over becomes NaN (a
  // sum that is NaN stays so through both joins), so that nothing it did not compute looks like a result.  All of its stretch,
  // from the start, so that the loop need not keep anything for this.
  if (!running) {
    if constexpr (GROUPED) {
#pragma unroll
      for (int n = 0; n < NT; ++n) l_run[n] = NAN;
    } else {
      c.seek(begin, pre, p.B, p.Hkv, p.row_tiles);
      item_begin = begin - c.tile;
      for (int at = begin; at < end; ++at) {
        const bool item_ends = c.tile + 1 == c.tiles;
        if (item_ends || at + 1 == end) {
          const int i = c.rt * ROWS + lane, token = i / p.G;
          if (lane < ROWS && i < n_rows) {
            if (item_ends && item_begin >= begin) {
              uint32_t* to = reinterpret_cast<uint32_t*>(p.out) + (((int64_t)c.b * p.T + token) * p.Hq + c.kvh * p.G + (i - token * p.G)) * (HD / 2);
              for (int k = 0; k < HD / 2; ++k) to[k] = two_outputs(NAN, NAN, p.bf16);
            } else {
              const int64_t part = 2 * (int64_t)me + (item_begin >= begin);
              *reinterpret_cast<float2*>(p.part_ml + (part * p.rows + lane) * 2) = make_float2(0.f, NAN);
            }
          }
          item_begin = at + 1;
        }
        c.next(pre, p.B, p.Hkv, p.row_tiles);
      }
    }
    // and its copies that are under way land before its shared memory goes
    for (; used < asked; ++used) {
      int nobody = 0;
      mbar_wait(my_bars + slot * 8, parity, &nobody, nullptr, 1);
      if (++slot == SL) { slot = 0; parity ^= 1; }
    }
  }
  if constexpr (GROUPED) {
    // ---- the warps of the CTA, then the CTAs of the item, join in order ----
    // a warp's part goes over its ring, which nothing writes any more: o [ROWS][HD] (zero where it had no tile)
    float* mine = reinterpret_cast<float*>(ring + warp * SL * HALF);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < NM; k += 4)
            *reinterpret_cast<float4*>(mine + (8 * n + 2 * t + e) * HD + D * g + h * NM + k) =
                make_float4(o[n][k][2 * h + e], o[n][k + 1][2 * h + e], o[n][k + 2][2 * h + e], o[n][k + 3][2 * h + e]);
      if (t == 0) s_ml[warp][8 * n + g] = make_float2(m_run[n], l_run[n]);
    }
    __syncthreads();
    const int live = min(ROWS, n_rows - c.rt * ROWS);                     // rows that exist
    if (tid < AW * ROWS) {               // the factor of every warp's part of a row
      const int w = tid / ROWS, r = tid - w * ROWS;
      float2 ml[AW];
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < AW; ++k) { ml[k] = s_ml[k][r]; m = fmaxf(m, ml[k].x); }
      const float ref = m == -INFINITY ? 0.f : m;
      s_f[w][r] = ex2(s_ml[w][r].x - ref);
      if (w == 0) {
        float l = 0.f;
#pragma unroll
        for (int k = 0; k < AW; ++k) l += ml[k].y * ex2(ml[k].x - ref);
        s_all[0][r] = make_float2(m, l);
      }
    }
    __syncthreads();
    constexpr int PER = (ROWS * HD / 2 + AW * 32 - 1) / (AW * 32);        // pairs of outputs a thread
    const int pairs = live * (HD / 2);
    float2 sum[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = tid + i * AW * 32, r = at / (HD / 2);
      if (at >= pairs) break;
      sum[i] = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < AW; ++w) {
        const float2 x = *reinterpret_cast<const float2*>(ring + w * SL * HALF + at * 8);
        sum[i].x += x.x * s_f[w][r];
        sum[i].y += x.y * s_f[w][r];
      }
    }
    if (p.group > 1) {
      // the CTAs leave their parts with the first one, behind its rings; before that, all of them run
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      const int rank = (int)cluster_ctarank();
      float2* inbox = reinterpret_cast<float2*>(ring + AW * SL * HALF);
      if (rank > 0) {
        cg::cluster_group cl = cg::this_cluster();
        float2* to = cl.map_shared_rank(inbox, 0) + (rank - 1) * (ROWS * HD / 2);
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (tid + i * AW * 32 < pairs) to[tid + i * AW * 32] = sum[i];
        if (tid < live) cl.map_shared_rank(&s_all[0][0], 0)[rank * ROWS + tid] = s_all[0][tid];
      }
      cluster_sync_all();
      if (rank > 0) return;
    }
    if (tid < ROWS && tid < live) {      // factors of the CTAs' parts, the sum's reciprocal in them
      float2 ml[MAX_GROUP];
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int k = 0; k < MAX_GROUP; ++k)
        if (k < p.group) { ml[k] = s_all[k][tid]; m = fmaxf(m, ml[k].x); }
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int k = 0; k < MAX_GROUP; ++k)
        if (k < p.group) { ml[k].x = ex2(ml[k].x - ref); l += ml[k].y * ml[k].x; }
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int k = 0; k < MAX_GROUP; ++k)
        if (k < p.group) s_all[k][tid].x = ml[k].x * inv;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = tid + i * AW * 32, r = at / (HD / 2), d = at - r * (HD / 2);
      if (at >= pairs) break;
      const float2* inbox = reinterpret_cast<const float2*>(ring + AW * SL * HALF);
      float x = sum[i].x * s_all[0][r].x, y = sum[i].y * s_all[0][r].x;
#pragma unroll
      for (int k = 1; k < MAX_GROUP; ++k)
        if (k < p.group) {
          const float2 part = inbox[(k - 1) * (ROWS * HD / 2) + at];
          x += part.x * s_all[k][r].x;
          y += part.y * s_all[k][r].x;
        }
      const int row_i = c.rt * ROWS + r, token = row_i / p.G;
      const int64_t row = ((int64_t)c.b * p.T + token) * p.Hq + c.kvh * p.G + (row_i - token * p.G);
      reinterpret_cast<uint32_t*>(p.out)[(row * HD) / 2 + d] = two_outputs(x, y, p.bf16);
    }
  }
}

// One CTA per output row of an item that was split (2048 rows: 6.4 us; a thread for four dimensions of a row, or a CTA for
// an item's rows, brought fewer bytes under way and took 2 to 4 us longer): its warps take every fourth part, in order, and join in order.  Where the
// parts lie follows from the lengths alone, so that is worked out while the first kernel still runs.
template <int HD, int TILE>
__global__ void __launch_bounds__(128) kv8_merge_kernel(const Kv8AttnParams p, int warps) {
  constexpr int V = HD / 32, AHEAD = 4;
  __shared__ float sm_o[4][HD];
  __shared__ float2 sm_ml[4];
  __shared__ int sm_n[4][2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.x, token = blockIdx.y, b = blockIdx.z;
  const int kvh = h / p.G, i = token * p.G + h - kvh * p.G;
  const int nt_rows = p.rows > 8 ? 16 : 8, rt = i / nt_rows, r = i - rt * nt_rows;
  const int items = p.Hkv * p.row_tiles;
  int before = 0, all = 0;
  for (int k = tid; k < p.B; k += 128) {
    const int v = tiles_of<TILE>(p.ctx_len[k], p.max_ctx);
    all += v;
    if (k < b) before += v;
  }
  all = __reduce_add_sync(~0u, all);
  before = __reduce_add_sync(~0u, before);
  if (lane == 0) { sm_n[warp][0] = all; sm_n[warp][1] = before; }
  __syncthreads();
  all = sm_n[0][0] + sm_n[1][0] + sm_n[2][0] + sm_n[3][0];
  before = sm_n[0][1] + sm_n[1][1] + sm_n[2][1] + sm_n[3][1];
  const int per_warp = stretch_of(all * items, warps);
  const int tiles = tiles_of<TILE>(p.ctx_len[b], p.max_ctx);
  const int begin = before * items + (kvh * p.row_tiles + rt) * tiles;
  const int w0 = begin / per_warp, w1 = (begin + tiles - 1) / per_warp;
  if (w0 == w1) {                        // finished by its warp; one CTA keeps this kernel from ending before the first one
    if (h + token + b == 0) pdl_wait();
    return;
  }
  const int n = w1 - w0 + 1;
  pdl_wait();
  pdl_launch_dependents();
  float acc[V], mm = -INFINITY, ll = 0.f;
#pragma unroll
  for (int c = 0; c < V; ++c) acc[c] = 0.f;
  for (int k0 = warp; k0 < n; k0 += 4 * AHEAD) {           // several parts' loads under way at a time
    float2 ml[AHEAD];
    float x[AHEAD][V];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int k = min(k0 + 4 * j, n - 1);
      const int64_t part = (2 * (int64_t)(w0 + k) + (k == 0)) * p.rows + r;
      ml[j] = __ldcg(reinterpret_cast<const float2*>(p.part_ml + part * 2));
#pragma unroll
      for (int c = 0; c < V; ++c) x[j][c] = __ldcg(p.part_o + part * HD + c * 32 + lane);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (k0 + 4 * j >= n) break;
      const float mn = fmaxf(mm, ml[j].x), ref = mn == -INFINITY ? 0.f : mn;
      const float a = ex2(mm - ref), f = ex2(ml[j].x - ref);
      ll = ll * a + ml[j].y * f;
#pragma unroll
      for (int c = 0; c < V; ++c) acc[c] = acc[c] * a + x[j][c] * f;
      mm = mn;
    }
  }
#pragma unroll
  for (int c = 0; c < V; ++c) sm_o[warp][c * 32 + lane] = acc[c];
  if (lane == 0) sm_ml[warp] = make_float2(mm, ll);
  __syncthreads();
  if (tid < HD / 2) {
    float m = fmaxf(fmaxf(sm_ml[0].x, sm_ml[1].x), fmaxf(sm_ml[2].x, sm_ml[3].x));
    m = m == -INFINITY ? 0.f : m;
    float l = 0.f, x = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = ex2(sm_ml[w].x - m);
      l += sm_ml[w].y * f;
      x += sm_o[w][2 * tid] * f;
      y += sm_o[w][2 * tid + 1] * f;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t row = ((int64_t)b * p.T + token) * p.Hq + h;
    reinterpret_cast<uint32_t*>(p.out)[(row * HD) / 2 + tid] = two_outputs(x * inv, y * inv, p.bf16);
  }
}

// How a call is cut: query rows of a KV head, and tiles handed out as stretches or to groups.
struct Shape { int nt, row_tiles, rows, group, tile; };

constexpr int MIN_TILE = 32, MAX_TILE = 64;
constexpr int GROUP_BYTES = 512 << 10;

Shape shape_of(int B, int T, int Hq, int Hkv, int hd, int max_ctx) {
  Shape s;
  const int rows = T * (Hq / Hkv);
  s.nt = rows > 8 ? 2 : 1;
  s.row_tiles = (rows + 8 * s.nt - 1) / (8 * s.nt);
  s.rows = rows < 8 * s.nt ? rows : 8 * s.nt;
  // Groups: all items at once, one wave of clusters as large as the SMs allow (no larger than the tiles can use), and not
  // more than half a megabyte for a CTA to read, so that an uneven batch, whose longest sequence then sets the time,
  // loses about what the second kernel costs.  With 32 KV heads of 128, groups and stretches take: 1 sequence of 700
  // 6.7 and 10.0 us, of 8192 (512 KB a CTA) 20.7 and 27.5 us; 4 of 2048 (512 KB) 20.2 and 23.1 us, of 1 to 2048 19.8 and
  // 18.0 us; 4 of 4096 (1 MB) 32.9 and 32.6 us, of 1 to 4096 32.4 and 23.0 us.  All of it goes by max_ctx, for the lengths are on
  // the device: a cap far above them costs the way it leads to.  16 sequences of 1025 to 1152, 64 / 8 heads: 13.0 us with a cap up to
  // 2048, 16.7 us from 4096 on (stretches); one of 1000, 32 heads: 6.0 us up to 8192, 9.6 us with 16384; two of 300, 8 KV heads:
  // 5.7 us with their own length, 9.3 us with 2048 and more (clusters of 8 for 10 tiles; stretches 7.2 us).
  const long long items = (long long)B * Hkv * s.row_tiles;
  const int warps = s.nt == 1 ? WARPS<128, 1> : WARPS<128, 2>;
  int group = 1;
  while (group < MAX_GROUP && items * group * 2 <= sm_count() && (long long)group * warps * MIN_TILE < max_ctx) group *= 2;
  const bool grouped = items <= sm_count() && 2LL * max_ctx * hd <= (long long)GROUP_BYTES * group;
  s.group = grouped ? group : 0;
  // Stretches: smaller tiles where a warp would get few of them, and the odd one too many would show.  With 32 KV heads,
  // tiles of 32 and 64 take: 8 sequences of 640 (1.4 tiles of 64 a warp) 16.7 and 17.3 us, 8 of 1280 24.7 and 23.3 us,
  // 16 of 1280 41.1 and 36.4 us.
  const long long tiles = items * ((max_ctx + MAX_TILE - 1) / MAX_TILE);
  s.tile = grouped || (s.nt == 1 && tiles < 2LL * warps * sm_count()) ? MIN_TILE : MAX_TILE;
  return s;
}

int warps_of(const Shape& s) { return (s.nt == 1 ? WARPS<128, 1> : WARPS<128, 2>) * sm_count(); }

size_t parts_of(const Shape& s) { return (size_t)2 * warps_of(s) * s.rows; }

size_t scratch_of(const Shape& s, int hd, int max_ctx) {
  if (s.group > 0 || max_ctx <= s.tile) return 0;          // joined in the first kernel, or no item has a second tile
  return parts_of(s) * (hd + 2) * sizeof(float);
}

template <int HD, int CODE, int NT, int TILE, int SUB, bool GROUPED>
es_status_t launch_sub(const Kv8Maps& maps, const Kv8AttnParams& p, cudaStream_t s) {
  constexpr int AW = WARPS<HD, NT>;
  constexpr int RINGS = AW * SLOTS<HD, NT, TILE> * TILE * HD + 1024; // and room to align them
  constexpr int INBOX = (MAX_GROUP - 1) * 8 * NT * HD * 4; // parts of the other CTAs of a group
  auto kern = kv8_attn_kernel<HD, CODE, NT, TILE, SUB, GROUPED>;
  static std::atomic<uint64_t> allowed{0};
  ES_CUDA_CHECK(allow_shared_memory(kern, RINGS + (GROUPED ? INBOX : (KV8_MAX_B + 1) * (int)sizeof(int)), &allowed));
  ES_CUDA_CHECK(launch_clusters(kern, GROUPED && p.group > 1 ? p.group : 0, dim3(GROUPED ? p.B * p.Hkv * p.row_tiles * p.group : sm_count()), dim3(AW * 32),
                                RINGS + (GROUPED ? (p.group > 1 ? INBOX : 0) : (size_t)(p.B + 1) * sizeof(int)), s, tunables().pdl != 0, maps, p));
  if (!GROUPED && p.max_ctx > TILE)
    ES_CUDA_CHECK(launch_kernel(kv8_merge_kernel<HD, TILE>, dim3(p.Hq, p.T, p.B), dim3(128), 0, s, tunables().pdl != 0, p, AW * sm_count()));
  return ES_OK;
}

// Sub-tiles of the softmax: as much of a tile as lies in one page (two row blocks: 32 tokens at most, for registers).
template <int HD, int CODE, int NT>
es_status_t launch_tile(const Kv8Maps& maps, const Kv8AttnParams& p, const Shape& sh, cudaStream_t s) {
  const bool small = p.P == 16;
  if (sh.group > 0) return small ? launch_sub<HD, CODE, NT, 32, 16, true>(maps, p, s) : launch_sub<HD, CODE, NT, 32, 32, true>(maps, p, s);
  if constexpr (NT == 1) {
    if (sh.tile == 32) return small ? launch_sub<HD, CODE, 1, 32, 16, false>(maps, p, s) : launch_sub<HD, CODE, 1, 32, 32, false>(maps, p, s);
    if (p.P >= 64) return launch_sub<HD, CODE, 1, 64, 64, false>(maps, p, s);
  }
  return small ? launch_sub<HD, CODE, NT, 64, 16, false>(maps, p, s) : launch_sub<HD, CODE, NT, 64, 32, false>(maps, p, s);
}

template <int HD, int CODE>
es_status_t launch(const Kv8Maps& maps, const Kv8AttnParams& p, const Shape& sh, cudaStream_t s) {
  return sh.nt == 1 ? launch_tile<HD, CODE, 1>(maps, p, sh, s) : launch_tile<HD, CODE, 2>(maps, p, sh, s);
}

es_status_t check_heads(int B, int T, int Hq, int Hkv, int hd, int page_tokens, int max_ctx) {
  if (B <= 0 || T <= 0 || Hq <= 0 || Hkv <= 0 || hd <= 0 || page_tokens <= 0 || max_ctx <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (Hq % Hkv != 0) return fail(ES_ERR_SHAPE, "Hq must be a multiple of Hkv");
  if (hd != 64 && hd != 128) return fail(ES_ERR_SHAPE, "head_dim must be 64 or 128");
  if (max_ctx > (1 << 30)) return fail(ES_ERR_RANGE, "max_ctx exceeds 2^30");
  if (B > KV8_MAX_B) return fail(ES_ERR_RANGE, "B = %d exceeds %d sequences", B, KV8_MAX_B);
  if (T > 65535 || (long long)T * (Hq / Hkv) > 65535) return fail(ES_ERR_RANGE, "T * (Hq / Hkv) exceeds one launch");
  const Shape s = shape_of(B, T, Hq, Hkv, hd, max_ctx);
  if ((long long)B * Hkv * s.row_tiles * ((max_ctx + MIN_TILE - 1) / MIN_TILE) > (1LL << 30))
    return fail(ES_ERR_RANGE, "B * heads * max_ctx exceeds one launch");
  return ES_OK;
}

}  // namespace
}  // namespace es

extern "C" {

size_t es_op_decode_attention_kv8_scratch_bytes(int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t hd,
                                                int32_t page_tokens, int32_t max_ctx) {
  using namespace es;
  if (check_heads(B, T, Hq, Hkv, hd, page_tokens, max_ctx) != ES_OK) return 0;
  return scratch_of(shape_of(B, T, Hq, Hkv, hd, max_ctx), hd, max_ctx);
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
  if (((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)scratch) % 16 || (uintptr_t)out % 4)
    return fail(ES_ERR_INVALID_ARG, "q, pages and scratch must be 16-byte aligned");
  const Shape sh = shape_of(B, T, Hq, Hkv, hd, max_ctx);
  const size_t need = scratch_of(sh, hd, max_ctx);
  if (scratch_bytes < need || (need && !scratch)) return fail(ES_ERR_WORKSPACE, "scratch: %zu bytes given, %zu needed", scratch ? scratch_bytes : (size_t)0, need);
  int log2P = 0;
  while ((1 << log2P) < page_tokens) ++log2P;
  // pages as 128-byte lines (of one token, or of two when hd is 64); a copy takes what lies together of a tile.  The
  // helper's matrix of 64 fp16 columns moves bytes as they are
  Kv8Maps maps;
  const int64_t lines = (int64_t)n_pages * Hkv * page_tokens * hd / 128;
  const int box_lines = (page_tokens < sh.tile ? page_tokens : sh.tile) * hd / 128;
  if (lines > INT32_MAX) return fail(ES_ERR_RANGE, "a page pool exceeds 2^31 lines of 128 bytes");
  ES_TRY(tma_encode_2d_f16(&maps.k, k_pages, lines, 64, 64, box_lines));
  ES_TRY(tma_encode_2d_f16(&maps.v, v_pages, lines, 64, 64, box_lines));
  float* part = (float*)scratch;
  const size_t parts = parts_of(sh);
  Kv8AttnParams p{q, q_stride, k_scale, v_scale, block_table, ctx_len, out, part, part + parts * hd, B, T, Hq, Hkv, Hq / Hkv,
                  page_tokens, log2P, pages_per_seq, n_pages, max_ctx, sh.row_tiles, sh.rows,
                  (int16_t)(dtype == ES_DTYPE_BF16), (int16_t)(tunables().kv8_give_up != 0), sh.group};
  cudaStream_t s = (cudaStream_t)stream;
  if (hd == 128) return code == CODE_I8 ? launch<128, CODE_I8>(maps, p, sh, s) : launch<128, CODE_E4M3>(maps, p, sh, s);
  return code == CODE_I8 ? launch<64, CODE_I8>(maps, p, sh, s) : launch<64, CODE_E4M3>(maps, p, sh, s);
}

}  // extern "C"
