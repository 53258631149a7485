// Decode attention for a batch whose sequences share long prefixes (tcgen05 / TMEM / TMA): a prefix is read once per KV head
// for all of its sequences' queries, a sequence's own keys once for its own.
//
//   out = sum_k exp(s_k - m) v_k / sum_k exp(s_k - m),   s_k = q . k / sqrt(hd),  over the prefix's keys and the own ones
//
// A segment is a prefix or the own keys of one sequence.  Its rows are the query heads of a KV head's group, of all tokens
// that see it: a whole group of sequences makes one product with many rows where one sequence makes G.  An item is a segment,
// a KV head and a row tile (as many whole tokens as 128 rows hold); its keys come in tiles of 64.  The tiles of all items form
// one line, each item with OV places more for what starting and ending it costs, cut into equal stretches, one for each
// resident CTA (two per SM), whatever the lengths: the host knows none.  Every piece of an item that lies in a stretch leaves
// (o, m, l) in fp32 in the scratch, and a second kernel joins, for each row, the pieces of its prefix and of its own keys in
// order of the line, so results do not depend on scheduling.
//
// Within a stretch, per tile:
//   S = Q K^T      M = 128 rows, N = 64 keys, fp32 in TMEM, two buffers: the product of the next tile runs beside this softmax
//   softmax        four warps, a row a thread: running maximum and sum in fp32.  P goes into TMEM in place of S, as two numbers of
//                  q's type (the rounded P and what that left, 16 and 22 bits: one alone is as coarse as the result, and its error
//                  shows where the terms of a row cancel); the two fill exactly the columns that S had.  Warps without rows (a
//                  single sequence has G) only keep the protocol.
//   O += P V       P from TMEM; fp32 in TMEM, rescaled when a row's maximum has grown by more than 8 (log2).  P is below 256; fp16
//                  has it 2^7 times as large (O and the sum too, so it cancels): good to 2^-32 of a row's largest weight.  The
//                  tensor cores' additions are cut off rather than rounded: 256 requests behind 16000 keys come out 2e-5 too small.
// K's place in the ring is free once S is complete, V's after P V; each has a warp that asks for the next.  The ring runs on
// over the items' borders, and the next item's Q is fetched while the last tile of the one before is finished.
//
// Nothing of a key that a row does not see reaches it: scores are masked by selection, V rows behind the length are zeroed
// in shared memory, pages that do not exist are read as zeros (a TMA box outside the tensor).  Of a draft's last tokens, which
// only later rows see, infinities and NaN in V are taken out of the product and added to the rows that see them at the end.  A sum
// that is no number, since either half of a weight may be zero or negative, is made anew from such values: see repair().
//
// Every wait is bounded by a second; the rows of a piece whose wait ran out become NaN.
#include <cuda.h>
#include <cuda_bf16.h>
#include <string.h>

#include "es_internal.cuh"
#include "launch.cuh"
#include "sm100.cuh"

namespace es {
namespace {

constexpr int KT = 64;                   // keys of a tile
constexpr int THREADS = 256;             // K and Q, MMA, V, records, four softmax warps
constexpr int TMEM_COLS = 256;           // S: two buffers of 64 columns, O: up to 128
constexpr float GAP = 8.0f;
constexpr int OV = 2;                    // places on the line that an item takes besides its tiles
constexpr int MIN_UNITS = 2 + OV;        // places of a stretch, at least
constexpr int MAX_SEGMENTS = 8192;

struct alignas(64) PrefixMaps { CUtensorMap q, q_own, k, v; };   // q_own: boxes of one sequence's rows

struct PrefixParams {
  const int *prefix_table, *prefix_len, *begin, *table, *ctx;
  const void* v_pages;
  void* out;
  int4* records;                         // scratch: two for every sequence, where its row's pieces are
  float *ml_p, *o_p, *ml_o, *o_o;        // pieces of prefixes and of own keys: [rows][2], [rows][hd]
  int B, T, Hq, Hkv, G, P, log2P, groups, prefix_pages, pps, n_pages, max_prefix, max_ctx;
  int TT;                                // tokens of a row tile
  int own_row_tiles, own_rows;           // of one sequence: row tiles; rows of the first (own_q: they fit a quarter of the tile)
  int own_q;
  int box;                               // tokens of a page that one copy brings
  float scale_log2e;
  float one;                             // 1, which the compiler does not know: with a known factor it makes one fused operation of two packed ones
};

// A piece of an item: what one CTA does of it.
struct Piece {
  int seg, group, kvh, rt;               // segment; group: it is a prefix
  int tok0, ntok;                        // its tokens (token = sequence * T + t)
  int len;                               // its keys
  int j0, j1;                            // tiles of the piece
};

__device__ __forceinline__ int tiles_of(int len) { return (len + KT - 1) / KT; }

// CTAs that share the line of `units` places, and which has which
__device__ __forceinline__ int active(int units, int ctas) { return max(1, min(ctas, units / MIN_UNITS)); }
__device__ __forceinline__ int start_of(int cta, int units, int n) { return (int)((long long)units * cta / n); }
__device__ __forceinline__ int cta_of(int unit, int units, int n) {
  // below 2^39 over below 2^30: a double's quotient is off by less than its distance from the next whole number
  return (int)(((double)(unit + 1) * n - 1.0) / (double)units);
}

// The pieces of a stretch, one after the other.  Only the first is searched for.
struct Walk {
  const PrefixParams& p;
  const int *line, *lens, *first;
  int u, end, item, a, row_tiles;                         // place on the line; item of the segment, place in the item
  Piece x;
  __device__ __forceinline__ Walk(const PrefixParams& p_, const int* line_, const int* lens_, const int* first_, int u_, int end_)
      : p(p_), line(line_), lens(lens_), first(first_), u(u_), end(end_), item(-1) {}
  __device__ __forceinline__ void segment(int s) {
    x.seg = s;
    x.group = s < p.groups;
    x.len = lens[s];
    if (x.group) {
      x.tok0 = first[s] * p.T;
      x.ntok = (first[s + 1] - first[s]) * p.T;
      row_tiles = (x.ntok + p.TT - 1) / p.TT;
    } else {
      x.tok0 = (s - p.groups) * p.T;
      x.ntok = p.T;
      row_tiles = p.own_row_tiles;
    }
  }
  __device__ __forceinline__ bool next() {
    while (u < end) {
      if (item < 0) {
        int lo = 0, hi = p.groups + p.B;                  // line[lo] <= u < line[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (line[mid] <= u) lo = mid; else hi = mid;
        }
        segment(lo);
        const int k = tiles_of(x.len) + OV, r = u - line[lo];
        item = r / k;
        a = r - item * k;
        x.kvh = item / row_tiles;
        x.rt = item - x.kvh * row_tiles;
      } else {                                            // the item before has ended: the stretch goes on
        a = 0;
        if (++x.rt == row_tiles) { x.rt = 0; ++x.kvh; }
        if (x.kvh == p.Hkv) {
          int s = x.seg + 1;
          while (line[s + 1] == u) ++s;                   // segments without places; u < end <= line[segments]
          segment(s);
          x.kvh = x.rt = 0;
        }
      }
      const int take = min(tiles_of(x.len) + OV - a, end - u);
      x.j0 = max(0, a - OV);
      x.j1 = max(0, a + take - OV);
      u += take;
      if (x.j1 > x.j0) return true;
    }
    return false;
  }
};

// Rows of a single sequence that fit a quarter of the tile go to one of the four by turns: the warp that has the quarter, and the
// part of the SM it runs on, differ between the CTAs that share an SM.
__device__ __forceinline__ int row_offset(const PrefixParams& p, const Piece& x) { return !x.group && p.own_q ? 32 * ((x.seg + x.kvh) & 3) : 0; }

// First row of a piece's partials, in the prefixes' or the own keys' part of the scratch: the rows of the items before it, and
// a tile's worth for each CTA before this one.
__device__ __forceinline__ int64_t piece_row(const PrefixParams& p, const Piece& x, int cta) {
  const int64_t before = (int64_t)x.tok0 * p.Hq + ((int64_t)x.kvh * x.ntok + (int64_t)x.rt * p.TT) * p.G;
  return before + (int64_t)cta * ((x.group ? p.TT : min(p.TT, p.T)) * p.G);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

// Two values rounded to q's type, and what that left of them.
template <bool BF16>
__device__ __forceinline__ uint32_t round_pair(float a, float b) {
  if (BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <bool BF16>
__device__ __forceinline__ uint32_t rest_pair(uint32_t w, float a, float b) {
  const float x = BF16 ? add_lo_bf16(w, -a) : add_lo_f16(w, -a), y = BF16 ? add_hi_bf16(w, -b) : add_hi_f16(w, -b);
  return round_pair<BF16>(-x, -y);
}

// The sums o of 32 columns, of keys k0 .. k1 - 1: infinities and NaN in V are added of the keys from `tail` on, which the product did
// not get.  Columns that are no number (the weights are) are made anew over all of these keys: the values that are not finite
// decide them alone; without one they stay what they are.  v: these columns of the KV head's first row in the pool.
template <int HD, bool BF16>
__device__ __noinline__ void repair(const int* pages, const uint16_t* v, int n_pages, int Hkv, int log2P, int k0, int k1, int tail, float* o) {
  uint32_t unknown = 0, found = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (o[i] != o[i]) { unknown |= 1u << i; o[i] = 0.f; }
  uint32_t open = unknown;                                     // not yet NaN for good
  for (int key = k1 - 1; key >= k0 && (key >= tail || open); --key) {
    const int page = pages[key >> log2P];
    if ((unsigned)page >= (unsigned)n_pages) continue;
    const uint16_t* at = v + ((((int64_t)page * Hkv) << log2P) + (key & ((1 << log2P) - 1))) * HD;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float f = BF16 ? __uint_as_float((uint32_t)at[i] << 16) : __half2float(*reinterpret_cast<const __half*>(at + i));
      if (isfinite(f)) continue;
      o[i] += f;
      found |= 1u << i;
      if (o[i] != o[i]) open &= ~(1u << i);
    }
  }
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if ((unknown & ~found) >> i & 1) o[i] = __uint_as_float(0x7fffffffu);
}

template <int HD>
struct Smem {
  static constexpr int HALVES = HD / 64;
  static constexpr int Q_BYTES = 128 * HD * 2, KV_BYTES = KT * HD * 2;
  static constexpr int BARS = 16;
  static constexpr size_t FIXED = 1024 + Q_BYTES + 4 * KV_BYTES + BARS * 8 + 128;
};

// Inclusive scan over the block of one value a thread, by `join`; the total goes to everyone.
template <class Join>
__device__ __forceinline__ int block_scan(int v, int* totals, int* all, Join join) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v = join(v, x); }
  __syncthreads();                                             // `totals` may still be read
  if (lane == 31) totals[warp] = v;
  __syncthreads();
  int sum = totals[0], before = 0;
#pragma unroll
  for (int w = 1; w < THREADS / 32; ++w) {
    if (w == warp) before = sum;
    sum = join(sum, totals[w]);
  }
  *all = sum;
  return warp ? join(before, v) : v;
}

template <int HD, bool BF16>
__global__ void __launch_bounds__(THREADS, 2) prefix_attn_kernel(const __grid_constant__ PrefixMaps maps, const PrefixParams p) {
  using L = Smem<HD>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char* q_s = smem;                                   // [halves][128 rows][128 B]
  unsigned char* k_s = q_s + L::Q_BYTES;                       // [2 stages][halves][64 rows][128 B]
  unsigned char* v_s = k_s + 2 * L::KV_BYTES;
  uint64_t* bars = (uint64_t*)(v_s + 2 * L::KV_BYTES);
  uint64_t *q_full = bars, *q_empty = bars + 1, *k_full = bars + 2, *k_empty = bars + 4, *v_full = bars + 6, *v_empty = bars + 8, *s_full = bars + 10,
           *p_full = bars + 12, *pv_done = bars + 14;           // [2] each but Q's, by the tile's parity
  uint32_t* tmem_slot = (uint32_t*)(bars + L::BARS);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  volatile int* pages_seen = (volatile int*)(tmem_slot + 2);   // [4] of the latest tiles: which 16 tokens lie in pages that exist
  volatile int* tail_bad = (volatile int*)(tmem_slot + 6);     // [2] of the latest pieces: the piece, if its last tokens hold a V that is no number.
                                                               // A warp may be one piece ahead of another, not two: p_full takes all four
  int* totals = (int*)(tmem_slot + 8);                         // [8]
  int* line = (int*)(tmem_slot + 16);                          // [segments + 1] places before
  int* lens = line + p.groups + p.B + 1;                       // [segments] keys
  int* first = lens + p.groups + p.B;                          // [groups + 1] first sequences

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    prefetch_tmap(&maps.q);
    prefetch_tmap(&maps.k);
    prefetch_tmap(&maps.v);
    for (int i = 0; i < L::BARS; ++i) mbar_init(smem_u32(&bars[i]), (i == 12 || i == 13) ? 4 : 1);   // p_full: four warps
    *abort_flag = 0;
    tail_bad[0] = tail_bad[1] = -1;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), TMEM_COLS);
  pdl_wait();

  // ---- the line ----
  const int segments = p.groups + p.B, per = (segments + THREADS) / THREADS, s0 = (int)threadIdx.x * per;      // `per` segments a thread
  for (int s = threadIdx.x; s <= segments; s += THREADS) {     // both loads are under way together
    const int g = p.groups && s <= p.groups ? p.begin[s] : 0;
    const int n = s < p.groups ? p.prefix_len[s] : s < segments ? p.ctx[s - p.groups] : 0;
    if (s < segments) lens[s] = min(max(n, 0), s < p.groups ? p.max_prefix : p.max_ctx);
    if (p.groups && s <= p.groups) first[s] = min(max(g, 0), p.B);
  }
  __syncthreads();
  {
    int all, sum = 0;
    const int to = p.groups ? min(s0 + per, p.groups + 1) : 0;
    bool disorder = false;
    for (int s = max(s0, 1); s < to; ++s) disorder |= first[s] < first[s - 1];
    if (__syncthreads_or(disorder)) {
      // a group begins no earlier than those before it end
      int top = 0;
      for (int s = s0; s < to; ++s) top = max(top, first[s]);
      top = block_scan(top, totals, &all, [](int a, int b) { return max(a, b); });
      int before = __shfl_up_sync(0xffffffffu, top, 1);
      if (lane == 0) { before = 0; for (int w = 0; w < warp; ++w) before = max(before, totals[w]); }
      for (int s = s0; s < to; ++s) { before = max(before, first[s]); first[s] = before; }
      __syncthreads();
    }
    auto places = [&](int s) {
      const int row_tiles = s < p.groups ? ((first[s + 1] - first[s]) * p.T + p.TT - 1) / p.TT : p.own_row_tiles;
      return lens[s] > 0 ? p.Hkv * row_tiles * (tiles_of(lens[s]) + OV) : 0;
    };
    for (int s = s0; s < min(s0 + per, segments); ++s) sum += places(s);
    int at = block_scan(sum, totals, &all, [](int a, int b) { return a + b; }) - sum;
    for (int s = s0; s < min(s0 + per, segments); ++s) { line[s] = at; at += places(s); }
    if (threadIdx.x == 0) line[segments] = all;
  }
  tc_fence_before();
  __syncthreads();
  pdl_launch_dependents();          // every CTA has its TMEM before a kernel behind this one can take any and then wait for this one's end
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot, tmem_s = tmem_base, tmem_o = tmem_base + 128;
  const int units = line[segments], ctas = active(units, (int)gridDim.x), cta = (int)blockIdx.x;
  const int u0 = cta < ctas ? start_of(cta, units, ctas) : 0, u1 = cta < ctas ? start_of(cta + 1, units, ctas) : 0;
  Walk walk(p, line, lens, first, u0, u1);
  const Piece& x = walk.x;

  if (warp == 0 || warp == 2) {
    // ---- TMA: K (and Q) or V; a lane per page of a tile ----
    const bool key = warp == 0;
    const int chunks = KT / p.box;                             // copies along the tile's keys
    const int lines = p.n_pages * p.Hkv * p.P;                 // outside the tensor: zeros
    uint64_t *full = key ? k_full : v_full, *empty = key ? k_empty : v_empty;
    unsigned char* ring = key ? k_s : v_s;
    const CUtensorMap* map = key ? &maps.k : &maps.v;
    int it = 0;
    bool ok = true;
    for (int pieces = 0; ok && walk.next(); ++pieces) {
      const int* pages = x.group ? p.prefix_table + (int64_t)x.seg * p.prefix_pages : p.table + (int64_t)(x.seg - p.groups) * p.pps;
      for (int j = x.j0; j < x.j1; ++j, ++it) {
        const int s = it & 1;
        int row = lines, here = 0;
        if (lane < chunks) {
          const int t0 = j * KT + lane * p.box;
          if (t0 < x.len) {
            const int page = pages[t0 >> p.log2P];
            if ((unsigned)page < (unsigned)p.n_pages) {
              row = (page * p.Hkv + x.kvh) * p.P + (t0 & (p.P - 1));
              here = ((1 << (p.box / 16)) - 1) << (lane * (p.box / 16));
            }
          }
        }
        here = __reduce_or_sync(0xffffffffu, here);
        ok = mbar_wait_soon(smem_u32(&empty[s]), ((it >> 1) & 1) ^ 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t fb = smem_u32(&full[s]);
        if (lane == 0) {
          if (key) pages_seen[it & 3] = here;                  // read by the softmax of this tile, which is over when K of it + 4 is asked for
          mbar_expect_tx(fb, L::KV_BYTES);
        }
        __syncwarp();
        if (lane < chunks) {
#pragma unroll
          for (int h = 0; h < L::HALVES; ++h) tma_load_2d(smem_u32(ring + s * L::KV_BYTES + h * (KT * 128) + lane * p.box * 128), map, h * 64, row, fb);
        }
        if (key && j == x.j0) {                                // the first tile is under way before Q's place is free
          ok = mbar_wait_soon(smem_u32(q_empty), (pieces & 1) ^ 1, abort_flag);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (lane == 0) {
            const bool few = !x.group && p.own_q;
            mbar_expect_tx(smem_u32(q_full), (few ? p.own_rows : p.TT * p.G) * HD * 2);
#pragma unroll
            for (int h = 0; h < L::HALVES; ++h)
              tma_load_3d(smem_u32(q_s + h * (128 * 128) + row_offset(p, x) * 128), few ? &maps.q_own : &maps.q, h * 64, x.kvh * p.G, x.tok0 + x.rt * p.TT,
                          smem_u32(q_full));
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      // ---- MMA: whichever of the next S product and the next P V is ready ----
      constexpr uint32_t type = BF16 ? (1u << 7) | (1u << 10) : 0u;
      constexpr uint32_t idesc_s = umma_idesc_f16(128, KT) | type;
      constexpr uint32_t idesc_o = umma_idesc_f16(128, HD) | type | (1u << 16);        // V is MN-major
      Walk ahead(p, line, lens, first, u0, u1);
      bool more_s = ahead.next(), more_o = walk.next();
      int s_it = 0, s_left = ahead.x.j1 - ahead.x.j0, s_piece = 0, o_it = 0, o_left = x.j1 - x.j0;
      bool s_first = true, o_first = true;
      uint64_t idle_since = 0;
      while (more_o) {
        bool progressed = false;
        if (more_s && s_it <= o_it + 1 && mbar_test(smem_u32(&k_full[s_it & 1]), (s_it >> 1) & 1) && (!s_first || mbar_test(smem_u32(q_full), s_piece & 1))) {
          tc_fence_after();
          const int s = s_it & 1;
          const uint32_t kb = smem_u32(k_s + s * L::KV_BYTES);
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            const int hf = k / 4, kk = k % 4;
            umma_f16(tmem_s + (uint32_t)(s * KT), umma_desc_sw128(smem_u32(q_s + hf * (128 * 128)) + kk * 32), umma_desc_sw128(kb + hf * (KT * 128) + kk * 32), idesc_s,
                     k > 0 ? 1u : 0u);
          }
          umma_commit(smem_u32(&s_full[s]));
          umma_commit(smem_u32(&k_empty[s]));
          ++s_it;
          s_first = false;
          if (--s_left == 0) {                                 // the piece's last S product frees Q
            umma_commit(smem_u32(q_empty));
            more_s = ahead.next();
            s_left = ahead.x.j1 - ahead.x.j0;
            ++s_piece;
            s_first = true;
          }
          progressed = true;
        }
        // P is complete (and with it, on a piece's first tile, the way of the earlier O out of TMEM: the same warps did both)
        if (s_it > o_it && mbar_test(smem_u32(&p_full[o_it & 1]), (o_it >> 1) & 1) && mbar_test(smem_u32(&v_full[o_it & 1]), (o_it >> 1) & 1)) {
          tc_fence_after();
          const int s = o_it & 1;
          const uint32_t vb = smem_u32(v_s + s * L::KV_BYTES);
#pragma unroll
          for (int k = 0; k < KT / 8; ++k)                     // 16 keys, their weights' first halves and then the second
            umma_f16_ts(tmem_o, tmem_s + (uint32_t)(s * KT + k * 8), umma_desc_sw128_mn(vb + (k >> 1) * (16 * 128), KT * 128, 1024), idesc_o,
                        (!o_first || k > 0) ? 1u : 0u);
          umma_commit(smem_u32(&v_empty[s]));
          umma_commit(smem_u32(&pv_done[s]));
          ++o_it;
          o_first = false;
          if (--o_left == 0) {
            more_o = walk.next();
            o_left = x.j1 - x.j0;
            o_first = true;
          }
          progressed = true;
        }
        if (progressed) {
          idle_since = 0;
        } else {
          if (*abort_flag) break;
          const uint64_t now = global_timer_ns();
          if (idle_since == 0) idle_since = now;
          if (now - idle_since > 1000000000ull) { *abort_flag = 1; break; }      // a second without progress
        }
      }
    }
  } else if (warp == 3) {
    // ---- for the second kernel: where the pieces of a sequence's rows are ----
    for (int b = cta + lane * (int)gridDim.x; b < p.B; b += 32 * (int)gridDim.x) {
      int lo = -1, hi = p.groups;                              // first[lo] <= b < first[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= b) lo = mid; else hi = mid;
      }
      int4 r = make_int4(0, 0, 0, 0);
      if (p.groups && lo >= 0 && b < first[lo + 1]) r = make_int4(line[lo], tiles_of(lens[lo]), first[lo] * p.T, (first[lo + 1] - first[lo]) * p.T);
      p.records[2 * b] = r;
      p.records[2 * b + 1] = make_int4(line[p.groups + b], tiles_of(lens[p.groups + b]), units, 0);
    }
  } else {
    // ---- softmax: thread = row, TMEM lane quarter = warp % 4 ----
    const int quarter = warp & 3, e = (int)threadIdx.x - 128;
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const int token0 = (quarter * 32 + lane) / p.G, lane_token = lane / p.G;
    int it = 0;
    bool ok = true;
    for (int pieces = 0; walk.next(); ++pieces) {
      const int off = row_offset(p, x), r = quarter * 32 + lane - off;
      const int token = x.rt * p.TT + (off ? lane_token : token0);                            // of the segment
      const bool real = r >= 0 && r < (x.group ? p.TT * p.G : p.own_rows) && token < x.ntok;
      const bool idle = !__any_sync(0xffffffffu, real);
      const int lim = !real ? 0 : x.group ? x.len : min(x.len, x.len - p.T + token + 1);      // keys that the row sees
      const int tail = x.group ? x.len : max(0, x.len - p.T + 1);                             // keys from here on are seen by some rows only
      float m_ref = -INFINITY, l_run = 0.f;
      for (int j = x.j0; j < x.j1 && ok; ++j, ++it) {
        const int s = it & 1, k0 = j * KT;
        ok = mbar_wait_soon(smem_u32(&s_full[s]), (it >> 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        bool move = false;
        float alpha = 1.f;
        if (!idle) {
          uint32_t sr[2][32];
          const uint32_t ts = tmem_s + (uint32_t)(s * KT) + lane_off;
          tmem_ld_issue(ts, sr[0]);
          tmem_ld_issue(ts + 32, sr[1]);
          tmem_ld_wait(sr[0]);
          tmem_ld_wait(sr[1]);
          float sc[KT];
#pragma unroll
          for (int c = 0; c < KT; ++c) sc[c] = __uint_as_float(sr[c / 32][c % 32]);
          const int nk = lim - k0, seen = pages_seen[it & 3];
          if (__any_sync(0xffffffffu, nk < KT) || seen != 15) {
#pragma unroll
            for (int c = 0; c < KT; ++c) sc[c] = (c < nk && ((seen >> (c / 16)) & 1)) ? sc[c] : -INFINITY;
          }
          float mx4[4] = {sc[0], sc[1], sc[2], sc[3]};
#pragma unroll
          for (int c = 4; c < KT - 4; c += 8)
#pragma unroll
            for (int q = 0; q < 4; ++q) mx4[q] = max3(mx4[q], sc[c + 2 * q], sc[c + 2 * q + 1]);
          float mx = max3(max3(mx4[0], mx4[1], mx4[2]), mx4[3], max3(max3(sc[KT - 4], sc[KT - 3], sc[KT - 2]), sc[KT - 1], -INFINITY));
          mx = __fmul_rn(mx, p.scale_log2e);                   // rounded, as the scores below are
          // m_ref: what exponents are counted from, LIFT below the maximum that it was taken of.  An exponent is the rounded score's
          // distance from it, as the maximum's is: it exceeds LIFT + GAP for no score, however large a score's own step is.
          constexpr float LIFT = BF16 ? 0.f : 7.f;
          move = mx - m_ref > LIFT + GAP;
          const float m_new = move ? mx - LIFT : m_ref, m_use = m_new == -INFINITY ? 0.f : m_new;
          alpha = move ? ex2(m_ref - m_use) : 1.f;
          const uint64_t scale2 = pack_f32x2(p.scale_log2e, p.scale_log2e), minus2 = pack_f32x2(-m_use, -m_use), one2 = pack_f32x2(p.one, p.one);
          uint64_t sum[2] = {0, 0};
#pragma unroll
          for (int half = 0; half < 2; ++half) {               // 16 keys take 8 columns for their weights and 8 for the rest of them
            uint32_t packed[32];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int c = half * 32 + 2 * i, at = (i >> 3) * 16 + (i & 7);
              const float2 t = unpack_f32x2(fma_f32x2(mul_f32x2(pack_f32x2(sc[c], sc[c + 1]), scale2), one2, minus2));
              const float a = ex2(t.x), b = ex2(t.y);
              packed[at] = round_pair<BF16>(a, b);
              packed[at + 8] = rest_pair<BF16>(packed[at], a, b);
              sum[i & 1] = fma_f32x2(pack_f32x2(a, b), one2, sum[i & 1]);
            }
            tmem_st32_words_issue(ts + half * 32, packed);
          }
          const float2 s0 = unpack_f32x2(sum[0]), s1 = unpack_f32x2(sum[1]);
          l_run = l_run * alpha + ((s0.x + s0.y) + (s1.x + s1.y));
          tmem_st_wait();
          m_ref = m_new;
        }
        if (x.len - k0 < KT || k0 + KT > tail) {
          // V is touched: keys behind the length become zeros; of keys that only later tokens see, what is no number leaves the product
          ok = mbar_wait_soon(smem_u32(&v_full[s]), (it >> 1) & 1, abort_flag);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          unsigned char* vt = v_s + s * L::KV_BYTES;
          const int from = min(KT, x.len - k0);
          for (int i = e; i < (KT - from) * (HD / 8); i += 128) {
            const int row = from + i / (HD / 8), c = i % (HD / 8);
            *reinterpret_cast<uint4*>(vt + (c >> 3) * (KT * 128) + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          if (tail < x.len) {
            const int f = max(0, tail - k0);
            for (int i = e; i < (from - f) * (HD / 2); i += 128) {
              const int row = f + i / (HD / 2), c = i % (HD / 2);
              uint32_t* at = reinterpret_cast<uint32_t*>(vt + (c >> 5) * (KT * 128) + row * 128 + (c & 31) * 4);
              const uint32_t w = *at, inf = BF16 ? 0x7f80u : 0x7c00u;
              uint32_t keep = 0xffffffffu;
              if ((w & inf) == inf) keep &= 0xffff0000u;
              if (((w >> 16) & inf) == inf) keep &= 0xffffu;
              if (keep != 0xffffffffu) { *at = w & keep; tail_bad[pieces & 1] = pieces; }
            }
          }
          fence_proxy_async_smem();
        }
        if (j > x.j0 && __any_sync(0xffffffffu, move)) {
          // O is rescaled once P V of the tile before has landed
          ok = mbar_wait_soon(smem_u32(&pv_done[s ^ 1]), ((it - 1) >> 1) & 1, abort_flag);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            float o[32];
            tmem_ld32(tmem_o + lane_off + c, o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= alpha;
            tmem_st32(tmem_o + lane_off + c, o);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&p_full[s]));
      }
      if (ok) {
        ok = mbar_wait_soon(smem_u32(&pv_done[(it - 1) & 1]), ((it - 1) >> 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
      }
      // the piece's part of its rows
      const int64_t row = piece_row(p, x, cta) + r;
      float* ml = (x.group ? p.ml_p : p.ml_o) + row * 2;
      float* po = (x.group ? p.o_p : p.o_o) + row * HD;
      if (!idle) {
        if (real) *reinterpret_cast<float2*>(ml) = ok ? make_float2(m_ref, l_run) : make_float2(0.f, __uint_as_float(0x7fffffffu));
        const bool bad = tail_bad[pieces & 1] == pieces;
        if (ok) {
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            float o[32];
            __syncwarp();
            tmem_ld32(tmem_o + lane_off + c, o);
            uint64_t z = 0;                                    // no number if one of them is none
#pragma unroll
            for (int i = 0; i < 32; i += 2) z = fma_f32x2(pack_f32x2(o[i], o[i + 1]), 0, z);
            const float2 zz = unpack_f32x2(z);
            if ((bad || !(zz.x + zz.y == 0.f)) && l_run < INFINITY) {
              float t[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) t[i] = o[i];
              repair<HD, BF16>(x.group ? p.prefix_table + (int64_t)x.seg * p.prefix_pages : p.table + (int64_t)(x.seg - p.groups) * p.pps,
                               (const uint16_t*)p.v_pages + (int64_t)x.kvh * p.P * HD + c, p.n_pages, p.Hkv, p.log2P, x.j0 * KT, min(lim, x.j1 * KT), tail, t);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = t[i];
            }
            if (real) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(po + c + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
            }
          }
        }
      }
      tc_fence_before();
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    if (*abort_flag) settle();
    tmem_dealloc(tmem_base, TMEM_COLS);
  }
}

// ---- the pieces of a row, joined in order of the line: a warp per token and head ------------------

constexpr int JOIN_WARPS = 4;

template <int HD, bool BF16>
__global__ void __launch_bounds__(JOIN_WARPS * 32) prefix_join_kernel(const PrefixParams p, const int ctas) {
  pdl_launch_dependents();
  constexpr int D = HD / 32;                                   // values of a lane
  const int lane = threadIdx.x & 31;
  const unsigned at = blockIdx.x * JOIN_WARPS + (threadIdx.x >> 5);             // below 2^26 + 4
  const int token = (int)(at / (unsigned)p.Hq), h = (int)(at - (unsigned)token * p.Hq), kvh = h / p.G, g = h - kvh * p.G, b = token / p.T;
  pdl_wait();
  if (b >= p.B) return;
  const int4 shared = p.records[2 * b], mine = p.records[2 * b + 1];
  const int units = mine.z, n = active(units, ctas);
  float top = -INFINITY, sum = 0.f, o[D];
#pragma unroll
  for (int i = 0; i < D; ++i) o[i] = 0.f;
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    const int tiles = part == 0 ? shared.y : mine.y;
    if (tiles == 0) continue;
    Piece x;
    x.group = part == 0;
    x.tok0 = x.group ? shared.z : b * p.T;
    x.ntok = x.group ? shared.w : p.T;
    x.kvh = kvh;
    const int local = token - x.tok0, row_tiles = (x.ntok + p.TT - 1) / p.TT;
    x.rt = local / p.TT;
    const int u = (x.group ? shared.x : mine.x) + (kvh * row_tiles + x.rt) * (tiles + OV) + OV, c0 = cta_of(u, units, n), c1 = cta_of(u + tiles - 1, units, n);
    const int64_t row0 = piece_row(p, x, 0) + (local - x.rt * p.TT) * p.G + g, step = piece_row(p, x, 1) - piece_row(p, x, 0);
    const float *ml = x.group ? p.ml_p : p.ml_o, *po = x.group ? p.o_p : p.o_o;
    for (int base = c0; base <= c1; base += 32) {
      const int c = base + lane;
      float2 v = make_float2(-INFINITY, 0.f);
      if (c <= c1) v = *reinterpret_cast<const float2*>(ml + (row0 + c * step) * 2);
      float m = v.x;
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
      const float m_new = fmaxf(top, m);
      const float use = m_new == -INFINITY ? 0.f : m_new, old = ex2(top - use), f = ex2(v.x - use);
      float l = v.y * f;
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
      sum = sum * old + l;
      top = m_new;
#pragma unroll
      for (int i = 0; i < D; ++i) o[i] *= old;
      const int k = min(32, c1 - base + 1);
#pragma unroll 4
      for (int q = 0; q < k; ++q) {
        const float w = __shfl_sync(0xffffffffu, f, q);
        const float* src = po + (row0 + (base + q) * step) * HD + lane * D;
        if (D == 4) {
          const float4 t = *reinterpret_cast<const float4*>(src);
          o[0] = fmaf(t.x, w, o[0]); o[1] = fmaf(t.y, w, o[1]); o[2] = fmaf(t.z, w, o[2]); o[D - 1] = fmaf(t.w, w, o[D - 1]);
        } else {
          const float2 t = *reinterpret_cast<const float2*>(src);
          o[0] = fmaf(t.x, w, o[0]); o[1] = fmaf(t.y, w, o[1]);
        }
      }
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* out = (uint16_t*)p.out + (int64_t)at * HD + lane * D;
  uint32_t w[D / 2];
#pragma unroll
  for (int i = 0; i < D; i += 2) {
    if (BF16) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(o[i] * inv, o[i + 1] * inv);
      w[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
    } else {
      const __half2 v = __floats2half2_rn(o[i] * inv, o[i + 1] * inv);
      w[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
    }
  }
  if (D == 4) *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[D / 2 - 1]);
  else *reinterpret_cast<uint32_t*>(out) = w[0];
}

// ---- host ------------------------------------------------------------------------------------------

struct Layout {
  size_t records, ml_p, o_p, ml_o, o_o, bytes;
};

int tokens_of_tile(int G) { return 128 / G; }

Layout layout_of(int groups, int B, int T, int Hq, int G, int hd) {
  const int TT = tokens_of_tile(G);
  const int64_t ctas = 2LL * sm_count(), rows = (int64_t)B * T * Hq;
  const int64_t rows_p = groups ? rows + ctas * (TT * G) : 0, rows_o = rows + ctas * ((TT < T ? TT : T) * G);
  Layout l;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  l.records = take((size_t)B * 2 * sizeof(int4));
  l.ml_p = take((size_t)rows_p * 8);
  l.o_p = take((size_t)rows_p * hd * 4);
  l.ml_o = take((size_t)rows_o * 8);
  l.o_o = take((size_t)rows_o * hd * 4);
  l.bytes = at;
  return l;
}

es_status_t check_sizes(int groups, int B, int T, int Hq, int Hkv, int hd) {
  if (groups < 0 || B <= 0 || T <= 0 || Hq <= 0 || Hkv <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (Hq % Hkv || Hq / Hkv > 128) return fail(ES_ERR_SHAPE, "Hq must be a multiple of Hkv, at most 128 times as many");
  if (hd != 64 && hd != 128) return fail(ES_ERR_SHAPE, "head_dim must be 64 or 128");
  if ((long long)groups + B > MAX_SEGMENTS) return fail(ES_ERR_RANGE, "more than %d prefixes and sequences", MAX_SEGMENTS);
  if ((long long)B * T * Hq > (1 << 26)) return fail(ES_ERR_RANGE, "more than 2^26 query heads");
  return ES_OK;
}

template <int HD, bool BF16>
es_status_t launch(const PrefixMaps& maps, const PrefixParams& p, cudaStream_t s) {
  auto kern = prefix_attn_kernel<HD, BF16>;
  const size_t smem = Smem<HD>::FIXED + (size_t)(2 * (p.groups + p.B) + p.groups + 2) * 4;
  static std::atomic<uint64_t> allowed{0};
  ES_CUDA_CHECK(allow_shared_memory(kern, 227 * 1024, &allowed));
  const bool pdl = tunables().pdl != 0;
  // two CTAs share an SM while both fit
  const int ctas = (smem <= 112 * 1024 ? 2 : 1) * sm_count();
  ES_CUDA_CHECK(launch_kernel(kern, dim3(ctas), dim3(THREADS), smem, s, pdl, maps, p));
  const int64_t rows = (int64_t)p.B * p.T * p.Hq;
  ES_CUDA_CHECK(launch_kernel(prefix_join_kernel<HD, BF16>, dim3((unsigned)((rows + JOIN_WARPS - 1) / JOIN_WARPS)), dim3(JOIN_WARPS * 32), 0, s, pdl, p, ctas));
  return ES_OK;
}

}  // namespace
}  // namespace es

using namespace es;

extern "C" size_t es_op_decode_attention_prefix_scratch_bytes(int32_t groups, int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t hd) {
  if (check_sizes(groups, B, T, Hq, Hkv, hd) != ES_OK) return 0;
  return layout_of(groups, B, T, Hq, Hq / Hkv, hd).bytes;
}

extern "C" es_status_t es_op_decode_attention_prefix(const void* q, int32_t dtype, int64_t q_stride, const void* k_pages, const void* v_pages,
                                                     const int32_t* prefix_table, const int32_t* prefix_len, const int32_t* group_begin, int32_t groups,
                                                     int32_t prefix_pages, const int32_t* block_table, const int32_t* ctx_len, void* out, int32_t B, int32_t T,
                                                     int32_t Hq, int32_t Hkv, int32_t hd, int32_t page_tokens, int32_t pages_per_seq, int32_t n_pages,
                                                     int32_t max_prefix, int32_t max_ctx, void* scratch, size_t scratch_bytes, void* stream) {
  if (dtype != ES_DTYPE_F16 && dtype != ES_DTYPE_BF16) return fail(ES_ERR_INVALID_ARG, "q and pages must be fp16 or bf16");
  ES_TRY(check_sizes(groups, B, T, Hq, Hkv, hd));
  if (!q || !k_pages || !v_pages || !block_table || !ctx_len || !out || (groups && (!prefix_table || !prefix_len || !group_begin)))
    return fail(ES_ERR_INVALID_ARG, "null argument");
  if (page_tokens < 16 || (page_tokens & (page_tokens - 1))) return fail(ES_ERR_SHAPE, "page_tokens must be a power of two, at least 16");
  if (n_pages <= 0 || pages_per_seq <= 0 || max_ctx <= 0 || (groups && (prefix_pages <= 0 || max_prefix <= 0))) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if ((long long)max_ctx > (long long)page_tokens * pages_per_seq || (groups && (long long)max_prefix > (long long)page_tokens * prefix_pages))
    return fail(ES_ERR_RANGE, "max_ctx or max_prefix exceeds its block table");
  if ((long long)n_pages * Hkv * page_tokens > INT32_MAX - 256) return fail(ES_ERR_RANGE, "a page pool exceeds 2^31 rows");
  if (max_ctx > (1 << 30) || max_prefix > (1 << 30)) return fail(ES_ERR_RANGE, "max_ctx or max_prefix exceeds 2^30");
  if (q_stride % 8 || q_stride < (int64_t)Hq * hd || q_stride > (1LL << 38)) return fail(ES_ERR_INVALID_ARG, "q_stride must be a multiple of 8, at least Hq * hd");
  if (((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)scratch) % 16 || (uintptr_t)out % 8)
    return fail(ES_ERR_INVALID_ARG, "q, pages and scratch must be 16-byte aligned, out 8-byte aligned");
  const int G = Hq / Hkv, TT = tokens_of_tile(G);
  // tiles on the line: every token's row tiles, a part of one more for each group
  const long long own_tiles = (max_ctx + KT - 1) / KT + OV, prefix_tiles = groups ? (max_prefix + KT - 1) / KT + OV : 0;
  const long long line = Hkv * (B * (long long)((T + TT - 1) / TT) * own_tiles + ((long long)B * T / TT + 1 + groups) * prefix_tiles);
  if (line > (1LL << 30)) return fail(ES_ERR_RANGE, "heads * tokens * keys exceed one launch");
  const Layout l = layout_of(groups, B, T, Hq, G, hd);
  if (!scratch || scratch_bytes < l.bytes) return fail(ES_ERR_WORKSPACE, "scratch: %zu bytes given, %zu needed", scratch ? scratch_bytes : (size_t)0, l.bytes);

  PrefixParams p{};
  p.prefix_table = prefix_table; p.prefix_len = prefix_len; p.begin = group_begin; p.table = block_table; p.ctx = ctx_len;
  p.v_pages = v_pages;
  p.out = out;
  char* base = (char*)scratch;
  p.records = (int4*)(base + l.records);
  p.ml_p = (float*)(base + l.ml_p); p.o_p = (float*)(base + l.o_p); p.ml_o = (float*)(base + l.ml_o); p.o_o = (float*)(base + l.o_o);
  p.B = B; p.T = T; p.Hq = Hq; p.Hkv = Hkv; p.G = G; p.P = page_tokens; p.groups = groups;
  while ((1 << p.log2P) < page_tokens) ++p.log2P;
  p.prefix_pages = prefix_pages; p.pps = pages_per_seq; p.n_pages = n_pages; p.max_prefix = groups ? max_prefix : 0; p.max_ctx = max_ctx;
  p.TT = TT;
  p.own_row_tiles = (T + TT - 1) / TT;
  p.own_rows = (T < TT ? T : TT) * G;
  p.own_q = p.own_rows <= 32;
  p.box = page_tokens < KT ? page_tokens : KT;
  p.scale_log2e = 1.4426950408889634f / sqrtf((float)hd);
  p.one = 1.f;
  PrefixMaps maps = {};
  ES_TRY(tma_encode_3d_f16(&maps.q, q, (int64_t)B * T, Hq, hd, q_stride, TT, G));
  if (p.own_q) ES_TRY(tma_encode_3d_f16(&maps.q_own, q, (int64_t)B * T, Hq, hd, q_stride, T, G));
  const int64_t lines = (int64_t)n_pages * Hkv * page_tokens;
  ES_TRY(tma_encode_2d_f16(&maps.k, k_pages, lines, hd, hd, p.box));
  ES_TRY(tma_encode_2d_f16(&maps.v, v_pages, lines, hd, hd, p.box));
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == ES_DTYPE_F16) return hd == 128 ? launch<128, false>(maps, p, s) : launch<64, false>(maps, p, s);
  return hd == 128 ? launch<128, true>(maps, p, s) : launch<64, true>(maps, p, s);
}
