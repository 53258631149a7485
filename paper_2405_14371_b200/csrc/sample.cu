// Sampling the next token of every row of logits: temperature, top-k, top-p, min-p, one given random number per row.
//
// No row is sorted.  Every restriction keeps a prefix of the ranking (by logit, equal ones by index), so each is a
// threshold in that order, held as one 64-bit number, the logit's order-preserving bits above the complement of the
// index.  A histogram over the distance from the largest logit (counts, and weights where top-p asks for them) says in
// which bin a threshold lies; the few elements of that bin are collected, ranked and searched.  A bin with more elements
// than the list takes (many equal logits) is descended by the bits of its keys instead.  The draw is a search for a
// running weight in order of index.
//
// Weights are integers, w = round(2^44 exp2((x - max) log2(e) / temperature)) out of 64-bit arithmetic, so every sum
// is exact whatever its order: thresholds and tokens depend on the inputs alone, and the borders are as sharp as the
// exponential (2^-39).
//
// A row belongs to a cluster of 1 to 8 CTAs, each holding a slice of the row in shared memory as fp32: the logits are read
// from HBM once, whatever the number of passes.
#include <cooperative_groups.h>
#include <limits.h>

#include "es_internal.cuh"
#include "kv8.cuh"
#include "launch.cuh"

namespace cg = cooperative_groups;

namespace es {
namespace {

typedef unsigned long long u64;

constexpr int ST = 512;                       // threads of a CTA
constexpr int SW = ST / 32;
constexpr int CHUNK = 128;                    // elements a warp sums at a time: the grain of the search
constexpr int MAX_CLUSTER = 8;
constexpr int MAX_V = 262144;                 // 2^18 weights of 2^44 stay below 2^63
constexpr int MAX_SLICE = MAX_V / MAX_CLUSTER;
constexpr int NB = 1024;                      // bins of the histogram
constexpr int LIST = 1024;                    // elements of a bin that are ranked directly
constexpr int FEW = 256;                      // candidates that the first CTA finishes by itself
constexpr double UNIT = 17592186044416.0;     // 2^44, the largest weight
constexpr float REACH = 46.f;                 // weights further than this (log2) below the largest round to zero

struct SampleParams {
  const void* logits;
  int64_t row_stride;
  const float *u, *temperature, *top_p, *min_p;
  const int* top_k;
  int* tokens;
  float* logprobs;
  int V, slice;                               // elements per CTA, a multiple of CHUNK
};

struct Shared {
  // one entry per CTA of the cluster, written by that CTA into everybody's copy: after the next cluster barrier each reads
  // its own memory
  u64 total[MAX_CLUSTER];
  u64 best[MAX_CLUSTER];                      // largest (key, index)
  float least[MAX_CLUSTER];                   // smallest finite logit
  int found;                                  // a chosen index, from the CTA that found it
  // from the first CTA
  int pick_bin, pick_count;                   // a bin, and how many elements it holds
  u64 pick_up_to;                             // elements up to and including that bin
  u64 pick_target;                            // rank (counts) or mass to reach within the bin
  u64 pick_pair;                              // threshold found in the list
  // this CTA's own
  u64 all_mass;
  int list_n;
  int few_n;                                  // first CTA: candidates that have arrived
  int base;
  u64 warp_a[SW], warp_b[SW];
  int digit;                                  // descent by key bits
  u64 digit_above, digit_here;
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// order-preserving integer of a float that is not NaN
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
  return v;
}
__device__ __forceinline__ u64 warp_scan(u64 v) {        // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 o = __shfl_up_sync(~0u, v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// 2^f on [-1/2, 1/2] by the polynomial through 9 Chebyshev nodes: relative error below 2^-39.7.
__device__ __forceinline__ double exp2_poly(double f) {
  double v = 1.3255224878668817e-6;
  v = fma(v, f, 1.53100794022492974e-5);
  v = fma(v, f, 1.54034558524538394e-4);
  v = fma(v, f, 1.33334505680006457e-3);
  v = fma(v, f, 9.61812915940255819e-3);
  v = fma(v, f, 5.55041094120593299e-2);
  v = fma(v, f, 2.40226506958129882e-1);
  v = fma(v, f, 6.93147180545933455e-1);
  return fma(v, f, 1.0);
}

// f of the whole, f in [0, 1): the integer part of f * all, exactly, and whether something was left (f * 2^64 is an
// integer for every fp32 f from 2^-40 on; a double cannot hold `all`)
__device__ __forceinline__ u64 share_of(float f, u64 all, bool* more) {
  const u64 fixed = (u64)((double)f * 18446744073709551616.0);
  *more = fixed * all != 0;
  return __umul64hi(fixed, all);
}

__device__ __forceinline__ u64 pair_key(uint32_t key, int index) { return ((u64)key << 32) | (uint32_t)~index; }

// One row's working state; every method is called by all threads of the cluster.
template <int ranks>
struct Row {
  float* x;                                   // slice in shared memory, padded with -infinity to a multiple of CHUNK
  u64* csum;                                  // [slice / CHUNK]
  uint32_t *cnt, *part;                       // [NB] counts, [3][NB] weights in three fields of 15 bits
  uint4* inbox;                               // [ranks][NB / ranks] this CTA's share of the bins, from every CTA
  uint32_t* ccnt;                             // [NB] the cluster's counts   (first CTA)
  u64* cmass;                                 // [NB] ... and weights
  u64 *list, *lweight;                        // [LIST] elements of a bin and their weights (first CTA)
  u64 *mine, *dhist, *dcomb;                  // this CTA's elements of a bin; sums of a descent by key bits
  Shared* sm;
  int n, first, rank;                         // padded elements, global index of the first, this CTA
  float xmax, bin_scale;
  double c;                                   // log2(e) / temperature
  float cf;
  u64 keep;                                   // kept: elements not below this in the ranking
  u64 least;                                  // ... whose weight is at least this

  __device__ __forceinline__ u64 weight(float v) const {
    if (v == xmax) return 1ull << 44;
    // far below: zero without 64-bit work (also -infinity, and anything finite below an infinite maximum)
    if (!(fmaf(v, 0.5f, -0.5f * xmax) * cf > -0.5f * REACH)) return 0;
    const double t = ((double)v - (double)xmax) * c;
    const double magic = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to an integer, which its low bits hold
    const double r = t + magic;
    const double f = t - (r - magic);
    const double scale = __hiloint2double((1023 + 44 + __double2loint(r)) << 20, 0);      // -47 <= r <= 0
    return (u64)__double_as_longlong(fma(exp2_poly(f), scale, 4503599627370496.0)) - 0x4330000000000000ull;
  }
  __device__ __forceinline__ bool kept(float v, int i) const { return pair_key(key_of(v), i) >= keep; }
  // bins grow with the distance from the largest logit; equal logits share one
  __device__ __forceinline__ int bin_of(float v) const {
    return v == xmax ? 0 : (int)fminf((xmax - v) * bin_scale, (float)(NB - 1));
  }

  // chunk sums of f(value, index) in csum, every CTA's sum in sm->total; returns the cluster's
  template <class F>
  __device__ u64 sums(F f) {
    cg::cluster_group cl = cg::this_cluster();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int ch = warp; ch < n / CHUNK; ch += SW) {
      const float4 v = *reinterpret_cast<const float4*>(x + ch * CHUNK + lane * 4);
      const int i = first + ch * CHUNK + lane * 4;
      const u64 s = warp_sum(f(v.x, i) + f(v.y, i + 1) + f(v.z, i + 2) + f(v.w, i + 3));
      if (lane == 0) csum[ch] = s;
    }
    __syncthreads();
    if (warp == 0) {
      u64 s = 0;
      for (int ch = lane; ch < n / CHUNK; ch += 32) s += csum[ch];
      s = warp_sum(s);
      if (lane < ranks) cl.map_shared_rank(sm, lane)->total[rank] = s;
    }
    cl.sync();
    u64 all = 0;
#pragma unroll
    for (int r = 0; r < ranks; ++r) all += sm->total[r];
    return all;
  }

  // after sums(f), in one warp: the first index of this CTA at which the running sum of f exceeds `target`, or -1 where
  // that is in another CTA
  template <class F>
  __device__ int find_here(F f, u64 target) {
    const int lane = threadIdx.x & 31;
    u64 run = 0;
    for (int r = 0; r < rank; ++r) run += sm->total[r];
    if (run > target || target >= run + sm->total[rank]) return -1;
    int ch = 0;
    for (int base = 0; base < n / CHUNK; base += 32) {
      const u64 v = base + lane < n / CHUNK ? csum[base + lane] : 0;
      const u64 inc = run + warp_scan(v);
      const unsigned hit = __ballot_sync(~0u, inc > target);
      if (hit) {
        const int l = __ffs(hit) - 1;
        ch = base + l;
        run = __shfl_sync(~0u, inc - v, l);
        break;
      }
      run = __shfl_sync(~0u, inc, 31);
    }
    const float4 v = *reinterpret_cast<const float4*>(x + ch * CHUNK + lane * 4);
    const int i = first + ch * CHUNK + lane * 4;
    const u64 a = f(v.x, i), b = a + f(v.y, i + 1), d = b + f(v.z, i + 2), e = d + f(v.w, i + 3);
    const u64 inc = run + warp_scan(e), base = inc - e;
    const unsigned hit = __ballot_sync(~0u, inc > target);
    const int at = i + (base + a > target ? 0 : base + b > target ? 1 : base + d > target ? 2 : 3);
    return __shfl_sync(~0u, at, __ffs(hit) - 1);
  }

  // the same, in every CTA
  template <class F>
  __device__ int find(F f, u64 target) {
    cg::cluster_group cl = cg::this_cluster();
    if (threadIdx.x < 32) {
      const int got = find_here(f, target);
      if (got >= 0 && threadIdx.x < ranks) cl.map_shared_rank(sm, threadIdx.x)->found = got;
    }
    cl.sync();
    const int got = sm->found;
    cl.sync();                                // before anybody's next use of `found` and `total`
    return got;
  }

  // The largest key at which the running sum of f, keys descending, reaches `target` (>= 1, <= the whole sum);
  // *above = sum over larger keys, *here = sum at the key.
  template <class F>
  __device__ uint32_t descend(F f, u64 target, u64* above, u64* here) {
    cg::cluster_group cl = cg::this_cluster();
    uint32_t prefix = 0;
    u64 run = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < 256; i += ST) dhist[i] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += ST) {
        const float v = x[i];
        const uint32_t k = key_of(v);
        if (shift == 24 || (k >> (shift + 8)) == prefix) {
          const u64 w = f(v, first + i);
          if (w) atomicAdd(&dhist[(k >> shift) & 255], w);
        }
      }
      cl.sync();
      for (int i = threadIdx.x; i < 256; i += ST) {
        u64 s = 0;
        for (int r = 0; r < ranks; ++r) s += cl.map_shared_rank(dhist, r)[i];
        dcomb[i] = s;
      }
      cl.sync();
      if (threadIdx.x < 32) {                 // lane l holds bins 255 - 8 l down to 248 - 8 l
        const int lane = threadIdx.x;
        u64 v[8], s = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) { v[j] = dcomb[255 - 8 * lane - j]; s += v[j]; }
        const u64 inc = run + warp_scan(s);
        const unsigned hit = __ballot_sync(~0u, inc >= target);
        if (hit && lane == __ffs(hit) - 1) {
          u64 r = inc - s;
          int j = 0;
          while (j < 7 && r + v[j] < target) r += v[j++];
          sm->digit = 255 - 8 * lane - j;
          sm->digit_above = r;
          sm->digit_here = v[j];
        }
      }
      __syncthreads();
      prefix = (prefix << 8) | (uint32_t)sm->digit;
      run = sm->digit_above;
      *here = sm->digit_here;
      __syncthreads();
    }
    *above = run;
    return prefix;
  }

  // Counts per bin, and weights where asked, summed over the cluster in the first CTA.
  __device__ void histogram(bool mass) {
    cg::cluster_group cl = cg::this_cluster();
    for (int i = threadIdx.x; i < (mass ? NB : NB / 4); i += ST) reinterpret_cast<uint4*>(cnt)[i] = make_uint4(0, 0, 0, 0);     // part follows cnt
    __syncthreads();
    for (int i = threadIdx.x * 4; i < n; i += ST * 4) {
      const float4 v4 = *reinterpret_cast<const float4*>(x + i);
      const float v[4] = {v4.x, v4.y, v4.z, v4.w};
      int b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) { b[j] = bin_of(v[j]); atomicAdd(&cnt[b[j]], 1u); }
      if (mass) {
        u64 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = weight(v[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (w[j]) {
            atomicAdd(&part[b[j]], (uint32_t)w[j] & 0x7fffu);
            atomicAdd(&part[NB + b[j]], (uint32_t)(w[j] >> 15) & 0x7fffu);
            atomicAdd(&part[2 * NB + b[j]], (uint32_t)(w[j] >> 30));
          }
      }
    }
    __syncthreads();
    // every CTA hands the bins out, each share to the CTA that adds it up; the sums go to the first CTA
    constexpr int share = NB / ranks;
    if (ranks > 1) {
      for (int b = threadIdx.x; b < NB; b += ST) {
        uint4* to = cl.map_shared_rank(inbox, b / share) + rank * share + b % share;
        *to = mass ? make_uint4(cnt[b], part[b], part[NB + b], part[2 * NB + b]) : make_uint4(cnt[b], 0, 0, 0);
      }
      cl.sync();
    }
    uint32_t* to_cnt = cl.map_shared_rank(ccnt, 0);
    u64* to_mass = cl.map_shared_rank(cmass, 0);
    for (int i = threadIdx.x; i < share; i += ST) {
      uint32_t k = 0;
      u64 w = 0;
      if (ranks == 1) {
        k = cnt[i];
        if (mass) w = part[i] + ((u64)part[NB + i] << 15) + ((u64)part[2 * NB + i] << 30);
      } else {
#pragma unroll
        for (int r = 0; r < ranks; ++r) {
          const uint4 v = inbox[r * share + i];
          k += v.x;
          w += v.y + ((u64)v.z << 15) + ((u64)v.w << 30);
        }
      }
      to_cnt[rank * share + i] = k;
      if (mass) to_mass[rank * share + i] = w;
    }
    cl.sync();
  }

  // Inclusive block sums of a and b.
  __device__ __forceinline__ void scan2(u64& a, u64& b) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    a = warp_scan(a);
    b = warp_scan(b);
    if (lane == 31) { sm->warp_a[warp] = a; sm->warp_b[warp] = b; }
    __syncthreads();
    u64 wa = lane < warp ? sm->warp_a[lane & (SW - 1)] : 0, wb = lane < warp ? sm->warp_b[lane & (SW - 1)] : 0;      // SW = 16 <= 32
    a += warp_sum(wa);
    b += warp_sum(wb);
    __syncthreads();
  }

  __device__ __forceinline__ void publish(int bin, int count, u64 target, u64 up_to) {      // by one thread
    cg::cluster_group cl = cg::this_cluster();
#pragma unroll
    for (int i = 0; i < ranks; ++i) {
      Shared* to = cl.map_shared_rank(sm, i);
      to->pick_bin = bin; to->pick_count = count; to->pick_target = target; to->pick_up_to = up_to;
    }
  }
  __device__ __forceinline__ void publish_pair(u64 pair) {
    cg::cluster_group cl = cg::this_cluster();
    for (int i = 0; i < ranks; ++i) cl.map_shared_rank(sm, i)->pick_pair = pair;
  }

  // The elements whose bin lies in [lo, hi] (at most LIST in all) go to the first CTA's list: each CTA gathers its own, then
  // takes room for them there with one remote addition to `counter`.
  __device__ void collect(int lo, int hi, int* counter) {
    cg::cluster_group cl = cg::this_cluster();
    if (threadIdx.x == 0) sm->list_n = 0;
    __syncthreads();
    for (int i = threadIdx.x * 4; i < n; i += ST * 4) {
      const float4 v4 = *reinterpret_cast<const float4*>(x + i);
      const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int b = bin_of(v[j]);
        if (b >= lo && b <= hi) {
          const int at = atomicAdd(&sm->list_n, 1);
          if (at < LIST) mine[at] = pair_key(key_of(v[j]), first + i + j);
        }
      }
    }
    __syncthreads();
    const int m = min(sm->list_n, LIST);
    if (m > 0) {                              // uniform over the CTA
      if (threadIdx.x == 0) sm->base = atomicAdd(cl.map_shared_rank(counter, 0), m);
      __syncthreads();
      u64* to = cl.map_shared_rank(list, 0) + sm->base;
      for (int i = threadIdx.x; i < m && sm->base + i < LIST; i += ST) to[i] = mine[i];
    }
    cl.sync();
  }

  __device__ __forceinline__ u64 block_sum(u64 v) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_sum(v);
    if (lane == 0) sm->warp_a[warp] = v;
    __syncthreads();
    const u64 all = warp_sum(lane < SW ? sm->warp_a[lane] : 0);
    __syncthreads();
    return all;
  }

  // First CTA, all m <= FEW candidates in the list: thresholds and draw, every element against every other.
  // `whole`: the mass that top_p is a share of, or 0: that of the top_k first.
  __device__ void finish_few(int m, u64 top_k, bool by_mass, float top_p, u64 whole, float u, int* token, float* logprob) {
    int q = 2;                                // threads of an element
    while (q < 16 && m * q * 2 <= ST) q *= 2;
    const int e = threadIdx.x / q, part_of = threadIdx.x & (q - 1);
    if (threadIdx.x < m) lweight[threadIdx.x] = weight(of_key((uint32_t)(list[threadIdx.x] >> 32)));
    __syncthreads();
    const u64 pair = e < m ? list[e] : 0, w = e < m ? lweight[e] : 0;
    u64 above = 0;                            // weight of what ranks before
    int before = 0;
#pragma unroll 4
    for (int j = part_of; j < m; j += q)
      if (list[j] > pair) { ++before; above += lweight[j]; }
    for (int d = 1; d < q; d <<= 1) {
      before += __shfl_xor_sync(~0u, before, d);
      above += __shfl_xor_sync(~0u, above, d);
    }
    const bool first_of = e < m && part_of == 0;
    bool keep = e < m && (u64)before < top_k;
    if (by_mass) {
      const u64 all = whole ? whole : block_sum(first_of && keep ? w : 0);
      bool more;
      u64 target = share_of(fmaxf(top_p, 0.f), all, &more);
      target += more;
      keep = keep && (above < target || before == 0);
    }
    keep = keep && w >= least;
    const u64 all = block_sum(first_of && keep ? w : 0);
    u64* kept_weight = lweight;
    __syncthreads();
    if (first_of) kept_weight[e] = keep ? w : 0;
    __syncthreads();
    bool more;
    u64 target = u < 1.f ? share_of(u, all, &more) : all;
    if (target >= all) target = all - 1;
    u64 run = 0;                              // weight up to and including this index: the low word orders downwards
#pragma unroll 4
    for (int j = part_of; j < m; j += q)
      if ((uint32_t)list[j] >= (uint32_t)pair) run += kept_weight[j];
    for (int d = 1; d < q; d <<= 1) run += __shfl_xor_sync(~0u, run, d);
    if (first_of && keep && run > target && run - w <= target) {
      *token = (int)~(uint32_t)pair;
      const float v = of_key((uint32_t)(pair >> 32));
      const double t = v == xmax ? 0.0 : ((double)v - (double)xmax) * c;
      if (logprob) *logprob = (float)((t - log2((double)all) + 44.0) * 0.6931471805599453);
    }
  }

  // First CTA, list of m elements: the one at which, in ranking order, the running count (or, by_mass, weight) reaches
  // `target` is handed to `chosen` with the running weight up to and including it.
  template <class G>
  __device__ void choose(int m, bool by_mass, bool weights, u64 target, G chosen) {
    if (weights) {
      for (int i = threadIdx.x; i < m; i += ST) lweight[i] = weight(of_key((uint32_t)(list[i] >> 32)));
      __syncthreads();
    }
    if (m <= ST / 2) {                        // every element against every other, several threads an element
      int q = 2;
      while (q < 16 && m * q * 2 <= ST) q *= 2;
      const int e = threadIdx.x / q;
      const u64 mine = e < m ? list[e] : ~0ull;
      u64 before = 0, mass = 0;
#pragma unroll 4
      for (int j = threadIdx.x & (q - 1); j < m; j += q) {
        const u64 other = list[j];
        before += other > mine;
        if (weights && other >= mine) mass += lweight[j];
      }
      for (int d = 1; d < q; d <<= 1) {
        before += __shfl_xor_sync(~0u, before, d);
        mass += __shfl_xor_sync(~0u, mass, d);
      }
      if (e < m && (threadIdx.x & (q - 1)) == 0) {
        const bool hit = by_mass ? mass >= target && mass - lweight[e] < target : before + 1 == target;
        if (hit) chosen(mine, mass);
      }
      __syncthreads();
      return;
    }
    int size = ST;                            // many: bitonic, descending, padded with zeros
    while (size < m) size *= 2;
    for (int i = m + threadIdx.x; i < size; i += ST) { list[i] = 0; lweight[i] = 0; }
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        for (int i = threadIdx.x; i < size / 2; i += ST) {
          const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
          const u64 a = list[lo], b = list[hi];
          if ((a < b) == ((lo & k) == 0)) {
            list[lo] = b; list[hi] = a;
            const u64 wa = lweight[lo];
            lweight[lo] = lweight[hi]; lweight[hi] = wa;
          }
        }
        __syncthreads();
      }
    const int each = size / ST, at = threadIdx.x * each;          // 1 or 2 elements a thread
    u64 w = 0, nothing = 0;
    if (weights) for (int i = 0; i < each; ++i) w += lweight[at + i];
    u64 run = w;
    scan2(run, nothing);
    run -= w;
    for (int i = 0; i < each; ++i) {
      const u64 wi = weights ? lweight[at + i] : 0;
      const bool hit = at + i < m && (by_mass ? run < target && target <= run + wi : (u64)(at + i) + 1 == target);
      run += wi;
      if (hit) chosen(list[at + i], run);
    }
    __syncthreads();
  }
};

static_assert(SW == 16 && LIST == 2 * ST && NB == 2 * ST && 2 * LIST * 8 <= NB * 16, "scan2, choose and the bins of a thread");

template <int DT>
__device__ __forceinline__ float load_logit(const void* p, int64_t i) {
  float x;
  if (DT == ES_DTYPE_F32) x = __ldg(reinterpret_cast<const float*>(p) + i);
  else if (DT == ES_DTYPE_F16) x = __half2float(reinterpret_cast<const __half*>(p)[i]);
  else x = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
  return isnan(x) ? -INFINITY : x + 0.f;      // -0 becomes +0: equal numbers have equal keys
}

__host__ __device__ constexpr size_t sample_smem(int slice) {
  return (size_t)slice * 4 + (size_t)(slice / CHUNK) * 8 + (size_t)NB * (16 + 16 + 8 + 4);
}

template <int DT, int ranks>
__global__ void __launch_bounds__(ST, 2) sample_kernel(const SampleParams p) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ Shared shared;
  cg::cluster_group cl = cg::this_cluster();
  cluster_arrive();                           // "this CTA runs": nobody writes into it before
  const int rank = (int)cl.block_rank(), row = blockIdx.x / ranks;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // the row's settings, wanted after the logits: their latencies pass together
  const float T = p.temperature ? p.temperature[row] : 1.f, tp = p.top_p ? p.top_p[row] : 1.f;
  const float mp = p.min_p ? fminf(fmaxf(p.min_p[row], 0.f), 1.f) : 0.f, u = fminf(fmaxf(p.u[row], 0.f), 1.f);
  const int k = p.top_k ? p.top_k[row] : 0;
  Row<ranks> R;
  R.x = reinterpret_cast<float*>(dyn);
  // [slice] logits | [4][NB] the CTA's histogram, later its own elements of a bin and the list's weights, or the sums of a
  // descent | [NB] uint4 inbox of the histograms, later the list | the cluster's weights and counts | chunk sums
  R.cnt = reinterpret_cast<uint32_t*>(dyn + (size_t)p.slice * 4);
  R.part = R.cnt + NB;
  R.mine = R.dhist = reinterpret_cast<u64*>(R.cnt);
  R.dcomb = R.dhist + 256;
  R.lweight = R.mine + LIST;
  R.inbox = reinterpret_cast<uint4*>(R.part + 3 * NB);
  R.list = reinterpret_cast<u64*>(R.inbox);
  R.cmass = reinterpret_cast<u64*>(R.inbox + NB);
  R.csum = R.cmass + NB;
  R.ccnt = reinterpret_cast<uint32_t*>(R.csum + p.slice / CHUNK);
  R.sm = &shared;
  R.rank = rank;
  R.first = rank * p.slice;
  const int real = max(0, min(p.V - R.first, p.slice));
  R.n = (real + CHUNK - 1) / CHUNK * CHUNK;

  // ---- the slice comes in; largest logit at the lowest index, smallest finite one ----
  u64 best = 0;
  float least = INFINITY;
  const int64_t row_at = (int64_t)row * p.row_stride + R.first;
  constexpr int FLIGHT = 16;                  // loads of a thread under way at a time
  for (int base = 0; base < R.n; base += ST * FLIGHT) {
    float v[FLIGHT];
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j) {
      const int i = base + j * ST + tid;
      v[j] = i < real ? load_logit<DT>(p.logits, row_at + i) : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j) {
      const int i = base + j * ST + tid;
      if (i < R.n) {
        R.x[i] = v[j];
        const u64 b = pair_key(key_of(v[j]), R.first + i);
        best = b > best ? b : best;
        if (v[j] > -INFINITY) least = fminf(least, v[j]);
      }
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const u64 o = __shfl_xor_sync(~0u, best, d);
    best = o > best ? o : best;
    least = fminf(least, __shfl_xor_sync(~0u, least, d));
  }
  if (lane == 0) { shared.warp_a[warp] = best; shared.warp_b[warp] = __float_as_uint(least); }
  __syncthreads();
  cluster_wait();
  if (warp == 0) {
    best = lane < SW ? shared.warp_a[lane] : 0;
    least = lane < SW ? __uint_as_float((uint32_t)shared.warp_b[lane]) : INFINITY;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      const u64 o = __shfl_xor_sync(~0u, best, d);
      best = o > best ? o : best;
      least = fminf(least, __shfl_xor_sync(~0u, least, d));
    }
    if (lane < ranks) {
      Shared* to = cl.map_shared_rank(&shared, lane);
      to->best[rank] = best;
      to->least[rank] = least;
    }
    if (lane == 0) { shared.few_n = 0; shared.pick_bin = 0; shared.pick_count = 0; shared.pick_target = 1; shared.pick_pair = 0; }
  }
  cl.sync();
  best = 0;
  least = INFINITY;
#pragma unroll
  for (int r = 0; r < ranks; ++r) {
    best = shared.best[r] > best ? shared.best[r] : best;
    least = fminf(least, shared.least[r]);
  }

  R.xmax = of_key((uint32_t)(best >> 32));
  const int top = (int)~(uint32_t)best;
  if (R.xmax == -INFINITY || !(T > 0.f)) {    // nothing to draw from, or no drawing
    if (rank == 0 && tid == 0) {
      p.tokens[row] = R.xmax == -INFINITY ? -1 : top;
      if (p.logprobs) p.logprobs[row] = R.xmax == -INFINITY ? -INFINITY : 0.f;
    }
    return;
  }
  R.c = 1.4426950408889634 / (double)T;
  R.cf = (float)R.c;
  R.keep = 0;
  {
    const u64 w = (u64)ceil((double)mp * UNIT);
    R.least = w < 1 ? 1 : w;
  }
  const bool by_count = k > 0 && k < p.V, by_mass = tp < 1.f;
  if (by_count || by_mass) {
    const float span = fminf(R.xmax - least, REACH / R.cf);
    R.bin_scale = span > 0.f ? fminf((NB - 1) / span, 1e37f) : 0.f;
    // weights are left out of the histogram where the count alone is likely to leave few candidates; if it does not, a
    // second one makes up for it
    const bool count_first = by_count && by_mass && k <= FEW;
    R.histogram(by_mass && !count_first);
    // first CTA: inclusive sums up to this thread's second bin (bins 2 tid and 2 tid + 1)
    u64 counts = 0, masses = 0, m0 = 0, m1 = 0;
    uint32_t c0 = 0, c1 = 0;
    auto pick_mass = [&]() {                  // first CTA: the bin in which the mass is reached, of the kept mass so far
      const u64 all = shared.all_mass;
      bool more;
      u64 target = share_of(fmaxf(tp, 0.f), all, &more);
      target += more;
      target = target < 1 ? 1 : target > all ? all : target;
      const u64 a = masses - m0 - m1, b = masses - m1;
      if (a < target && target <= b) R.publish(2 * tid, (int)c0, target - a, counts - c1);
      if (b < target && target <= masses) R.publish(2 * tid + 1, (int)c1, target - b, counts);
    };
    if (rank == 0) {
      c0 = R.ccnt[2 * tid]; c1 = R.ccnt[2 * tid + 1];
      counts = (u64)c0 + c1;
      if (by_mass && !count_first) { m0 = R.cmass[2 * tid]; m1 = R.cmass[2 * tid + 1]; masses = m0 + m1; }
      R.scan2(counts, masses);
      if (tid == ST - 1) shared.all_mass = masses;
      __syncthreads();
      if (by_count) {
        const u64 a = counts - c0 - c1, b = counts - c1;
        if (a < (u64)k && (u64)k <= b) { R.publish(2 * tid, (int)c0, k - a, b); shared.all_mass = masses - m0 - m1; }
        if (b < (u64)k && (u64)k <= counts) { R.publish(2 * tid + 1, (int)c1, k - b, counts); shared.all_mass = masses - m1; }
      } else {
        pick_mass();
      }
    }
    cl.sync();
    if (shared.pick_up_to <= FEW) {           // the other CTAs hand over their candidates and are done
      const int m = (int)shared.pick_up_to, last_bin = shared.pick_bin;
      R.collect(0, last_bin, &shared.few_n);
      if (rank == 0) R.finish_few(m, by_count ? (u64)k : ~0ull, by_mass, tp, by_count ? 0 : shared.all_mass, u, p.tokens + row, p.logprobs ? p.logprobs + row : nullptr);
      return;
    }
    if (count_first) {
      const int bin = shared.pick_bin;
      R.histogram(true);
      if (rank == 0) {
        m0 = R.cmass[2 * tid]; m1 = R.cmass[2 * tid + 1];
        masses = m0 + m1;
        u64 nothing = 0;
        R.scan2(masses, nothing);
        if (tid == bin / 2) shared.all_mass = masses - m1 - (bin & 1 ? 0 : m0);
        __syncthreads();
      }
    }
    int listed = -1;                          // the bin that the list holds
    if (by_count) {
      const u64 want = shared.pick_target;
      const int bin = shared.pick_bin, m = shared.pick_count;
      if (m <= LIST) {
        listed = bin;
        R.collect(bin, bin, &shared.few_n);
        if (rank == 0) {                      // the mass of the bin's kept elements joins that of the bins before
          R.choose(m, false, by_mass, want, [&](u64 pair, u64 mass) { R.publish_pair(pair); shared.all_mass += mass; });
          if (by_mass) pick_mass();
          if (tid == 0) shared.few_n = 0;
        }
        cl.sync();
        R.keep = shared.pick_pair;
      } else {                                // too many for the list: by the bits of their keys
        u64 above, here;
        const uint32_t key = R.descend([&](float v, int) { return (u64)(R.bin_of(v) == bin); }, want, &above, &here);
        int cut = INT_MAX;
        if (here > want - above) {
          auto tie = [&](float v, int) { return (u64)(key_of(v) == key); };
          R.sums(tie);
          cut = R.find(tie, want - above - 1);
        }
        R.keep = ((u64)key << 32) | (cut == INT_MAX ? 0u : (uint32_t)~cut);
        if (by_mass) {
          const u64 s = R.sums([&](float v, int i) { return R.bin_of(v) == bin && R.kept(v, i) ? R.weight(v) : 0ull; });
          if (rank == 0) {
            if (tid == 0) shared.all_mass += s;
            __syncthreads();
            pick_mass();
          }
          cl.sync();
        }
      }
    }
    if (by_mass) {
      const u64 target = shared.pick_target;
      const int bin = shared.pick_bin, m = shared.pick_count;
      if (m <= LIST) {
        if (listed != bin) R.collect(bin, bin, &shared.few_n);
        if (rank == 0) R.choose(m, true, true, target, [&](u64 pair, u64) { R.publish_pair(pair); });
        cl.sync();
        R.keep = shared.pick_pair > R.keep ? shared.pick_pair : R.keep;
      } else {
        u64 above, here;
        const uint32_t key = R.descend([&](float v, int) { return R.bin_of(v) == bin ? R.weight(v) : 0ull; }, target, &above, &here);
        const u64 w = R.weight(of_key(key));
        const u64 want = (target - above + w - 1) / w;            // of the here / w elements with this key
        int cut = INT_MAX;
        if (want < here / w) {
          auto tie = [&](float v, int) { return (u64)(key_of(v) == key); };
          R.sums(tie);
          cut = R.find(tie, want - 1);
        }
        const u64 pr = ((u64)key << 32) | (cut == INT_MAX ? 0u : (uint32_t)~cut);
        R.keep = pr > R.keep ? pr : R.keep;
      }
    }
  }
  auto last = [&](float v, int i) { const u64 w = R.kept(v, i) ? R.weight(v) : 0ull; return w >= R.least ? w : 0ull; };
  const u64 all = R.sums(last);
  if (warp > 0) return;                       // nothing is read from another CTA any more
  bool more;
  u64 target = u < 1.f ? share_of(u, all, &more) : all;
  if (target >= all) target = all - 1;
  const int token = R.find_here(last, target);
  if (token >= 0 && lane == 0) {
    const float v = R.x[token - R.first];
    const double t = v == R.xmax ? 0.0 : ((double)v - (double)R.xmax) * R.c;
    p.tokens[row] = token;
    if (p.logprobs) p.logprobs[row] = (float)((t - log2((double)all) + 44.0) * 0.6931471805599453);
  }
}

template <int DT, int ranks>
es_status_t launch_ranks(const SampleParams& p, int B, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  ES_CUDA_CHECK(allow_shared_memory(sample_kernel<DT, ranks>, (int)sample_smem(MAX_SLICE), &allowed));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(B * ranks));
  cfg.blockDim = dim3(ST);
  cfg.dynamicSmemBytes = sample_smem(p.slice);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ranks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ES_CUDA_CHECK(cudaLaunchKernelEx(&cfg, sample_kernel<DT, ranks>, p));
  return ES_OK;
}

template <int DT>
es_status_t launch_sample(const SampleParams& p, int B, int ranks, cudaStream_t s) {
  switch (ranks) {
    case 1: return launch_ranks<DT, 1>(p, B, s);
    case 2: return launch_ranks<DT, 2>(p, B, s);
    case 4: return launch_ranks<DT, 4>(p, B, s);
    default: return launch_ranks<DT, 8>(p, B, s);
  }
}

}  // namespace
}  // namespace es

extern "C" {

es_status_t es_op_sample(const void* logits, int32_t dtype, int64_t row_stride, const float* u, const float* temperature,
                         const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens, float* logprobs,
                         int32_t B, int32_t V, void* stream) {
  using namespace es;
  if (!logits || !u || !tokens) return fail(ES_ERR_INVALID_ARG, "null argument");
  if (B <= 0 || V <= 0) return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (dtype != ES_DTYPE_F32 && dtype != ES_DTYPE_F16 && dtype != ES_DTYPE_BF16) return fail(ES_ERR_INVALID_ARG, "logits must be fp32, fp16 or bf16");
  if (row_stride < V) return fail(ES_ERR_INVALID_ARG, "row_stride is smaller than V");
  if (V > MAX_V) return fail(ES_ERR_RANGE, "V = %d exceeds %d", V, MAX_V);
  if (B > (1 << 24)) return fail(ES_ERR_RANGE, "too many rows");
  // slices of at most 16384 elements (two CTAs share an SM then: one works while the other's logits arrive), and smaller
  // ones while the machine has room for more CTAs
  int ranks = 1;
  while (ranks < MAX_CLUSTER && (V > 16384LL * ranks || ((long long)B * ranks < sm_count() && V > 2048 * ranks))) ranks *= 2;
  const int slice = ((V + ranks - 1) / ranks + CHUNK - 1) / CHUNK * CHUNK;
  SampleParams p{logits, row_stride, u, temperature, top_p, min_p, top_k, tokens, logprobs, V, slice};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == ES_DTYPE_F32) return launch_sample<ES_DTYPE_F32>(p, B, ranks, s);
  if (dtype == ES_DTYPE_F16) return launch_sample<ES_DTYPE_F16>(p, B, ranks, s);
  return launch_sample<ES_DTYPE_BF16>(p, B, ranks, s);
}

}  // extern "C"
