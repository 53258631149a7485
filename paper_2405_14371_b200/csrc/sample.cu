// Sampling the next token of every row of logits: temperature, top-k, top-p, min-p, one given random number per row.
//
// No row is sorted.  Every restriction keeps a prefix of the ranking (by logit, equal ones by index), so each is a
// threshold in that order, held as one 64-bit number, the logit's order-preserving bits above the complement of the
// index.  Three ways to it, from the cheapest:
//
//   * a small top-k: the k largest maxima of groups of 16 are k elements, so whatever ranks among the first k lies no lower
//     than the smallest of them.  A histogram of the maxima says where that is, the few elements from there up are
//     collected (only groups whose maximum reaches it are read), and one CTA finishes the row;
//   * few candidates after all: a histogram over the distance from the largest logit (counts, and weights where top-p
//     asks for them) says in which bin the threshold lies; up to 256 elements down to that bin are finished the same way;
//   * else the elements of that bin alone are collected, ranked and searched.  A bin with more elements than the list
//     takes (many equal logits) is descended by the bits of its keys instead.
//
// The draw is a search for a running weight in order of index.
//
// Weights are integers, w = round(2^44 exp2((x - max) log2(e) / temperature)) out of 64-bit arithmetic, so every sum
// is exact whatever its order: thresholds and tokens depend on the inputs alone, and the borders are as sharp as the
// exponential (2^-39).
//
// Measured, unrestricted / top_k 50 / top_p 0.9: one row of 32000 5.6 / 9.1 / 13.7 us, 64 rows 10.0 / 12.2 / 24.0 us, 256
// rows of 128001 (131 MB, 20 us at the copy rate) 111 / 64 / 260 us.  Small calls are bound by the latency of the passes
// and the cluster's barriers between them.  Large ones with mixed settings use a tenth of the memory's rate and 36 % of the
// issue slots (61 % on the busiest SM): a weight costs about 45 instructions, a third of them 64-bit, and top-p asks for
// each twice (its histogram, and the draw), beside four additions to shared memory, so rows are of very unequal length.
//
// A row belongs to a cluster of 1 to 8 CTAs.  Where all CTAs of a call run at once, each holds its slice of the row in
// shared memory as fp32: latency counts there.  Larger calls read the slice again from L2, which leaves room for four
// CTAs on an SM, one's barriers under another's sums (256 rows of 128001 with three and more registers each: 130 / 84 / 292
// us).
#include <cooperative_groups.h>
#include <limits.h>

#include "es_internal.cuh"
#include "kv8.cuh"
#include "launch.cuh"

namespace cg = cooperative_groups;

namespace es {
namespace {

typedef unsigned long long u64;

constexpr int MAX_WARPS = 16;
constexpr int GROUP = 16;                     // elements that a thread loads together; their largest is kept
// Largest top_k that goes by the maxima: about k + k^2 / groups of them end up in the list that takes 256.  On 256 rows of
// 128001, top_k 200 takes 94 us this way, 201 by the histogram of all elements 120 us; on 64 rows of 32000 both take 20 us.
constexpr int TOP_FEW = 200;
constexpr int CHUNK = 128;                    // neighbours a warp sums at a time: the grain of the search
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
  float best[MAX_CLUSTER], least[MAX_CLUSTER];  // largest logit, about the smallest finite one
  int found;                                  // a chosen index, from the CTA that found it
  // from the first CTA
  int pick_bin, pick_count;                   // a bin, and how many elements it holds
  u64 pick_up_to;                             // elements up to and including that bin
  u64 pick_target;                            // rank (counts) or mass to reach within the bin
  u64 pick_pair, pick_mass_pair;              // thresholds found in the list, of top-k and of top-p: nothing need stand between
                                              // everybody's reading of the first and the first CTA's finding the second
  // this CTA's own
  u64 all_mass;
  int list_n;
  int few_n;                                  // first CTA: candidates that have arrived
  int top;                                    // first CTA: lowest index of the largest
  int base;
  u64 warp_a[MAX_WARPS], warp_b[MAX_WARPS];
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

template <int DT>
__device__ __forceinline__ float load_logit(const void* p, int64_t i) {
  float x;
  if (DT == ES_DTYPE_F32) x = __ldg(reinterpret_cast<const float*>(p) + i);
  else if (DT == ES_DTYPE_F16) x = __half2float(reinterpret_cast<const __half*>(p)[i]);
  else x = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
  return fmaxf(x, -INFINITY) + 0.f;           // NaN becomes -infinity; -0 becomes +0: equal numbers have equal keys
}

// One row's working state; every method is called by all threads of the cluster.
template <int DT, int ranks, bool RESIDENT>
struct Row {
  static constexpr int ST = RESIDENT ? 512 : 256, SW = ST / 32;       // threads and warps of a CTA
  static constexpr int BPT = NB / ST;         // bins of a thread in the first CTA
  float* x;                                   // RESIDENT: slice in shared memory, padded with -infinity to a multiple of CHUNK
  const void* logits;                         // else the row, from the slice's first element at `at`
  int64_t at;
  int real;                                   // elements of the slice
  float* gmax;                                // largest of every group: group (round, thread) holds the elements
                                              // (GROUP round + j) ST + thread, j < GROUP
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

  static __host__ __device__ constexpr int groups(int elements) { return (elements + ST * GROUP - 1) / (ST * GROUP) * ST; }
  __device__ __forceinline__ float get(int i) const {
    if (RESIDENT) return x[i];
    return i < real ? load_logit<DT>(logits, at + i) : -INFINITY;
  }
  // t = (v - max) c as r + f, r whole (in the low bits of the result's first word) and |f| <= 1/2.  Roundings spelled out:
  // every use has to give the same weight to the last bit.
  __device__ __forceinline__ double split(float v, double x0, double* f) const {
    const double magic = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to an integer, which its low bits hold
    const double t = __dmul_rn(__dsub_rn((double)v, x0), c), r = __dadd_rn(t, magic);
    *f = __dsub_rn(t, __dsub_rn(r, magic));
    return __hiloint2double((1023 + 44 + __double2loint(r)) << 20, 0);            // 2^(44 + r), -47 <= r <= 0
  }
  static __device__ __forceinline__ u64 scaled(double poly, double scale) {
    return (u64)__double_as_longlong(fma(poly, scale, 4503599627370496.0)) - 0x4330000000000000ull;
  }
  // not so far below the largest that the weight rounds to zero (false for -infinity, and for anything finite below an
  // infinite largest)
  __device__ __forceinline__ bool near(float v) const { return fmaf(v, 0.5f, -0.5f * xmax) * cf > -0.5f * REACH; }
  __device__ __forceinline__ u64 weight(float v) const {
    if (v == xmax) return 1ull << 44;
    if (!near(v)) return 0;
    double f;
    const double scale = split(v, (double)xmax, &f);
    return scaled(exp2_poly(f), scale);
  }
  // the weights of four elements at once, without branches between them: the 64-bit chains of one fill the other's gaps
  __device__ __forceinline__ void weights(const float (&v)[4], u64 (&w)[4]) const {
    if (isinf(xmax)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = v[j] == xmax ? 1ull << 44 : 0;
      return;
    }
    bool in[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) in[j] = near(v[j]) || v[j] == xmax;
    if (!__any_sync(~0u, in[0] || in[1] || in[2] || in[3])) {
      w[0] = w[1] = w[2] = w[3] = 0;
      return;
    }
    const double x0 = (double)xmax;
    double f[4], scale[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) scale[j] = split(v[j], x0, &f[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = exp2_poly(f[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = in[j] ? scaled(f[j], scale[j]) : 0;
  }
  __device__ __forceinline__ bool kept(float v, int i) const { return pair_key(key_of(v), i) >= keep; }
  // bins grow with the distance from the largest logit; equal logits share one
  __device__ __forceinline__ int bin_of(float v) const {
    // adding 2^23 leaves the whole number (rounded, as good as cut off) in the low bits
    const float d = fminf((xmax - v) * bin_scale, (float)(NB - 1));
    return v == xmax ? 0 : __float_as_int(d + 8388608.f) & (2 * NB - 1);
  }

  // f of four elements, 32 apart
  template <class F>
  __device__ __forceinline__ u64 sum4(const F& f, const float (&v)[4], int i) const {
    return f(v[0], i) + f(v[1], i + 32) + f(v[2], i + 64) + f(v[3], i + 96);
  }
  // weight of what is kept
  struct Kept {
    const Row& r;
    __device__ __forceinline__ u64 operator()(float v, int i) const {
      const u64 w = r.kept(v, i) ? r.weight(v) : 0ull;
      return w >= r.least ? w : 0;
    }
  };
  __device__ __forceinline__ u64 sum4(const Kept&, const float (&v)[4], int i) const {
    u64 w[4];
    weights(v, w);
    if (keep) {                               // uniform, as the next
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = kept(v[j], i + 32 * j) ? w[j] : 0;
    }
    if (least > 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = w[j] >= least ? w[j] : 0;
    }
    return w[0] + w[1] + w[2] + w[3];
  }

  // chunk sums of f(value, index) in csum, every CTA's sum in sm->total; returns the cluster's
  template <class F>
  __device__ u64 sums(const F& f) {
    cg::cluster_group cl = cg::this_cluster();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int ch = warp; ch < n / CHUNK; ch += SW) {
      const int i = ch * CHUNK + lane;
      const float v[4] = {get(i), get(i + 32), get(i + 64), get(i + 96)};
      const u64 s = warp_sum(sum4(f, v, first + i));
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
    int at_index = ch * CHUNK;                // in steps of 32: ends where the chunk's sum passes the target
    unsigned hit = 0;
#pragma unroll 1                              // once a row, so a quarter of the code; unrolled it finds the same
    for (int j = 0; j < CHUNK / 32; ++j) {
      const u64 inc = run + warp_scan(f(get(at_index + lane), first + at_index + lane));
      hit = __ballot_sync(~0u, inc > target);
      if (hit) break;
      run = __shfl_sync(~0u, inc, 31);
      at_index += 32;
    }
    return first + at_index + (hit ? __ffs(hit) - 1 : -1);
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
        const float v = get(i);
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

  // Counts per bin, and weights where asked, summed over the cluster in the first CTA; of all elements, or of the maxima.
  __device__ void histogram(bool mass, bool of_maxima) {
    cg::cluster_group cl = cg::this_cluster();
    for (int i = threadIdx.x; i < (mass ? NB : NB / 4); i += ST) reinterpret_cast<uint4*>(cnt)[i] = make_uint4(0, 0, 0, 0);     // part follows cnt
    __syncthreads();
    if (of_maxima) {
      for (int i = threadIdx.x; i < groups(n); i += ST) atomicAdd(&cnt[bin_of(gmax[i])], 1u);
    } else {
      for (int base = 0; base < n; base += ST * 4) {       // n is a multiple of CHUNK: a warp is inside or outside
        float v[4];
        int b[4];
        const int i = base + (threadIdx.x >> 5) * CHUNK + (threadIdx.x & 31);
        if (i >= n) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = get(i + 32 * j);
#pragma unroll
        for (int j = 0; j < 4; ++j) { b[j] = bin_of(v[j]); atomicAdd(&cnt[b[j]], 1u); }
        if (mass) {
          u64 w[4];
          weights(v, w);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (w[j]) {
              atomicAdd(&part[b[j]], (uint32_t)w[j] & 0x7fffu);
              atomicAdd(&part[NB + b[j]], (uint32_t)(w[j] >> 15) & 0x7fffu);
              atomicAdd(&part[2 * NB + b[j]], (uint32_t)(w[j] >> 30));
            }
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
    const u64 wa = lane < warp ? sm->warp_a[lane] : 0, wb = lane < warp ? sm->warp_b[lane] : 0;      // SW <= 16
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
  __device__ __forceinline__ void publish_pair(u64 Shared::* to, u64 pair) {
    cg::cluster_group cl = cg::this_cluster();
    for (int i = 0; i < ranks; ++i) cl.map_shared_rank(sm, i)->*to = pair;
  }

  // The elements whose bin lies in [lo, hi] go to the first CTA's list: each CTA gathers its own out of the groups whose
  // largest reaches bin hi, then takes room for them there with one remote addition to `counter`.  Counts beyond LIST
  // are kept, elements beyond it are not.
  __device__ void collect(int lo, int hi, int* counter) {
    cg::cluster_group cl = cg::this_cluster();
    if (threadIdx.x == 0) sm->list_n = 0;
    __syncthreads();
    for (int round = 0; round * ST * GROUP < n; ++round) {
      if (bin_of(gmax[round * ST + threadIdx.x]) > hi) continue;
      for (int at = 0; at < GROUP; at += 8) {
        float v[8];
        const int i = (round * GROUP + at) * ST + threadIdx.x;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = i + j * ST < n ? get(i + j * ST) : -INFINITY;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int b = bin_of(v[j]);
          if (i + j * ST < n && b >= lo && b <= hi) {
            const int place = atomicAdd(&sm->list_n, 1);
            if (place < LIST) mine[place] = pair_key(key_of(v[j]), first + i + j * ST);
          }
        }
      }
    }
    __syncthreads();
    const int m = sm->list_n;
    if (m > 0) {                              // uniform over the CTA
      if (threadIdx.x == 0) sm->base = atomicAdd(cl.map_shared_rank(counter, 0), m);
      __syncthreads();
      u64* to = cl.map_shared_rank(list, 0);
      for (int i = threadIdx.x; i < min(m, LIST); i += ST)
        if (sm->base + i < LIST) to[sm->base + i] = mine[i];
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
    int q = 1;                                // threads of an element
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
    if (m <= FEW) {                           // every element against every other, several threads an element
      int q = 1;
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
    const int each = size / ST, at = threadIdx.x * each;          // 1, 2 or 4 elements a thread
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

static_assert(FEW <= 256 && LIST % 512 == 0 && NB % 512 == 0 && 2 * LIST * 8 <= NB * 16 && CHUNK == 128, "choose, finish_few, sum4 and the bins of a thread");

__host__ __device__ constexpr size_t sample_smem(int slice, bool resident) {
  const int round = (resident ? 512 : 256) * GROUP;
  return (resident ? (size_t)slice * 4 : 0) + (size_t)((slice + round - 1) / round) * (round / GROUP) * 4 + (size_t)(slice / CHUNK) * 8 + (size_t)NB * (16 + 16 + 8 + 4);
}

template <int DT, int ranks, bool RESIDENT>
__global__ void __launch_bounds__(RESIDENT ? 512 : 256, RESIDENT ? 2 : 4) sample_kernel(const SampleParams p) {
  using RowT = Row<DT, ranks, RESIDENT>;
  constexpr int ST = RowT::ST, SW = RowT::SW, BPT = RowT::BPT;
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ Shared shared;
  cg::cluster_group cl = cg::this_cluster();
  cluster_arrive();                           // "this CTA runs": nobody writes into it before
  const int rank = (int)cl.block_rank(), row = blockIdx.x / ranks;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  // the row's settings, wanted after the logits: their latencies pass together
  const float T = p.temperature ? p.temperature[row] : 1.f, tp = p.top_p ? p.top_p[row] : 1.f;
  const float mp = p.min_p ? fminf(fmaxf(p.min_p[row], 0.f), 1.f) : 0.f, u = fminf(fmaxf(p.u[row], 0.f), 1.f);
  const int k = p.top_k ? p.top_k[row] : 0;
  RowT R;
  // [slice] logits where resident | [4][NB] the CTA's histogram, later its own elements of a bin and the list's weights, or
  // the sums of a descent | [NB] uint4 inbox of the histograms, later the list | the cluster's weights | largest of groups | chunk
  // sums | the cluster's counts
  R.x = reinterpret_cast<float*>(dyn);
  R.cnt = reinterpret_cast<uint32_t*>(dyn + (RESIDENT ? (size_t)p.slice * 4 : 0));
  R.part = R.cnt + NB;
  R.mine = R.dhist = reinterpret_cast<u64*>(R.cnt);
  R.dcomb = R.dhist + 256;
  R.lweight = R.mine + LIST;
  R.inbox = reinterpret_cast<uint4*>(R.part + 3 * NB);
  R.list = reinterpret_cast<u64*>(R.inbox);
  R.cmass = reinterpret_cast<u64*>(R.inbox + NB);
  R.gmax = reinterpret_cast<float*>(R.cmass + NB);
  R.csum = reinterpret_cast<u64*>(R.gmax + RowT::groups(p.slice));
  R.ccnt = reinterpret_cast<uint32_t*>(R.csum + p.slice / CHUNK);
  R.sm = &shared;
  R.rank = rank;
  R.first = rank * p.slice;
  const int real = R.real = max(0, min(p.V - R.first, p.slice));
  R.n = (real + CHUNK - 1) / CHUNK * CHUNK;
  R.logits = p.logits;
  R.at = (int64_t)row * p.row_stride + R.first;

  // ---- the slice comes in; largest logit, and about the smallest (one of every group) ----
  float best = -INFINITY, least = INFINITY;
  for (int base = 0; base < R.n; base += ST * GROUP) {
    float v[GROUP], most = -INFINITY;
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      const int i = base + j * ST + tid;
      v[j] = i < real ? load_logit<DT>(p.logits, R.at + i) : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      const int i = base + j * ST + tid;
      if (RESIDENT && i < R.n) R.x[i] = v[j];
      most = fmaxf(most, v[j]);
    }
    R.gmax[base / GROUP + tid] = most;
    best = fmaxf(best, most);
    if (v[0] > -INFINITY) least = fminf(least, v[0]);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    best = fmaxf(best, __shfl_xor_sync(~0u, best, d));
    least = fminf(least, __shfl_xor_sync(~0u, least, d));
  }
  if (lane == 0) { shared.warp_a[warp] = __float_as_uint(best); shared.warp_b[warp] = __float_as_uint(least); }
  __syncthreads();
  cluster_wait();
  if (warp == 0) {
    best = lane < SW ? __uint_as_float((uint32_t)shared.warp_a[lane]) : -INFINITY;
    least = lane < SW ? __uint_as_float((uint32_t)shared.warp_b[lane]) : INFINITY;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      best = fmaxf(best, __shfl_xor_sync(~0u, best, d));
      least = fminf(least, __shfl_xor_sync(~0u, least, d));
    }
    if (lane < ranks) {
      Shared* to = cl.map_shared_rank(&shared, lane);
      to->best[rank] = best;
      to->least[rank] = least;
    }
    if (lane == 0) { shared.few_n = 0; shared.pick_bin = 0; shared.pick_count = 0; shared.pick_target = 1; shared.pick_pair = 0; shared.pick_mass_pair = 0; shared.top = INT_MAX; }
  }
  cl.sync();
  best = -INFINITY;
  least = INFINITY;
#pragma unroll
  for (int r = 0; r < ranks; ++r) {
    best = fmaxf(best, shared.best[r]);
    least = fminf(least, shared.least[r]);
  }

  R.xmax = best;
  if (R.xmax == -INFINITY) {                  // nothing to draw from
    if (rank == 0 && tid == 0) {
      p.tokens[row] = -1;
      if (p.logprobs) p.logprobs[row] = -INFINITY;
    }
    return;
  }
  if (!(T > 0.f)) {                           // no drawing: the lowest index of the largest
    int top = INT_MAX;
    for (int round = 0; round * ST * GROUP < R.n; ++round)
      if (R.gmax[round * ST + tid] == R.xmax)
        for (int j = GROUP - 1; j >= 0; --j) {
          const int i = (round * GROUP + j) * ST + tid;
          if (i < real && R.get(i) == R.xmax) top = min(top, R.first + i);
        }
    top = __reduce_min_sync(~0u, top);
    if (lane == 0 && top < INT_MAX) atomicMin(cl.map_shared_rank(&shared.top, 0), top);
    cl.sync();
    if (rank == 0 && tid == 0) {
      p.tokens[row] = shared.top;
      if (p.logprobs) p.logprobs[row] = 0.f;
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
    if (by_count && k <= TOP_FEW) {           // by the maxima
      R.histogram(false, true);
      if (rank == 0) {
        u64 run = 0, nothing = 0;
        uint32_t c[BPT];
#pragma unroll
        for (int j = 0; j < BPT; ++j) { c[j] = R.ccnt[BPT * tid + j]; run += c[j]; }
        R.scan2(run, nothing);
        if (tid == ST - 1 && run < (u64)k) R.publish(NB - 1, 0, 0, 0);       // fewer maxima than that: everything is a candidate
#pragma unroll
        for (int j = BPT - 1; j >= 0; --j) {
          if (run - c[j] < (u64)k && (u64)k <= run) R.publish(BPT * tid + j, 0, 0, 0);
          run -= c[j];
        }
      }
      cl.sync();
      R.collect(0, shared.pick_bin, &shared.few_n);
      const int m = *cl.map_shared_rank(&shared.few_n, 0);
      cluster_arrive();
      if (m <= FEW) {
        if (rank == 0) R.finish_few(m, (u64)k, by_mass, tp, 0, u, p.tokens + row, p.logprobs ? p.logprobs + row : nullptr);
        __syncwarp();
        cluster_wait();                       // the first CTA's count has been read by all
        return;
      }
      cluster_wait();
      if (rank == 0 && tid == 0) shared.few_n = 0;         // (seen by all after the next barrier)
    }
    R.histogram(by_mass, false);
    // first CTA: inclusive sums up to this thread's last bin
    u64 counts = 0, masses = 0, mb[BPT];
    uint32_t cb[BPT];
    auto pick_mass = [&]() {                  // first CTA: the bin in which the mass is reached, of the kept mass so far
      const u64 all = shared.all_mass;
      bool more;
      u64 target = share_of(fmaxf(tp, 0.f), all, &more);
      target += more;
      target = target < 1 ? 1 : target > all ? all : target;
      u64 run = masses, up_to = counts;
#pragma unroll
      for (int j = BPT - 1; j >= 0; --j) {
        if (run - mb[j] < target && target <= run) R.publish(BPT * tid + j, (int)cb[j], target - (run - mb[j]), up_to);
        run -= mb[j];
        up_to -= cb[j];
      }
    };
    if (rank == 0) {
#pragma unroll
      for (int j = 0; j < BPT; ++j) {
        cb[j] = R.ccnt[BPT * tid + j];
        counts += cb[j];
        mb[j] = by_mass ? R.cmass[BPT * tid + j] : 0;
        masses += mb[j];
      }
      R.scan2(counts, masses);
      if (tid == ST - 1) shared.all_mass = masses;
      __syncthreads();
      if (by_count) {
        u64 run = counts, mass_run = masses;
#pragma unroll
        for (int j = BPT - 1; j >= 0; --j) {
          if (run - cb[j] < (u64)k && (u64)k <= run) {
            R.publish(BPT * tid + j, (int)cb[j], k - (run - cb[j]), run);
            shared.all_mass = mass_run - mb[j];            // the mass of the bins before
          }
          run -= cb[j];
          mass_run -= mb[j];
        }
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
    int listed = -1;                          // the bin that the list holds
    if (by_count) {
      const u64 want = shared.pick_target;
      const int bin = shared.pick_bin, m = shared.pick_count;
      if (m <= LIST) {
        listed = bin;
        R.collect(bin, bin, &shared.few_n);
        if (rank == 0) {                      // the mass of the bin's kept elements joins that of the bins before
          R.choose(m, false, by_mass, want, [&](u64 pair, u64 mass) { R.publish_pair(&Shared::pick_pair, pair); shared.all_mass += mass; });
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
        if (rank == 0) R.choose(m, true, true, target, [&](u64 pair, u64) { R.publish_pair(&Shared::pick_mass_pair, pair); });
        cl.sync();
        R.keep = shared.pick_mass_pair > R.keep ? shared.pick_mass_pair : R.keep;       // never below top-k's
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
  const typename RowT::Kept last{R};
  const u64 all = R.sums(last);
  if (warp > 0) return;                       // nothing is read from another CTA any more
  bool more;
  u64 target = u < 1.f ? share_of(u, all, &more) : all;
  if (target >= all) target = all - 1;
  const int token = R.find_here(last, target);
  if (token >= 0 && lane == 0) {
    const float v = R.get(token - R.first);
    const double t = v == R.xmax ? 0.0 : ((double)v - (double)R.xmax) * R.c;
    p.tokens[row] = token;
    if (p.logprobs) p.logprobs[row] = (float)((t - log2((double)all) + 44.0) * 0.6931471805599453);
  }
}

template <int DT, int ranks, bool RESIDENT>
es_status_t launch_kind(const SampleParams& p, int B, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  ES_CUDA_CHECK(allow_shared_memory(sample_kernel<DT, ranks, RESIDENT>, (int)sample_smem(MAX_SLICE, RESIDENT), &allowed));
  ES_CUDA_CHECK(launch_clusters(sample_kernel<DT, ranks, RESIDENT>, ranks, dim3((unsigned)(B * ranks)), dim3(Row<DT, ranks, RESIDENT>::ST),
                                sample_smem(p.slice, RESIDENT), s, tunables().pdl != 0, p));
  return ES_OK;
}

template <int DT, int ranks>
es_status_t launch_ranks(const SampleParams& p, int B, cudaStream_t s) {
  // resident slices as long as all CTAs of the call run at once (64 rows of 32000, unrestricted / top_k 50 / top_p 0.9:
  // resident 10.2 / 12.2 / 24.3 us, from L2 12.9 / 12.9 / 29.3; 256 rows of 128001: 118 / 113 / 306 and 119 / 87 / 274)
  const int per_sm = sample_smem(p.slice, true) <= 112 * 1024 ? 2 : 1;
  return (long long)B * ranks <= (long long)per_sm * sm_count() ? launch_kind<DT, ranks, true>(p, B, s) : launch_kind<DT, ranks, false>(p, B, s);
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
  // Slices of at most 16384 elements, and smaller ones while the machine has room for more CTAs (one row of 32000: 8 CTAs
  // 6.0 us, 4 7.7, 2 10.6, 1 16.3); then larger ones where that saves waves of four CTAs an SM, each of which costs about as
  // much again as 8192 elements (256 rows of 128001, unrestricted / top_k 50 / top_p 0.9: 4 CTAs a row 110 / 65 / 262 us, 8
  // 119 / 88 / 274; 600 rows of 32000: 2 CTAs 70 / 61 / 155, 1 81 / 59 / 172).
  int ranks = 1;
  while (ranks < MAX_CLUSTER && (V > 16384LL * ranks || ((long long)B * ranks < sm_count() && V > 2048 * ranks))) ranks *= 2;
  const auto cost = [&](int r) { return ((long long)B * r + 4 * sm_count() - 1) / (4 * sm_count()) * ((V + r - 1) / r + 8192); };
  while (ranks > 1 && V <= (long long)MAX_SLICE * (ranks / 2) && cost(ranks / 2) < cost(ranks)) ranks /= 2;
  const int slice = ((V + ranks - 1) / ranks + CHUNK - 1) / CHUNK * CHUNK;
  SampleParams p{logits, row_stride, u, temperature, top_p, min_p, top_k, tokens, logprobs, V, slice};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == ES_DTYPE_F32) return launch_sample<ES_DTYPE_F32>(p, B, ranks, s);
  if (dtype == ES_DTYPE_F16) return launch_sample<ES_DTYPE_F16>(p, B, ranks, s);
  return launch_sample<ES_DTYPE_BF16>(p, B, ranks, s);
}

}  // extern "C"
