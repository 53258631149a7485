// Sampling the next token of every row of logits: temperature, top-k, top-p, min-p, one given random number per row.
//
// Nothing is sorted.  All three restrictions keep a prefix of the ranking, so each is a threshold (a key and, among equal
// keys, a last index), found by descending the bits of the keys with sums over the elements of a bin: counts for top-k,
// weights for top-p.  The draw is a search for a running weight in order of index.
//
// Weights are integers, w = round(2^44 exp2((x - max) log2(e) / temperature)) out of a 64-bit exponential, so every sum
// is exact whatever its order: thresholds and tokens depend on the inputs alone, and the borders are as sharp as 2^-45
// of the largest weight.
//
// A row belongs to one CTA or to a cluster of 2, 4 or 8, each holding a slice of the row in shared memory as fp32: the
// logits are read from HBM once, whatever the number of passes.
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
constexpr int MAX_SLICE = 48 * 1024;          // elements of a slice: 192 KB and its chunk sums fit the 227 KB of a CTA
constexpr int MAX_V = 262144;                 // 2^18 weights of 2^44 stay below 2^63

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
  u64 hist[256];
  u64 comb[256];
  u64 total;                                  // this CTA's, read by the cluster
  u64 best;                                   // this CTA's largest (key, index)
  u64 warp_u64[SW];
  int found;                                  // a chosen index, written into every CTA by the one that finds it
  int pick_bin;
  u64 pick_above, pick_here;
};

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

// One row's working state; every method is called by all threads of the cluster.
struct Row {
  float* x;                                   // slice in shared memory, padded with -infinity to a multiple of CHUNK
  u64* csum;
  Shared* sm;
  int n, first, ranks, rank;                  // padded elements, global index of the first, CTAs
  float xmax;
  double c;                                   // log2(e) / temperature
  uint32_t key;                               // kept: keys above `key`, and those equal to it up to index `cut`
  int cut;
  u64 least;                                  // ... whose weight is at least this

  __device__ __forceinline__ u64 weight(float v) const {
    if (v == xmax) return 1ull << 44;
    const double t = ((double)v - (double)xmax) * c;
    if (!(t > -46.0)) return 0;               // also -infinity, and anything finite below an infinite maximum
    return __double2ull_rn(exp2(t) * 17592186044416.0);
  }
  __device__ __forceinline__ bool kept(uint32_t k, int i) const { return k > key || (k == key && i <= cut); }

  // chunk sums of f(value, index) in csum, the CTA's in sm->total; returns the cluster's
  template <class F>
  __device__ u64 sums(F f) {
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
      if (lane == 0) sm->total = s;
    }
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
    u64 all = 0;
    for (int r = 0; r < ranks; ++r) all += cl.map_shared_rank(sm, r)->total;
    return all;
  }

  // after sums(f): the first index at which the running sum of f exceeds `target` (< the cluster's sum), in every CTA
  template <class F>
  __device__ int find(F f, u64 target) {
    cg::cluster_group cl = cg::this_cluster();
    const int lane = threadIdx.x & 31;
    if (threadIdx.x < 32) {
      u64 before = 0;
      for (int r = 0; r < rank; ++r) before += cl.map_shared_rank(sm, r)->total;
      if (before <= target && target < before + sm->total) {
        u64 run = before;
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
        const int got = __shfl_sync(~0u, at, __ffs(hit) - 1);
        if (lane < ranks) cl.map_shared_rank(sm, lane)->found = got;
      }
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
      for (int i = threadIdx.x; i < 256; i += ST) sm->hist[i] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += ST) {
        const float v = x[i];
        const uint32_t k = key_of(v);
        if (shift == 24 || (k >> (shift + 8)) == prefix) {
          const u64 w = f(v, first + i);
          if (w) atomicAdd(&sm->hist[(k >> shift) & 255], w);
        }
      }
      cl.sync();
      for (int i = threadIdx.x; i < 256; i += ST) {
        u64 s = 0;
        for (int r = 0; r < ranks; ++r) s += cl.map_shared_rank(sm, r)->hist[i];
        sm->comb[i] = s;
      }
      cl.sync();
      if (threadIdx.x < 32) {                 // lane l holds bins 255 - 8 l down to 248 - 8 l
        const int lane = threadIdx.x;
        u64 v[8], s = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) { v[j] = sm->comb[255 - 8 * lane - j]; s += v[j]; }
        const u64 inc = run + warp_scan(s);
        const unsigned hit = __ballot_sync(~0u, inc >= target);
        if (hit && lane == __ffs(hit) - 1) {
          u64 r = inc - s;
          int j = 0;
          while (j < 7 && r + v[j] < target) r += v[j++];
          sm->pick_bin = 255 - 8 * lane - j;
          sm->pick_above = r;
          sm->pick_here = v[j];
        }
      }
      __syncthreads();
      prefix = (prefix << 8) | (uint32_t)sm->pick_bin;
      run = sm->pick_above;
      *here = sm->pick_here;
      __syncthreads();
    }
    *above = run;
    return prefix;
  }
};

template <int DT>
__device__ __forceinline__ float load_logit(const void* p, int64_t i) {
  float x;
  if (DT == ES_DTYPE_F32) x = __ldg(reinterpret_cast<const float*>(p) + i);
  else if (DT == ES_DTYPE_F16) x = __half2float(reinterpret_cast<const __half*>(p)[i]);
  else x = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
  return isnan(x) ? -INFINITY : x + 0.f;      // -0 becomes +0: equal numbers have equal keys
}

template <int DT>
__global__ void __launch_bounds__(ST) sample_kernel(const SampleParams p) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ Shared shared;
  cg::cluster_group cl = cg::this_cluster();
  const int ranks = (int)cl.num_blocks(), rank = (int)cl.block_rank(), row = blockIdx.x / ranks;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Row R;
  R.x = reinterpret_cast<float*>(dyn);
  R.csum = reinterpret_cast<u64*>(dyn + (size_t)p.slice * sizeof(float));
  R.sm = &shared;
  R.ranks = ranks;
  R.rank = rank;
  R.first = rank * p.slice;
  const int real = max(0, min(p.V - R.first, p.slice));
  R.n = (real + CHUNK - 1) / CHUNK * CHUNK;

  // ---- the slice comes in; largest logit, lowest index ----
  u64 best = 0;
  for (int i = tid; i < R.n; i += ST) {
    const float v = i < real ? load_logit<DT>(p.logits, (int64_t)row * p.row_stride + R.first + i) : -INFINITY;
    R.x[i] = v;
    const u64 b = ((u64)key_of(v) << 32) | (uint32_t)~(R.first + i);
    best = b > best ? b : best;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) { const u64 o = __shfl_xor_sync(~0u, best, d); best = o > best ? o : best; }
  if (lane == 0) shared.warp_u64[warp] = best;
  __syncthreads();
  if (warp == 0) {
    best = lane < SW ? shared.warp_u64[lane] : 0;
#pragma unroll
    for (int d = 16; d; d >>= 1) { const u64 o = __shfl_xor_sync(~0u, best, d); best = o > best ? o : best; }
    if (lane == 0) shared.best = best;
  }
  cl.sync();
  best = 0;
  for (int r = 0; r < ranks; ++r) { const u64 o = cl.map_shared_rank(&shared, r)->best; best = o > best ? o : best; }

  R.xmax = of_key((uint32_t)(best >> 32));
  const int top = (int)~(uint32_t)best;
  const float T = p.temperature ? p.temperature[row] : 1.f;
  int token = top;
  float logprob = 0.f;
  if (R.xmax == -INFINITY) {
    token = -1;
    logprob = -INFINITY;
  } else if (T > 0.f) {
    R.c = 1.4426950408889634 / (double)T;
    R.key = 0; R.cut = INT_MAX; R.least = 1;
    const int k = p.top_k ? p.top_k[row] : 0;
    if (k > 0 && k < p.V) {
      // padding is -infinity behind the last real index: it ranks last among equals
      u64 above, here;
      R.key = R.descend([](float, int) { return (u64)1; }, (u64)k, &above, &here);
      const u64 want = (u64)k - above;
      if (here > want) {
        auto f = [&](float v, int) { return (u64)(key_of(v) == R.key); };
        R.sums(f);
        R.cut = R.find(f, want - 1);
      }
    }
    auto f = [&](float v, int i) { return R.kept(key_of(v), i) ? R.weight(v) : 0ull; };
    const float tp = p.top_p ? p.top_p[row] : 1.f;
    if (tp < 1.f) {
      const u64 all = R.sums(f);
      cl.sync();
      u64 target = (u64)ceil((double)fmaxf(tp, 0.f) * (double)all);
      target = target < 1 ? 1 : target > all ? all : target;
      u64 above, here;
      const uint32_t key = R.descend(f, target, &above, &here);
      const u64 w = R.weight(of_key(key));
      const u64 want = (target - above + w - 1) / w;              // of the here / w kept ones with this key
      int cut = key == R.key ? R.cut : INT_MAX;
      if (want < here / w) {
        auto tie = [&](float v, int i) { return (u64)(key_of(v) == key && i <= cut); };
        R.sums(tie);
        cut = R.find(tie, want - 1);
      }
      R.key = key;
      R.cut = cut;
    }
    if (p.min_p) {
      const float m = fminf(fmaxf(p.min_p[row], 0.f), 1.f);
      const u64 w = (u64)ceil((double)m * 17592186044416.0);
      R.least = w < 1 ? 1 : w;
    }
    auto last = [&](float v, int i) { const u64 w = R.kept(key_of(v), i) ? R.weight(v) : 0ull; return w >= R.least ? w : 0ull; };
    const u64 all = R.sums(last);
    const float u = fminf(fmaxf(p.u[row], 0.f), 1.f);
    u64 target = (u64)((double)u * (double)all);
    if (target >= all) target = all - 1;
    token = R.find(last, target);
    // the drawn token's own logit, from whichever CTA holds it
    if (token >= R.first && token < R.first + real && tid == 0) {
      const double t = R.x[token - R.first] == R.xmax ? 0.0 : ((double)R.x[token - R.first] - (double)R.xmax) * R.c;
      logprob = (float)((t - log2((double)all) + 44.0) * 0.6931471805599453);
      p.tokens[row] = token;
      if (p.logprobs) p.logprobs[row] = logprob;
    }
    cl.sync();                                // no CTA leaves while another may still read its shared memory
    return;
  }
  if (rank == 0 && tid == 0) {
    p.tokens[row] = token;
    if (p.logprobs) p.logprobs[row] = logprob;
  }
  cl.sync();
}

template <int DT>
es_status_t launch_sample(const SampleParams& p, int B, int ranks, cudaStream_t s) {
  const size_t smem = (size_t)p.slice * sizeof(float) + (size_t)(p.slice / CHUNK) * sizeof(u64);
  ES_CUDA_CHECK(cudaFuncSetAttribute(sample_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SLICE * 4 + MAX_SLICE / CHUNK * 8));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((long long)B * ranks));
  cfg.blockDim = dim3(ST);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ranks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ES_CUDA_CHECK(cudaLaunchKernelEx(&cfg, sample_kernel<DT>, p));
  return ES_OK;
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
  // a cluster per row while the machine has CTAs to spare and slices stay above 4096 elements, or where one CTA cannot
  // hold the row
  int ranks = 1;
  while (ranks < MAX_CLUSTER && (V > (long long)ranks * MAX_SLICE || (2LL * B * ranks <= sm_count() && V > 4096 * ranks))) ranks *= 2;
  const int slice = ((V + ranks - 1) / ranks + CHUNK - 1) / CHUNK * CHUNK;
  SampleParams p{logits, row_stride, u, temperature, top_p, min_p, top_k, tokens, logprobs, V, slice};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == ES_DTYPE_F32) return launch_sample<ES_DTYPE_F32>(p, B, ranks, s);
  if (dtype == ES_DTYPE_F16) return launch_sample<ES_DTYPE_F16>(p, B, ranks, s);
  return launch_sample<ES_DTYPE_BF16>(p, B, ranks, s);
}

}  // extern "C"
