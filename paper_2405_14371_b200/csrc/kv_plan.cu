// Block tables and slot maps from request lengths: page allocation, page return and the row layout of a batch in one
// launch, without the host knowing any result.
//
// Everything is a prefix sum over the requests followed by independent writes:
//   rows_b = max(new - old, 0), need_b / give_b = pages gained / given up, and with R = sum(give), `have` pages on the
//   stack and avail = have + R:  b is served iff its inclusive row sum fits max_rows and its inclusive need sum fits avail.
// Both sums only grow with b, so the served requests that take pages are a prefix and the pop number of a page is
// the exclusive sum itself.  Pop i is entry avail - 1 - i of "the stack with the returned pages on it": a stack entry
// below `have`, else a returned page, found by a search in the sums of give.  When pops exceed returns no stack entry
// is written, and otherwise no stack entry is read, so pops and pushes need no order between them.
//
// One cluster does it all: every CTA scans the lengths for itself (a few KB out of L2, cheaper than handing sums around),
// then the CTAs share the page work, meet once, and share the rest.  The meeting orders table writes before the rows that
// read them.  Small calls are bound by latency and run as one CTA that makes the rows too; large ones leave the rows (12
// bytes each) to a second kernel over the whole machine.
//
// Bound by latency: 64 decoding requests take 4.0 us a call (a dependent chain of lengths, sums, stack, table and rows
// with barriers in it).  1024 requests of which a tenth brings prompts (75 000 rows) and a tenth returns 25 000 pages, and
// the same back (410 000 rows), take 27 us for both calls (7 MB, 1 us at the copy rate): 9 us each in the cluster, sums and
// three rounds of search, read and write, the rest the rows.
#include <cooperative_groups.h>
#include <limits.h>

#include "es_internal.cuh"
#include "launch.cuh"

namespace cg = cooperative_groups;

namespace es {
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_FEW = 128;      // threads of a call with few requests and rows: barriers and launch cost less
constexpr int PLAN_MAX_B = 8192;

struct PlanParams {
  const int *old_len, *new_len;
  int *table, *free_pages, *free_count;
  int B, pps, P, log2P, n_pages, max_rows, max_runs;
  int *row_offsets, *slot_map, *positions, *row_seq, *runs, *len_out;
};

// Pages given up and gained are entries of the table, at most 2^30.  Rows stop counting at `full`, one more than there is
// room for; sums of such numbers are the same in any order.
struct Sums { uint32_t give, rows, need; };

__device__ __forceinline__ Sums add(const Sums& a, const Sums& b, uint32_t full) { return {a.give + b.give, min(a.rows + b.rows, full), a.need + b.need}; }

// pages of a sequence
__device__ __forceinline__ int pages_of(const PlanParams& p, int len) { return (int)(((uint32_t)len + (uint32_t)p.P - 1) >> p.log2P); }

// inclusive scan over the block; `total` is the block's sum.  All threads call.
template <int WARPS>
__device__ __forceinline__ Sums block_scan(Sums v, Sums* warp_sums, Sums* total, uint32_t full) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Sums o = {__shfl_up_sync(~0u, v.give, d), __shfl_up_sync(~0u, v.rows, d), __shfl_up_sync(~0u, v.need, d)};
    if (lane >= d) v = add(v, o, full);
  }
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  if (warp == 0) {
    Sums w = lane < WARPS ? warp_sums[lane] : Sums{0, 0, 0};
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const Sums o = {__shfl_up_sync(~0u, w.give, d), __shfl_up_sync(~0u, w.rows, d), __shfl_up_sync(~0u, w.need, d)};
      if (lane >= d) w = add(w, o, full);
    }
    if (lane < WARPS) warp_sums[lane] = w;
  }
  __syncthreads();
  if (warp > 0) v = add(v, warp_sums[warp - 1], full);
  *total = warp_sums[WARPS - 1];
  __syncthreads();
  return v;
}

template <int WARPS>
__device__ __forceinline__ int block_scan_int(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(~0u, v, d);
    if (lane >= d) v += o;
  }
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  if (warp == 0) {
    int w = lane < WARPS ? warp_sums[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(~0u, w, d);
      if (lane >= d) w += o;
    }
    if (lane < WARPS) warp_sums[lane] = w;
  }
  __syncthreads();
  if (warp > 0) v += warp_sums[warp - 1];
  *total = warp_sums[WARPS - 1];
  __syncthreads();
  return v;
}

// The request that owns item i: the b with off[b] <= i < off[b + 1]; off[0] = 0, i < off[B].  A fixed number of steps
// without branches, so that the searches of several items overlap; `top` is the largest power of two not above B.
__device__ __forceinline__ int owner(const int* off, int B, int top, int i) {
  int b = 0;
  for (int step = top; step; step >>= 1) {
    const int mid = b + step;
    if (mid < B && off[mid] <= i) b = mid;
  }
  return b;
}

constexpr int FLIGHT = 4;          // items of a thread under way at a time

// slot of a position, -1 where the table holds no page
__device__ __forceinline__ int slot_of(const PlanParams& p, int seq, int pos) {
  const int lp = pos >> p.log2P, page = __ldcg(p.table + (int64_t)seq * p.pps + lp);
  return page >= 0 && page < p.n_pages ? page * p.P + (pos & (p.P - 1)) : -1;
}

template <bool ROWS, int THREADS>
__global__ void __launch_bounds__(THREADS, 1) kv_plan_kernel(const PlanParams p) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int WARPS = THREADS / 32;
  extern __shared__ int sm[];
  __shared__ Sums warp_sums[WARPS];
  __shared__ int warp_ints[WARPS];
  const int B = p.B, P = p.P, tid = threadIdx.x;
  int* s_old = sm;                 // [B]
  int* s_new = s_old + B;          // [B]   the length to hold: the request's, or the old one when refused
  int* row_off = s_new + B;        // [B + 1]
  int* need_off = row_off + B + 1; // [B + 1]   served requests only
  int* give_off = need_off + B + 1;
  int* run_off = give_off + B + 1;
  const int top = 1 << (31 - __clz(B));
  const int ranks = gridDim.x, rank = blockIdx.x;
  const bool alloc = p.free_pages != nullptr;
  const long long cap = (long long)p.pps * P;

  // ---- the sums (every CTA for itself) ----
  int have = 0;
  if (alloc) { have = __ldcg(p.free_count); have = have < 0 ? 0 : min(have, p.n_pages); }
  const uint32_t full = (uint32_t)p.max_rows + 1;
  Sums carry = {0, 0, 0};
  if (tid == 0) { row_off[0] = 0; need_off[0] = 0; give_off[0] = 0; run_off[0] = 0; }
  for (int base = 0; base < B; base += THREADS) {
    const int b = base + tid;
    int o = 0, n = 0;
    if (b < B) { o = __ldcg(p.old_len + b); n = __ldcg(p.new_len + b); }
    const bool ok = o >= 0 && o <= cap && n >= 0 && n <= cap;
    const int oo = ok ? o : 0, nn = ok ? n : 0;
    const int po = pages_of(p, oo), pn = pages_of(p, nn);
    Sums v = {(uint32_t)max(po - pn, 0), min((uint32_t)max(nn - oo, 0), full), (uint32_t)max(pn - po, 0)}, total;
    v = add(block_scan<WARPS>(v, warp_sums, &total, full), carry, full);
    if (b < B) {
      s_old[b] = o;
      s_new[b] = ok ? n : o;
      give_off[b + 1] = alloc ? (int)v.give : 0;
      row_off[b + 1] = (int)v.rows;
      need_off[b + 1] = (int)v.need;
    }
    carry = add(carry, total, full);
  }
  const int given = alloc ? (int)carry.give : 0;
  const long long avail = (long long)have + given;
  __syncthreads();

  // ---- who is served; the runs of the served ----
  int runs_before = 0, taken = 0;
  for (int base = 0; base < B; base += THREADS) {
    const int b = base + tid;
    int n_runs = 0;
    if (b < B) {
      const int o = s_old[b], n = s_new[b];
      if (n > o) {                                          // gains rows (a request with lengths out of range has n == o)
        const bool need = pages_of(p, n) > pages_of(p, o);
        const bool fits = row_off[b + 1] <= p.max_rows && (!alloc || !need || need_off[b + 1] <= avail);
        if (fits) n_runs = ((n - 1) >> p.log2P) - (o >> p.log2P) + 1;
        else s_new[b] = o;
      }
    }
    int total;
    n_runs = block_scan_int<WARPS>(n_runs, warp_ints, &total);
    if (b < B) run_off[b + 1] = runs_before + n_runs;
    runs_before += total;
  }
  __syncthreads();
  // The served requests that take pages are a prefix of those that need some (behind the first need sum beyond avail, or row sum
  // beyond max_rows, all of these are refused), so the pages taken are the inclusive need of the last of them.
  {
    int most = 0;
    for (int b = tid; b < B; b += THREADS)
      if (s_new[b] > s_old[b] && need_off[b + 1] > need_off[b]) most = max(most, need_off[b + 1]);
    most = __reduce_max_sync(~0u, most);
    if ((tid & 31) == 0) warp_ints[tid >> 5] = most;
    __syncthreads();
    taken = alloc ? __reduce_max_sync(~0u, warp_ints[tid & (WARPS - 1)]) : 0;
  }
  const int rows_all = min(row_off[B], p.max_rows);
  const int stride = THREADS * ranks, first = rank * THREADS + tid;

  // ---- pages: pops into the table, left-over returns onto the stack; who reads a returned entry, and only one does, clears it ----
  auto returned = [&](int i) -> int* {
    const int b = owner(give_off, B, top, i);
    return p.table + (int64_t)b * p.pps + pages_of(p, s_new[b]) + i - give_off[b];
  };
  if (alloc) {
    for (int base = first; base < taken; base += FLIGHT * stride) {
      int page[FLIGHT], *from[FLIGHT];
#pragma unroll
      for (int j = 0; j < FLIGHT; ++j) {
        const int i = base + j * stride;
        const long long v = avail - 1 - i;
        page[j] = -1;
        from[j] = i < taken && v >= have ? returned((int)(v - have)) : nullptr;
        if (i < taken) page[j] = __ldcg(from[j] ? from[j] : p.free_pages + v);
      }
#pragma unroll
      for (int j = 0; j < FLIGHT; ++j) {
        const int i = base + j * stride;
        if (i >= taken) break;
        if (from[j]) *from[j] = -1;
        const int b = owner(need_off, B, top, i);
        p.table[(int64_t)b * p.pps + pages_of(p, s_old[b]) + i - need_off[b]] = page[j];
      }
    }
    for (int base = first; base < given - taken; base += FLIGHT * stride) {
      int page[FLIGHT], *from[FLIGHT];
#pragma unroll
      for (int j = 0; j < FLIGHT; ++j) {
        from[j] = base + j * stride < given - taken ? returned(base + j * stride) : nullptr;
        if (from[j]) page[j] = __ldcg(from[j]);
      }
#pragma unroll
      for (int j = 0; j < FLIGHT; ++j) {
        if (!from[j]) break;
        *from[j] = -1;
        const long long at = have + (long long)base + j * stride;
        if (at < p.n_pages) p.free_pages[at] = page[j];
      }
    }
  }

  // ---- the CTAs meet: table entries written above are read below ----
  if (ranks > 1) cg::this_cluster().sync(); else __syncthreads();

  if (alloc && first == 0) *p.free_count = (int)min(avail - taken, (long long)p.n_pages);
  for (int b = first; b <= B; b += stride) p.row_offsets[b] = min(row_off[b], p.max_rows);
  for (int b = first; b < B; b += stride) p.len_out[b] = s_new[b];
  for (int base = first; base < p.max_runs; base += FLIGHT * stride) {            // run i: a page of its request, from the row that begins it
    int row[FLIGHT], page[FLIGHT];
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j) {
      const int i = base + j * stride;
      row[j] = page[j] = -1;
      if (i < runs_before) {
        const int b = owner(run_off, B, top, i), o = s_old[b], lp = (o >> p.log2P) + (i - run_off[b]);
        page[j] = __ldcg(p.table + (int64_t)b * p.pps + lp);
        row[j] = row_off[b] + max(lp * P - o, 0);
      }
    }
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j)
      if (base + j * stride < p.max_runs) p.runs[base + j * stride] = page[j] >= 0 && page[j] < p.n_pages ? row[j] : -1;
  }
  if (ROWS)
    for (int r = first; r < p.max_rows; r += stride) {
      int slot = -1, pos = -1, seq = -1;
      if (r < rows_all) {
        seq = owner(row_off, B, top, r);
        const int o = s_old[seq];
        pos = o + (r - row_off[seq]);
        if (s_new[seq] > o) slot = slot_of(p, seq, pos);
      }
      p.slot_map[r] = slot;
      p.positions[r] = pos;
      p.row_seq[r] = seq;
    }
}

// The rows of a large call.  A request was served exactly if its length became the new one; where it began follows.
__global__ void __launch_bounds__(PLAN_THREADS, 1) kv_plan_rows_kernel(const PlanParams p) {
  extern __shared__ int sm[];
  int* row_off = sm;               // [B + 1]
  const int B = p.B, top = 1 << (31 - __clz(B));
  pdl_wait();
  pdl_launch_dependents();
  for (int b = threadIdx.x; b <= B; b += PLAN_THREADS) row_off[b] = __ldcg(p.row_offsets + b);
  __syncthreads();
  const int rows_all = row_off[B];
  // neighbouring threads take neighbouring rows
  for (int64_t base = (int64_t)blockIdx.x * PLAN_THREADS + threadIdx.x; base < p.max_rows; base += (int64_t)gridDim.x * PLAN_THREADS) {
    const int r = (int)base;
    int slot = -1, pos = -1, seq = -1;
    if (r < rows_all) {
      seq = owner(row_off, B, top, r);
      const int held = __ldcg(p.len_out + seq), want = __ldcg(p.new_len + seq);
      const bool served = held == want;
      pos = served ? held - (row_off[seq + 1] - r) : held + (r - row_off[seq]);
      if (served) slot = slot_of(p, seq, pos);
    }
    p.slot_map[r] = slot;
    p.positions[r] = pos;
    p.row_seq[r] = seq;
  }
}

// CTAs of a large call's cluster: 16 where the device places such clusters (a call that returns 25 000 pages and one that
// takes as many: 27 us together, with 8 30 us), else the portable 8.
int plan_cluster() {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 8;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n) return n;
  const auto kern = kv_plan_kernel<false, PLAN_THREADS>;
  const size_t smem = (6 * PLAN_MAX_B + 4) * sizeof(int);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(16);
  cfg.blockDim = dim3(PLAN_THREADS);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 16;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int fit = 0;
  n = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
              cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) == cudaSuccess &&
              cudaOccupancyMaxActiveClusters(&fit, kern, &cfg) == cudaSuccess && fit > 0 ? 16 : 8;
  cudaGetLastError();                // a refusal of the size is an answer, not an error of this call
  known[dev].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace
}  // namespace es

extern "C" {

int32_t es_op_kv_plan_max_runs(int32_t B, int32_t max_rows, int32_t page_tokens) {
  if (B <= 0 || max_rows <= 0 || page_tokens <= 0) return 0;
  const long long n = (long long)max_rows / page_tokens + 2LL * B;      // n rows of a request touch at most n / P + 2 pages
  return (int32_t)(n < max_rows ? n : max_rows);
}

es_status_t es_op_kv_plan(const int32_t* old_len, const int32_t* new_len, int32_t* block_table, int32_t* free_pages,
                          int32_t* free_count, int32_t B, int32_t pages_per_seq, int32_t page_tokens, int32_t n_pages,
                          int32_t max_rows, int32_t* row_offsets, int32_t* slot_map, int32_t* positions,
                          int32_t* row_seq, int32_t* runs, int32_t* len_out, void* stream) {
  using namespace es;
  if (!old_len || !new_len || !block_table || !row_offsets || !slot_map || !positions || !row_seq || !runs || !len_out)
    return fail(ES_ERR_INVALID_ARG, "null argument");
  if (!free_pages != !free_count) return fail(ES_ERR_INVALID_ARG, "free_pages and free_count go together");
  if (B <= 0 || pages_per_seq <= 0 || page_tokens <= 0 || n_pages <= 0 || max_rows <= 0)
    return fail(ES_ERR_INVALID_ARG, "bad sizes");
  if (page_tokens < 16 || (page_tokens & (page_tokens - 1))) return fail(ES_ERR_SHAPE, "page_tokens must be a power of two >= 16");
  if (B > PLAN_MAX_B) return fail(ES_ERR_RANGE, "B = %d exceeds %d requests", B, PLAN_MAX_B);
  if ((long long)pages_per_seq * page_tokens > INT32_MAX || (long long)n_pages * page_tokens > INT32_MAX)
    return fail(ES_ERR_RANGE, "pages_per_seq or n_pages times page_tokens exceeds 2^31 - 1");
  if (max_rows > (1 << 30)) return fail(ES_ERR_RANGE, "max_rows exceeds 2^30");
  if ((long long)B * pages_per_seq > (1 << 30)) return fail(ES_ERR_RANGE, "the block table has more than 2^30 entries");
  if (len_out == new_len) return fail(ES_ERR_INVALID_ARG, "len_out may be old_len, not new_len");      // a large call's rows compare the two
  int log2P = 0;
  while ((1 << log2P) < page_tokens) ++log2P;
  PlanParams p{old_len, new_len, block_table, free_pages, free_count, B, pages_per_seq, page_tokens, log2P, n_pages, max_rows,
               es_op_kv_plan_max_runs(B, max_rows, page_tokens), row_offsets, slot_map, positions, row_seq, runs, len_out};
  const size_t smem = (size_t)(6 * B + 4) * sizeof(int);
  // One CTA as long as it writes the rows in less than the time that a cluster and a second launch cost: 1024 rows take 4.1 -
  // 4.3 us in one CTA and 5.8 - 6.2 us in two kernels, 2048 4.9 - 5.2 and 6.2 - 6.4, 4096 5.7 - 7.2 and 6.0 - 6.7.  128
  // threads for the smallest: 64 requests of one row 3.5 us, with 1024 threads 4.3 us; of eight rows 5.0 and 4.5 us.
  const bool small = max_rows <= 2048;
  const bool few = small && max_rows <= 2 * PLAN_FEW && B <= PLAN_FEW;
  auto kern = few ? kv_plan_kernel<true, PLAN_FEW> : small ? kv_plan_kernel<true, PLAN_THREADS> : kv_plan_kernel<false, PLAN_THREADS>;
  static std::atomic<uint64_t> allowed[2];
  if (smem > 48 * 1024) ES_CUDA_CHECK(allow_shared_memory(kern, (int)((6 * PLAN_MAX_B + 4) * sizeof(int)), &allowed[small]));
  const int ranks = small ? 1 : plan_cluster();
  ES_CUDA_CHECK(launch_clusters(kern, small ? 0 : ranks, dim3(ranks), dim3(few ? PLAN_FEW : PLAN_THREADS), smem, (cudaStream_t)stream, tunables().pdl != 0, p));
  if (!small) {
    const int blocks = (int)((max_rows + (long long)PLAN_THREADS - 1) / PLAN_THREADS);
    const int most = 2 * sm_count();
    ES_CUDA_CHECK(launch_kernel(kv_plan_rows_kernel, dim3(blocks < most ? blocks : most), dim3(PLAN_THREADS), (size_t)(B + 1) * sizeof(int),
                                (cudaStream_t)stream, tunables().pdl != 0, p));
  }
  return ES_OK;
}

}  // extern "C"
