// A paged K/V cache cut down to a budget by accumulated weight (focus_paged_evict).
//
//   evict_select  one workgroup per (sequence, KV head): the weight of the last row
//                 kept by a radix selection, eight bits a pass over an order-preserving
//                 integer of the weights, then one ordered pass that writes the kept
//                 rows (prefix counts settle which of the equal weights stay)
//   evict_copy    the kept rows and their weights to the pages of `out`
#include "paged.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kCopy = 256;

// Weights as integers of the same order; -0 counts as +0, every NaN as the greatest.
__device__ inline uint32_t order_of(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Rows kept of sequence b: min(length, budget), and what keep and out can hold.
__device__ inline int kept_rows(const focus_paged_evict_desc& d, int b, int n, int32_t* bits) {
  int m = d.budgets ? d.budgets[b] : d.budget;
  if (m < 0) *bits |= FOCUS_ERR_BOUNDS, m = 0;
  m = min(m, n);
  const int64_t room = min((int64_t)d.out.max_pages * d.out.page_rows, d.keep_rows);
  if (m > room) *bits |= FOCUS_ERR_CAPACITY, m = (int)room;
  return m;
}

// Exclusive prefix sum of x over the workgroup; *total: the sum.
__device__ inline int scan(int x, int* waves, int* total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  int y = x;
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const int z = __shfl_up(y, i);
    if (lane >= i) y += z;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = y;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += waves[w];
    sum += waves[w];
  }
  *total = sum;
  return before + y - x;
}

__global__ __launch_bounds__(kThreads) void evict_select(focus_paged_evict_desc d) {
  __shared__ int hist[256], waves[kWaves];
  __shared__ int s_bucket, s_rest;
  const int K = d.cache.n_kv_heads, b = blockIdx.x / K, g = blockIdx.x % K, tid = threadIdx.x;
  const int n = focus::paged_length(d.cache, b);
  int32_t bits = n != d.cache.length[b] ? FOCUS_ERR_CAPACITY : 0;
  const int m = kept_rows(d, b, n, &bits);
  if (bits && tid == 0 && g == 0) focus::raise_err(d.err, bits);
  const int recent = min(d.recent, m), old = n - recent, take = m - recent;
  const float* w = d.cache.weight + ((int64_t)b * K + g) * d.cache.weight_rows;
  int32_t* keep = d.keep + ((int64_t)b * K + g) * d.keep_rows;
  for (int64_t j = m + tid; j < d.keep_rows; j += kThreads) keep[j] = -1;
  for (int j = tid; j < recent; j += kThreads) keep[take + j] = old + j;
  if (take == 0) return;
  // threshold: the take-th greatest of the old rows; `equal` of the rows that equal it stay
  uint32_t prefix = 0;
  int equal = take;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    for (int r = tid; r < old; r += kThreads) {
      const uint32_t u = order_of(w[r]);
      if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift) & 255], 1);
    }
    __syncthreads();
    // rows in the buckets above this thread's
    const int x = tid < 256 ? hist[255 - tid] : 0;
    int total;
    const int above = scan(x, waves, &total);
    if (tid < 256 && above < equal && above + x >= equal) s_bucket = 255 - tid, s_rest = equal - above;
    __syncthreads();
    prefix |= (uint32_t)s_bucket << shift;
    equal = s_rest;
  }
  int at = 0, ties = 0;
  for (int r0 = 0; r0 < old; r0 += kThreads) {
    const int r = r0 + tid;
    const uint32_t u = r < old ? order_of(w[r]) : 0u;
    const bool tie = r < old && u == prefix;
    int total;
    const int before = scan(tie ? 1 : 0, waves, &total);
    const bool in = r < old && (u > prefix || (tie && ties + before < equal));
    ties += total;
    const int j = at + scan(in ? 1 : 0, waves, &total);
    if (in) keep[j] = r;
    at += total;
  }
}

__global__ __launch_bounds__(kCopy) void evict_copy(focus_paged_evict_desc d, int in_shift, int out_shift, int pieces,
                                                    int es) {
  const int K = d.cache.n_kv_heads, b = blockIdx.x / K, g = blockIdx.x % K;
  if (blockIdx.y == 0 && g == 0 && threadIdx.x == 0) {
    int32_t bits = 0;
    d.out.length[b] = kept_rows(d, b, focus::paged_length(d.cache, b), &bits);
  }
  const int32_t* keep = d.keep + ((int64_t)b * K + g) * d.keep_rows;
  const int per = kCopy / pieces, sub = threadIdx.x % pieces;
  if ((int)threadIdx.x >= per * pieces) return;
  for (int64_t j = (int64_t)blockIdx.y * per + threadIdx.x / pieces; j < d.keep_rows; j += (int64_t)gridDim.y * per) {
    const int r = keep[j];
    if (r < 0) break;
    const int64_t sp = focus::page_of(d.cache, b, r, in_shift), dp = focus::page_of(d.out, b, (int)j, out_shift);
    if (sub == 0 && d.out.weight)
      d.out.weight[((int64_t)b * K + g) * d.out.weight_rows + j] =
          d.cache.weight[((int64_t)b * K + g) * d.cache.weight_rows + r];
    if (sp < 0 || dp < 0) {
      if (sub == 0) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
      continue;
    }
    const int64_t src = focus::row_at(d.cache, sp, r, g) * es / 16 + sub, dst = focus::row_at(d.out, dp, (int)j, g) * es / 16 + sub;
    reinterpret_cast<uint4*>(d.out.k)[dst] = reinterpret_cast<const uint4*>(d.cache.k)[src];
    reinterpret_cast<uint4*>(d.out.v)[dst] = reinterpret_cast<const uint4*>(d.cache.v)[src];
  }
}

focus_status validate(const focus_paged_evict_desc* d) {
  focus_status st = focus::check_paged(d->cache);
  if (st == FOCUS_OK) st = focus::check_paged(d->out);
  if (st != FOCUS_OK) return st;
  if (d->cache.dtype != d->out.dtype || d->cache.n_kv_heads != d->out.n_kv_heads ||
      d->cache.head_dim != d->out.head_dim || d->cache.batch != d->out.batch)
    return FOCUS_E_SHAPE;
  if ((!d->budgets && d->budget < 0) || d->recent < 0 || d->keep_rows < 0) return FOCUS_E_ARG;
  if (d->keep_rows > INT32_MAX / 2 || (int64_t)d->cache.batch * d->cache.n_kv_heads > INT32_MAX / kThreads)
    return FOCUS_E_SHAPE;
  return FOCUS_OK;
}

}  // namespace

extern "C" size_t focus_paged_evict_workspace(const focus_paged_evict_desc*) { return 0; }

extern "C" focus_status focus_paged_evict(const focus_paged_evict_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  focus_status st = validate(d);
  if (st != FOCUS_OK) return st;
  if (d->cache.batch == 0) return FOCUS_OK;
  if (!d->cache.weight || (d->keep_rows > 0 && !d->keep)) return FOCUS_E_NULL;
  if (d->out.weight == d->cache.weight || (reinterpret_cast<uintptr_t>(d->keep) & 3u) ||
      (reinterpret_cast<uintptr_t>(d->budgets) & 3u))
    return FOCUS_E_ARG;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const uint32_t heads = (uint32_t)(d->cache.batch * d->cache.n_kv_heads);
  hipLaunchKernelGGL(evict_select, dim3(heads), dim3(kThreads), 0, s, *d);
  if ((st = focus::launch_status()) != FOCUS_OK) return st;
  const int es = (int)focus::elt_bytes(d->cache.dtype), pieces = d->cache.head_dim * es / 16;
  const int64_t y = focus::ceil_div(d->keep_rows > 0 ? d->keep_rows : 1, (kCopy / pieces) * 8);
  hipLaunchKernelGGL(evict_copy, dim3(heads, (uint32_t)(y > 1024 ? 1024 : y)), dim3(kCopy), 0, s, *d,
                     focus::page_shift(d->cache), focus::page_shift(d->out), pieces, es);
  return focus::launch_status();
}
