// Slots of a paged cache for rows that come and go (focus_paged_extend).
//
//   extend_tables   one workgroup: pages of dropped rows onto the free list, then pages for
//                   new rows off it, both in the order of sequences by prefix sums; lengths,
//                   starts, offsets
//   extend_rows     the maps of the new rows
//
// Pages move one at a time through a list whose length every step needs, so all of them are
// moved by one workgroup; what there is to do is a few words a sequence, a page and a row.
#include "paged.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kRowThreads = 256;

struct Args {
  focus_paged_extend_desc d;
  int shift;            // log2 page_rows
};

// Inclusive sum over the workgroup in 64 bits; `total` the sum of all.
__device__ int64_t group_scan(int64_t x, int64_t* s_part, int64_t& total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int64_t y = __shfl_up(x, k);
    if (lane >= k) x += y;
  }
  __syncthreads();  // the last scan's sums are read
  if (lane == 63) s_part[wave] = x;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int64_t y = s_part[w];
    if (w < wave) x += y;
    total += y;
  }
  return x;
}

// Index of the first of n ascending values greater than x (n if none is).
template <typename T> __device__ inline int first_above(const T* v, int n, int64_t x) {
  int lo = 0;
  while (n > 0) {
    const int half = n / 2;
    if (v[lo + half] <= x) lo += half + 1, n -= half + 1;
    else n = half;
  }
  return lo;
}

// A sequence of this call.
struct Seq {
  int64_t add, n;       // add 0 past the batch
};
__device__ inline Seq sequence(const Args& a, int b, int64_t cap, int32_t& bits) {
  if (b >= a.d.batch) return {0, 0};
  const int64_t n = a.d.length[b];
  const int64_t clipped = n < 0 ? 0 : n > cap ? cap : n;
  if (clipped != n) bits |= FOCUS_ERR_BOUNDS;
  return {a.d.add[b], clipped};
}

__global__ __launch_bounds__(kThreads) void extend_tables(Args a) {
  __shared__ int64_t s_part[kWaves], s_upto[kThreads];
  __shared__ int s_first[kThreads];
  const focus_paged_extend_desc& d = a.d;
  const int tid = threadIdx.x, P = d.page_rows;
  const int64_t cap = (int64_t)d.max_pages * P;
  auto pages = [&](int64_t rows) { return (rows + P - 1) >> a.shift; };
  int32_t bits = 0;
  int64_t count = d.free_count[0];
  if (count < 0 || count > d.free_cap) count = count < 0 ? 0 : d.free_cap, bits |= FOCUS_ERR_BOUNDS;

  // rows that go
  for (int b0 = 0; b0 < d.batch; b0 += kThreads) {
    const int b = b0 + tid;
    const Seq q = sequence(a, b, cap, bits);
    const int64_t left = q.add < 0 ? max(q.n + q.add, (int64_t)0) : q.n;
    const int64_t back = pages(q.n) - pages(left);
    int64_t total;
    const int64_t upto = group_scan(back, s_part, total);
    s_upto[tid] = upto;
    s_first[tid] = (int)pages(left);
    __syncthreads();
    for (int64_t i = tid; i < total; i += kThreads) {
      const int k = first_above(s_upto, kThreads, i);
      const int64_t before = k > 0 ? s_upto[k - 1] : 0;
      int32_t* entry = d.table + (int64_t)(b0 + k) * d.max_pages + s_first[k] + (i - before);
      if (count + i < d.free_cap) d.free_pages[count + i] = *entry;
      else bits |= FOCUS_ERR_CAPACITY;
      *entry = -1;
    }
    count = min(count + total, (int64_t)d.free_cap);
    if (b < d.batch && q.add <= 0) d.length[b] = (int)left, d.start[b] = (int)left;
  }
  __syncthreads();

  // rows that come
  int64_t rows = 0, needs = 0, taken = 0;  // of the sequences before; pages handed out
  for (int b0 = 0; b0 < d.batch; b0 += kThreads) {
    const int b = b0 + tid;
    int32_t unused = 0;
    Seq q = sequence(a, b, cap, unused);
    q.add = max(q.add, (int64_t)0);
    int64_t all_rows, all_needs;
    const int64_t end = rows + group_scan(q.add, s_part, all_rows);
    const bool fits = q.add > 0 && q.n + q.add <= cap && end <= d.n_rows;
    const int64_t need = fits ? pages(q.n + q.add) - pages(q.n) : 0;
    const int64_t upto = group_scan(need, s_part, all_needs);
    const bool served = fits && (need == 0 || needs + upto <= count);
    // (those that get pages are the first ones that need any)
    s_upto[tid] = upto;
    s_first[tid] = (int)pages(q.n);
    int64_t here;  // pages handed out by this round
    group_scan(served ? need : 0, s_part, here);
    for (int64_t i = tid; i < here; i += kThreads) {
      const int k = first_above(s_upto, kThreads, i);
      const int64_t before = k > 0 ? s_upto[k - 1] : 0;
      d.table[(int64_t)(b0 + k) * d.max_pages + s_first[k] + (i - before)] = d.free_pages[count - 1 - needs - i];
    }
    if (b < d.batch) {
      d.cu_rows[b + 1] = (int)min(end, (int64_t)INT32_MAX);
      if (q.add > 0) {
        d.start[b] = served ? (int)q.n : -1;
        d.length[b] = (int)(served ? q.n + q.add : q.n);
        if (!served) bits |= FOCUS_ERR_CAPACITY;
      }
    }
    rows += all_rows, needs += all_needs, taken += here;
  }
  if (tid == 0) d.cu_rows[0] = 0, d.free_count[0] = (int)(count - taken);
  if (bits) focus::raise_err(d.err, bits);
}

__global__ __launch_bounds__(kRowThreads) void extend_rows(Args a) {
  const focus_paged_extend_desc& d = a.d;
  const int64_t t = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
  if (t >= d.n_rows) return;
  int seq = -1, slot = -1, pos = -1;
  const int b = first_above(d.cu_rows + 1, d.batch, t);
  if (b < d.batch) {
    const int i = (int)(t - d.cu_rows[b]), start = d.start[b];
    seq = b;
    slot = start < 0 ? -1 : start + i;
    pos = d.first_pos ? (int)((uint32_t)d.first_pos[b] + (uint32_t)i) : slot;
  }
  if (d.row_seq) d.row_seq[t] = seq;
  if (d.row_slot) d.row_slot[t] = slot;
  if (d.row_pos) d.row_pos[t] = pos;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

extern "C" focus_status focus_paged_extend(const focus_paged_extend_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  if (d->batch < 0 || d->max_pages < 0 || d->free_cap < 0 || d->n_rows < 0) return FOCUS_E_ARG;
  if (d->page_rows < 8 || d->page_rows > 1024 || (d->page_rows & (d->page_rows - 1))) return FOCUS_E_UNSUPPORTED;
  if ((int64_t)d->max_pages * d->page_rows > INT32_MAX / 2 || d->n_rows > INT32_MAX) return FOCUS_E_SHAPE;
  if (!d->cu_rows || !d->free_count || (d->free_cap > 0 && !d->free_pages)) return FOCUS_E_NULL;
  if (d->batch > 0 && (!d->length || !d->add || !d->start || (d->max_pages > 0 && !d->table))) return FOCUS_E_NULL;
  for (const void* p : {(const void*)d->table, (const void*)d->length, (const void*)d->add, (const void*)d->free_pages,
                        (const void*)d->free_count, (const void*)d->first_pos, (const void*)d->start,
                        (const void*)d->cu_rows, (const void*)d->row_seq, (const void*)d->row_slot,
                        (const void*)d->row_pos, (const void*)d->err})
    if (!aligned4(p)) return FOCUS_E_ARG;
  Args a = {*d, __builtin_ctz((unsigned)d->page_rows)};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(extend_tables, dim3(1), dim3(kThreads), 0, s, a);
  const focus_status st = focus::launch_status();
  if (st != FOCUS_OK || d->n_rows == 0 || (!d->row_seq && !d->row_slot && !d->row_pos)) return st;
  hipLaunchKernelGGL(extend_rows, dim3((uint32_t)focus::ceil_div(d->n_rows, kRowThreads)), dim3(kRowThreads), 0, s, a);
  return focus::launch_status();
}
