// Slots of a paged cache for rows that come and go (focus_paged_extend).
//
//   extend_tables   one workgroup: pages of dropped rows onto the free list, then pages for
//                   new rows off it, both in the order of sequences by prefix sums; lengths,
//                   starts, offsets, and the maps of the new rows where these are few
//   extend_rows     the maps of many rows
//
// Pages move through one list in an order that is fixed, so all of them are moved by one
// workgroup; what there is to do is a few words a sequence, a page and a row, and what it takes
// is a chain of latencies: the lengths, the sums over the sequences, the pages, their entries.
// A step of 64 sequences takes 4.7 us, 500 prompts and endings of 123 000 rows and 2 200 pages
// 7.9 + 3.8; with sums by shuffles in 64 bits, two scans more and a second launch for every call
// 15 and 15.3.
#include "paged.h"

namespace {

constexpr int kFew = 256, kMany = 1024;  // threads of extend_tables for up to so many sequences, and for more
constexpr int kMapRounds = 8;            // rows that a thread of it maps at most
constexpr int kRowThreads = 256;

struct Args {
  focus_paged_extend_desc d;
  int shift;            // log2 page_rows
  bool maps;            // extend_tables writes the rows' maps
};

// Sum of two numbers from 0 up, at most 2^31 - 1.
__device__ inline int add_up(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)INT32_MAX); }

// Inclusive sums over the workgroup of three values from 0 up; the third may pass 2^31 - 1
// and stays there.  The caller's barriers keep s_part until all have read it.
template <int THREADS>
__device__ void group_scan(int (&x)[3], int (*s_part)[3], int (&total)[3]) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  x[0] = focus::wave_scan(x[0]);
  x[1] = focus::wave_scan(x[1]);
  x[2] = focus::wave_prefix(x[2], add_up);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (lane == 63) s_part[wave][i] = x[i];
    total[i] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int y = s_part[w][i];
      if (w < wave) x[i] = add_up(x[i], y);
      total[i] = add_up(total[i], y);
    }
}

// Index of the first of THREADS ascending values in LDS greater than x, where one is.
template <int THREADS> __device__ inline int first_above(const int* v, int x) {
  int lo = 0;
#pragma unroll
  for (int half = THREADS / 2; half > 0; half /= 2) lo += v[lo + half - 1] <= x ? half : 0;
  return lo;
}

// f(k, i) of items i = from .. to - 1, k the first sequence whose sum `upto` is greater than i;
// kTogether of a thread's at once, so that their searches and loads overlap.
constexpr int kTogether = 4;
template <int THREADS, typename Load, typename Store>
__device__ inline void each_page(const int* upto, int from, int to, Load load, Store store) {
  for (int i0 = from + (int)threadIdx.x; i0 < to; i0 += kTogether * THREADS) {
    int k[kTogether], page[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      if (i0 - (int)threadIdx.x + j * THREADS >= to) break;  // for all threads
      const int i = min(i0 + j * THREADS, to - 1);
      k[j] = first_above<THREADS>(upto, i);
      page[j] = load(k[j], i);
    }
#pragma unroll
    for (int j = 0; j < kTogether; ++j)
      if (to - i0 > j * THREADS) store(k[j], i0 + j * THREADS, page[j]);
  }
}

__device__ inline void write_row(const focus_paged_extend_desc& d, int t, int seq, int start, int i) {
  const int slot = start < 0 ? -1 : start + i;
  if (d.row_seq) d.row_seq[t] = seq;
  if (d.row_slot) d.row_slot[t] = slot;
  if (d.row_pos) d.row_pos[t] = seq < 0 ? -1 : d.first_pos ? (int)((uint32_t)d.first_pos[seq] + (uint32_t)i) : slot;
}

// A thread a sequence; more sequences than threads take rounds, all of which give back before
// any takes.  All sums over pages are below 2^31, as the tables' entries are.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void extend_tables(Args a) {
  __shared__ int s_part[THREADS / 64][3], s_upto[2][THREADS], s_first[2][THREADS], s_end[THREADS], s_start[THREADS], s_taken;
  const focus_paged_extend_desc& d = a.d;
  const int tid = threadIdx.x, P = d.page_rows, cap = d.max_pages * P;
  const bool once = d.batch <= THREADS;
  auto pages = [&](int rows) { return (rows + P - 1) >> a.shift; };
  int32_t bits = 0;

  // what sequence b asks for
  int n, left, come;  // rows; of these, when the dropped ones have gone; new ones
  bool room;          // the new ones fit the table
  int x[3], total[3];
  auto ask = [&](int b) {
    const int length = b < d.batch ? d.length[b] : 0, add = b < d.batch ? d.add[b] : 0;
    n = min(max(length, 0), cap);
    if (n != length) bits |= FOCUS_ERR_BOUNDS;
    left = add < 0 ? max(n + max(add, -n), 0) : n;
    come = max(add, 0);
    room = come <= cap - n;
    x[0] = pages(n) - pages(left), x[1] = come > 0 && room ? pages(n + come) - pages(n) : 0, x[2] = come;
  };

  ask(tid);
  const int free_count = d.free_count[0];
  int count = min(max(free_count, 0), d.free_cap);
  if (count != free_count) bits |= FOCUS_ERR_BOUNDS;
  for (int b0 = 0; b0 < d.batch; b0 += THREADS) {
    const int b = b0 + tid;
    if (b0 > 0) ask(b);
    group_scan<THREADS>(x, s_part, total);
    if (total[0] > 0) {
      s_upto[0][tid] = x[0], s_first[0][tid] = pages(left);
      __syncthreads();
      auto entry = [&](int k, int i) {
        const int before = k > 0 ? s_upto[0][k - 1] : 0;
        return d.table + (int64_t)(b0 + k) * d.max_pages + s_first[0][k] + (i - before);
      };
      each_page<THREADS>(s_upto[0], 0, total[0], [&](int k, int i) { return *entry(k, i); },
                         [&](int k, int i, int page) {
                           const int64_t to = (int64_t)count + i;
                           if (to < d.free_cap) d.free_pages[to] = page;
                           else bits |= FOCUS_ERR_CAPACITY;
                           *entry(k, i) = -1;
                         });
      count = (int)min((int64_t)count + total[0], (int64_t)d.free_cap);
    }
    if (b < d.batch && come == 0) d.length[b] = left, d.start[b] = left;
    if (!once || total[0] > 0) __syncthreads();
  }

  int rows = 0, needs = 0, taken = 0;  // of the sequences before; pages handed out
  for (int b0 = 0; b0 < d.batch; b0 += THREADS) {
    const int b = b0 + tid;
    if (!once) {
      int32_t told = bits;
      ask(b);
      bits = told;
      group_scan<THREADS>(x, s_part, total);
    }
    // Served while pages and maps last; both sums ascend, so those that get pages are the first
    // ones that need any.
    const int end = add_up(rows, x[2]), upto = needs + x[1];
    const bool lasts = end <= d.n_rows && upto <= count;
    const int need = pages(n + (room ? come : 0)) - pages(n);
    const bool served = come > 0 && room && end <= d.n_rows && (need == 0 || lasts);
    if (tid == 0) s_taken = needs;
    s_upto[1][tid] = upto, s_first[1][tid] = pages(n);
    s_end[tid] = end, s_start[tid] = come == 0 ? left : served ? n : -1;
    __syncthreads();
    const int last = focus::wave_max(lasts ? upto : 0);
    if (tid % 64 == 0) atomicMax(&s_taken, last);
    if (b < d.batch) {
      d.cu_rows[b + 1] = end;
      if (come > 0) {
        d.start[b] = served ? n : -1;
        d.length[b] = served ? n + come : n;
        if (!served) bits |= FOCUS_ERR_CAPACITY;
      }
    }
    __syncthreads();
    const int stop = s_taken;
    each_page<THREADS>(s_upto[1], needs, stop, [&](int, int i) { return d.free_pages[count - 1 - i]; },
                       [&](int k, int i, int page) {
                         const int before = k > 0 ? s_upto[1][k - 1] : needs;
                         d.table[(int64_t)(b0 + k) * d.max_pages + s_first[1][k] + (i - before)] = page;
                       });
    taken += stop - needs;
    rows = add_up(rows, total[2]), needs += total[1];
    if (!once) __syncthreads();
  }
  if (tid == 0) d.cu_rows[0] = 0, d.free_count[0] = count - taken;
  if (a.maps) {
    for (int t = tid; t < d.n_rows; t += THREADS) {
      if (t < rows) {
        const int b = first_above<THREADS>(s_end, t);
        write_row(d, t, b, s_start[b], t - (b > 0 ? s_end[b - 1] : 0));
      } else {
        write_row(d, t, -1, -1, 0);
      }
    }
  }
  if (bits) focus::raise_err(d.err, bits);
}

// A wave takes 64 rows: the first one's sequence by a search of 64 offsets at a time, the
// others' among the 64 sequences from there on, one a lane.
__global__ __launch_bounds__(kRowThreads) void extend_rows(Args a) {
  const focus_paged_extend_desc& d = a.d;
  const int64_t t64 = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
  const int lane = threadIdx.x % 64, t = (int)min(t64, d.n_rows - 1), t0 = (int)(t64 - lane);
  const int* ends = d.cu_rows + 1;
  int lo = 0, len = d.batch;
  while (len > 0) {
    const int step = (len + 63) / 64, last = lo + (lane + 1) * step - 1;  // of the lane's part
    const int parts = __popcll(__ballot(last < lo + len && ends[last] <= t0));
    lo += parts * step;
    len = min(step - 1, len - parts * step);
  }
  for (int b = lo;; b += 64) {
    const bool in = b + lane < d.batch;
    const int end = in ? ends[b + lane] : INT32_MAX, begin = d.cu_rows[min(b + lane, d.batch)];
    const int start = in ? d.start[b + lane] : -1;
    // this lane's sequence among them: those that end at its row or before come first
    int k = 0;
#pragma unroll
    for (int half = 32; half > 0; half /= 2) k += __shfl(end, k + half - 1) <= t ? half : 0;
    const bool here = __shfl(end, k) > t;
    const int from = __shfl(begin, k), to = __shfl(start, k);
    if (here && t >= from && t64 < d.n_rows) {
      if (b + k < d.batch) write_row(d, t, b + k, to, t - from);
      else write_row(d, t, -1, -1, 0);
    }
    // (a row before these sequences was written with the ones before)
    if (!__ballot(!here)) break;
  }
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

extern "C" focus_status focus_paged_extend(const focus_paged_extend_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  if (d->batch < 0 || d->max_pages < 0 || d->free_cap < 0 || d->n_rows < 0) return FOCUS_E_ARG;
  if (d->page_rows < 8 || d->page_rows > 1024 || (d->page_rows & (d->page_rows - 1))) return FOCUS_E_UNSUPPORTED;
  if ((int64_t)d->max_pages * d->page_rows > INT32_MAX / 2 || (int64_t)d->batch * d->max_pages >= INT32_MAX ||
      d->batch > INT32_MAX / 2 || d->n_rows >= INT32_MAX)
    return FOCUS_E_SHAPE;
  if (!d->cu_rows || !d->free_count || (d->free_cap > 0 && !d->free_pages)) return FOCUS_E_NULL;
  if (d->batch > 0 && (!d->length || !d->add || !d->start || (d->max_pages > 0 && !d->table))) return FOCUS_E_NULL;
  for (const void* p : {(const void*)d->table, (const void*)d->length, (const void*)d->add, (const void*)d->free_pages,
                        (const void*)d->free_count, (const void*)d->first_pos, (const void*)d->start,
                        (const void*)d->cu_rows, (const void*)d->row_seq, (const void*)d->row_slot,
                        (const void*)d->row_pos, (const void*)d->err})
    if (!aligned4(p)) return FOCUS_E_ARG;
  const int threads = d->batch <= kFew ? kFew : kMany;
  const bool any = d->n_rows > 0 && (d->row_seq || d->row_slot || d->row_pos);
  Args a = {*d, __builtin_ctz((unsigned)d->page_rows), any && d->batch <= threads && d->n_rows <= kMapRounds * threads};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (threads == kFew) hipLaunchKernelGGL(extend_tables<kFew>, dim3(1), dim3(kFew), 0, s, a);
  else hipLaunchKernelGGL(extend_tables<kMany>, dim3(1), dim3(kMany), 0, s, a);
  const focus_status st = focus::launch_status();
  if (st != FOCUS_OK || !any || a.maps) return st;
  hipLaunchKernelGGL(extend_rows, dim3((uint32_t)focus::ceil_div(d->n_rows, kRowThreads)), dim3(kRowThreads), 0, s, a);
  return focus::launch_status();
}
