// A paged K/V cache cut down to a budget by accumulated weight (focus_paged_evict).
//
// The weight of the last row kept is found by a radix selection over an order-preserving
// integer of the weights, in digits of 11, 11 and 10 bits (8 for short tables): a histogram of a digit among
// the rows that share the digits above says in which bucket the row lies and how many of
// it are still wanted.  Then the rows above that weight and the first of those that equal
// it are written in order; a wave holds consecutive rows, so one prefix sum over the
// waves places them.
//
//   evict_select  tables of up to 32 768 rows: one workgroup per (sequence, KV head), the
//                 weights in registers throughout; where a head's rows are few, or heads
//                 enough to fill the device, it copies them as well
//   evict_part    longer tables: a workgroup per 8 192 rows or more, one launch a digit, each
//                 adding up the histograms of the digit before, and a last one that writes
//                 the rows kept; what a workgroup's rows add to the ones before it follows
//                 from the same histograms
//   evict_stream  longer tables of heads enough for half of the device: one workgroup each
//   evict_copy    the kept rows and their weights to the pages of `out`
//
// The copy is HBM bound, the selection bound by the latency of its passes: 16 x 8 heads of
// 10 000 rows cut to 5 000 take 145 us, 12 of them the selection; 8 heads of 131 072 rows
// cut to 32 768 take 84 us, 25 of them the selection.  The first form (one workgroup a head,
// four digits of eight bits, the weights read for each) took 180 and 394.
#include "paged.h"

#include <algorithm>

namespace {

constexpr int kCopy = 256;
constexpr int kCopies = 4;  // of a histogram in LDS, lane by lane: [bin][copy]

// A workgroup's threads, and the digits (the uppermost first) it takes a weight's integer in.
template <int THREADS, int BITS> struct Form {
  static constexpr int kThreads = THREADS, kWaves = THREADS / 64, kBins = 1 << BITS, kDigits = (31 + BITS) / BITS;
  static constexpr int kPer = kBins / THREADS;  // bins a thread sums
  static_assert(kPer >= 1 && kPer <= 2, "one or two bins a thread");
  static constexpr __host__ __device__ int shift(int i) { return i == kDigits - 1 ? 0 : 32 - BITS * (i + 1); }
  static constexpr __device__ uint32_t mask(int i) { return i == kDigits - 1 ? (1u << (32 - BITS * i)) - 1 : kBins - 1u; }
  // the digits above digit i
  static constexpr __device__ uint32_t above(int i) { return i == 0 ? 0u : 0xffffffffu << shift(i - 1); }
};
using Wide = Form<1024, 11>;
using Small = Form<256, 8>;

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
template <typename F> __device__ inline int scan(int x, int* waves, int* total) {
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int y = focus::wave_scan(x);
  __syncthreads();
  if (lane == 63) waves[wave] = y;
  __syncthreads();
  const int sums = focus::wave_scan(lane < F::kWaves ? waves[lane] : 0);
  *total = __builtin_amdgcn_readlane(sums, F::kWaves - 1);
  return (wave ? __builtin_amdgcn_readlane(sums, wave - 1) : 0) + y - x;
}

// Lanes below this one whose bit of mask is set.
__device__ inline int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// What a workgroup knows of one (sequence, KV head).
struct Head {
  int b, g, n;
  int old, recent, take;  // rows before the recent ones; recent ones; how many old ones stay
  const float* w;
  int32_t* keep;
};
__device__ Head head_of(const focus_paged_evict_desc& d, int bg, bool report) {
  const int K = d.cache.n_kv_heads;
  Head h;
  h.b = bg / K, h.g = bg % K;
  h.n = focus::paged_length(d.cache, h.b);
  int32_t bits = h.n != d.cache.length[h.b] ? FOCUS_ERR_CAPACITY : 0;
  const int m = kept_rows(d, h.b, h.n, &bits);
  if (report && bits && h.g == 0 && threadIdx.x == 0) focus::raise_err(d.err, bits);
  h.recent = min(d.recent, m), h.old = h.n - h.recent, h.take = m - h.recent;
  h.w = d.cache.weight + (int64_t)bg * d.cache.weight_rows;
  h.keep = d.keep + (int64_t)bg * d.keep_rows;
  return h;
}

// The rows of a workgroup in registers, as integers of their weights' order: `used` of NR
// registers a thread, wave w the rows from first + 64 used w, a register's 64 rows
// consecutive.  0, which is no weight's integer (that of -inf is 0x7fffff), past the rows
// that a choice is made of.
template <int NR>
__device__ void load_keys(const float* w, int64_t rows, int first, int used, float (&x)[NR], int& row0) {
  row0 = first + (int)(threadIdx.x / 64) * 64 * used + (int)(threadIdx.x % 64);
#pragma unroll
  for (int i = 0; i < NR; ++i) x[i] = i < used && row0 + 64 * i < rows ? w[row0 + 64 * i] : 0.f;
}
template <int NR>
__device__ void order_keys(const Head& h, const float (&x)[NR], int row0, int used, uint32_t (&key)[NR]) {
#pragma unroll
  for (int i = 0; i < NR; ++i) key[i] = i < used && row0 + 64 * i < h.old ? order_of(x[i]) : 0u;
}

// Histogram of a digit among the rows that share the digits above it, added to hist
// (cleared by the caller).  Bucket 0 of digit 0 also counts what is no row, and so does bucket
// 0 of each next digit where the digits above are 0: behind all rows, of which no choice
// wants more than there are.  Atomics on one address go one after another, and the first digit, mostly the
// exponent, has few buckets that are full: lanes add to four copies in turn.  16 x 8 heads
// of 10 000 rows, 64 of them kept, the whole call, with weights all different / all equal:
// one copy 23.9 / 46.9 us, four 21.3 / 26.2, eight 22.0 / 24.2; lanes that share a bucket
// counted at once where they are many, one copy, 24.8 / 27.5.
template <typename F, int NR>
__device__ void count_digit(const uint32_t (&key)[NR], int used, int digit, uint32_t prefix, int* hist) {
  const uint32_t mask = F::above(digit), dm = F::mask(digit);
  const int shift = F::shift(digit);
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    if (i < used && (key[i] & mask) == prefix)
      atomicAdd(&hist[(key[i] >> shift & dm) * kCopies + threadIdx.x % kCopies], 1);
  }
}

// Clears the copies of a histogram; sums those of a bin.
template <typename F> __device__ inline void clear_hist(int* hist) {
  for (int i = threadIdx.x; i < F::kBins * kCopies / 4; i += F::kThreads) reinterpret_cast<int4*>(hist)[i] = make_int4(0, 0, 0, 0);
}
__device__ inline int bin_sum(const int* hist, int bin) {
  int sum = 0;
#pragma unroll
  for (int i = 0; i < kCopies / 4; ++i) {
    const int4 x = reinterpret_cast<const int4*>(hist + bin * kCopies)[i];
    sum += (x.x + x.y) + (x.z + x.w);
  }
  return sum;
}

// How far the selection has come: the rows above `level` stay and `equal` of those that
// share the digits found so far; done: none of those are left over (equal 0).
struct Level {
  uint32_t level;
  int equal, done;
};

// The level with one more digit: the last of the rows wanted lies in `bucket`, of `count`
// rows, of which `wanted` are.  Where the whole bucket stays, no further digit is needed: its
// rows are the ones above a level, unless that would be one below 0: with digits of 8 bits
// the integers of -2^127 and less, -inf among them, begin with a digit of 0.
template <typename F> constexpr __host__ __device__ Level refined(Level x, int digit, int bucket, int wanted, int count) {
  x.level |= (uint32_t)bucket << F::shift(digit);
  x.equal = wanted;
  if (digit < F::kDigits - 1 && wanted == count && x.level != 0) {
    x.level -= 1;
    x.equal = 0, x.done = 1;
  }
  return x;
}
constexpr Level kAllLow = refined<Small>({0, 256, 0}, 0, 0, 256, 256);
static_assert(kAllLow.level == 0 && kAllLow.equal == 256 && !kAllLow.done, "no level is below 0");
static_assert(refined<Small>(kAllLow, 1, 0x7f, 256, 256).level == 0x7effff, "the rows of -inf, 0x7fffff");
static_assert(refined<Wide>({0, 9, 0}, 0, 3, 2, 2).level == 0x5fffff, "the rows of -2^127 and less");

// The bucket that holds the last of the `equal` greatest rows of a digit's histogram (with
// at least so many rows; c: this thread's bins, kBins - 1 - kPer tid downwards), in every
// thread: the level with that digit.
template <typename F>
__device__ int next_level(const int (&c)[F::kPer], int digit, int* waves, int* found, Level& x) {
  const int tid = threadIdx.x;
  int sum = 0;
#pragma unroll
  for (int i = 0; i < F::kPer; ++i) sum += c[i];
  int total, above = scan<F>(sum, waves, &total);
#pragma unroll
  for (int i = 0; i < F::kPer; ++i) {
    if (above < x.equal && above + c[i] >= x.equal)
      found[0] = F::kBins - 1 - (tid * F::kPer + i), found[1] = x.equal - above, found[2] = c[i];
    above += c[i];
  }
  __syncthreads();
  const int bucket = found[0];
  x = refined<F>(x, digit, bucket, found[1], found[2]);
  __syncthreads();
  return bucket;
}

// Write the rows above `level` (> 0) and, of those equal to it, the ones that number less
// than `equal`; before these rows come before_above above it and before_equal equal to it,
// both raised by what these rows, of all the waves, add.
template <typename F, int NR>
__device__ void write_rows(const Head& h, const uint32_t (&key)[NR], int used, int row0, uint32_t level, int equal, int& before_above,
                           int& before_equal, int (*waves)[2]) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  int above = 0, ties = 0;  // of this wave
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    if (i < used) {
      above += __popcll(__ballot(key[i] > level));
      ties += __popcll(__ballot(key[i] == level));
    }
  }
  if (threadIdx.x % 64 == 0) waves[wave][0] = above, waves[wave][1] = ties;
  __syncthreads();
  const int lane = threadIdx.x % 64;
  const int sum_above = focus::wave_scan(lane < F::kWaves ? waves[lane][0] : 0);
  const int sum_ties = focus::wave_scan(lane < F::kWaves ? waves[lane][1] : 0);
  above = before_above + (wave ? __builtin_amdgcn_readlane(sum_above, wave - 1) : 0);
  ties = before_equal + (wave ? __builtin_amdgcn_readlane(sum_ties, wave - 1) : 0);
  before_above += __builtin_amdgcn_readlane(sum_above, F::kWaves - 1);
  before_equal += __builtin_amdgcn_readlane(sum_ties, F::kWaves - 1);
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    if (i >= used) continue;
    const uint64_t up = __ballot(key[i] > level), tie = __ballot(key[i] == level);
    if (tie) {
      const int t = ties + lanes_below(tie);
      if (key[i] > level || (key[i] == level && t < equal)) h.keep[above + lanes_below(up) + min(t, equal)] = row0 + 64 * i;
      ties += __popcll(tie);
    } else if (key[i] > level) {
      h.keep[above + lanes_below(up) + min(ties, equal)] = row0 + 64 * i;
    }
    above += __popcll(up);
  }
}

// The recent rows, and -1 past the rows kept; by `groups` workgroups of which this is `at`.
template <typename F>
__device__ void write_rest(const focus_paged_evict_desc& d, const Head& h, int at, int groups) {
  const int step = groups * F::kThreads;
  for (int j = at * F::kThreads + threadIdx.x; j < h.recent; j += step) h.keep[h.take + j] = h.old + j;
  for (int64_t j = h.take + h.recent + at * F::kThreads + threadIdx.x; j < d.keep_rows; j += step) h.keep[j] = -1;
}

struct Copy {
  int in_shift, out_shift, pieces, es;  // log2 page rows; 16-byte pieces of a row; element bytes
  bool lengths;                         // whether evict_select sets them (no length is read and written)
};

template <bool STREAM>
__device__ inline focus::u32x4 load_row(const void* pool, int64_t piece) {
  const focus::u32x4* p = reinterpret_cast<const focus::u32x4*>(pool) + piece;
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  return *p;
}

// Copies the kept rows j0, j0 + step, ... of one head, a 16-byte piece of each by one thread,
// four of them in flight.  Rows that a decode step has just read may still be in the last-level
// cache: they are loaded past it only where there are more than it may hold (16 x 8 heads,
// 5 000 rows of 256 bytes: 151 us past it, 155 through it; 8 heads, 32 768 rows: 87, 82; uneven
// lengths count as the longest: 4 of up to 70 806 rows, 4 heads, 29 570 kept: 85, 68).
template <bool STREAM>
__device__ void copy_rows(const focus_paged_evict_desc& d, const Copy& y, int b, int g, int64_t j0, int64_t step,
                          int64_t end, int sub) {
  constexpr int kFlight = 4;
  const int K = d.cache.n_kv_heads;
  const int64_t bg = (int64_t)b * K + g;
  const int32_t* keep = d.keep + bg * d.keep_rows;
  for (; j0 < end; j0 += step * kFlight) {
    int r[kFlight];
    int64_t src[kFlight], dst[kFlight];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) r[i] = j0 + i * step < end ? keep[j0 + i * step] : -1;
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      src[i] = dst[i] = -1;
      if (r[i] < 0) continue;
      const int j = (int)(j0 + i * step);
      const int64_t sp = focus::page_of(d.cache, b, r[i], y.in_shift), dp = focus::page_of(d.out, b, j, y.out_shift);
      if (sp < 0 || dp < 0) {
        if (sub == 0) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
        continue;
      }
      src[i] = focus::row_at(d.cache, sp, r[i], g) * y.es / 16 + sub;
      dst[i] = focus::row_at(d.out, dp, j, g) * y.es / 16 + sub;
    }
    focus::u32x4 k[kFlight], v[kFlight];
    float w[kFlight];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      if (src[i] >= 0) {
        k[i] = load_row<STREAM>(d.cache.k, src[i]);
        v[i] = load_row<STREAM>(d.cache.v, src[i]);
      }
      if (sub == 0 && r[i] >= 0 && d.out.weight) w[i] = d.cache.weight[bg * d.cache.weight_rows + r[i]];
    }
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      if (src[i] >= 0) {
        __builtin_nontemporal_store(k[i], reinterpret_cast<focus::u32x4*>(d.out.k) + dst[i]);
        __builtin_nontemporal_store(v[i], reinterpret_cast<focus::u32x4*>(d.out.v) + dst[i]);
      }
      if (sub == 0 && r[i] >= 0 && d.out.weight) d.out.weight[bg * d.out.weight_rows + j0 + i * step] = w[i];
    }
  }
}

// out.length of sequence b, by one thread.
__device__ void set_length(const focus_paged_evict_desc& d, int b) {
  int32_t bits = 0;
  d.out.length[b] = kept_rows(d, b, focus::paged_length(d.cache, b), &bits);
}

template <typename F, int NR, bool COPY>
__global__ __launch_bounds__(F::kThreads) void evict_select(focus_paged_evict_desc d, Copy y) {
  __shared__ __align__(16) int hist[F::kBins * kCopies];
  __shared__ int waves[F::kWaves], found[3], parts[F::kWaves][2];
  // few weights are read at once, up to the table's end, before the length is known
  const int64_t cap = (int64_t)d.cache.max_pages * d.cache.page_rows;
  float w[NR];
  int row0;
  int used = NR;
  if constexpr (NR <= 4) load_keys<NR>(d.cache.weight + (int64_t)blockIdx.x * d.cache.weight_rows, cap, 0, used, w, row0);
  const Head h = head_of(d, blockIdx.x, true);
  if (h.take > 0) {
    uint32_t key[NR];
    if constexpr (NR > 4) {
      used = (h.old + F::kThreads - 1) / F::kThreads;  // all waves alike
      load_keys<NR>(h.w, h.old, 0, used, w, row0);
    }
    order_keys<NR>(h, w, row0, used, key);
    Level x = {0, h.take, 0};
    for (int digit = 0; digit < F::kDigits && !x.done; ++digit) {
      clear_hist<F>(hist);
      __syncthreads();
      count_digit<F, NR>(key, used, digit, x.level, hist);
      __syncthreads();
      int c[F::kPer];
#pragma unroll
      for (int i = 0; i < F::kPer; ++i) c[i] = bin_sum(hist, F::kBins - 1 - (F::kPer * (int)threadIdx.x + i));
      next_level<F>(c, digit, waves, found, x);
    }
    int above = 0, ties = 0;
    write_rows<F, NR>(h, key, used, row0, x.level, x.equal, above, ties, parts);
  }
  write_rest<F>(d, h, 0, 1);
  if constexpr (COPY) {
    if (y.lengths && h.g == 0 && threadIdx.x == 0) d.out.length[h.b] = h.take + h.recent;
    __syncthreads();  // the kept rows are this workgroup's own
    const int per = F::kThreads / y.pieces;
    if ((int)threadIdx.x < per * y.pieces)
      copy_rows<false>(d, y, h.b, h.g, threadIdx.x / y.pieces, per, h.take + h.recent, threadIdx.x % y.pieces);
  }
}

// Long tables of many heads: one workgroup per (sequence, KV head), which reads the weights
// again for each digit and to write the rows.
__global__ __launch_bounds__(Wide::kThreads) void evict_stream(focus_paged_evict_desc d) {
  using F = Wide;
  constexpr int NR = 16, kRows = NR * F::kThreads;
  __shared__ __align__(16) int hist[F::kBins * kCopies];
  __shared__ int waves[F::kWaves], found[3], parts[2][F::kWaves][2];
  const Head h = head_of(d, blockIdx.x, true);
  write_rest<F>(d, h, 0, 1);
  if (h.take == 0) return;
  uint32_t key[NR];
  int row0;
  auto load = [&](int first) {
    float w[NR];
    load_keys<NR>(h.w, h.old, first, NR, w, row0);
    order_keys<NR>(h, w, row0, NR, key);
  };
  Level x = {0, h.take, 0};
  for (int digit = 0; digit < F::kDigits && !x.done; ++digit) {
    clear_hist<F>(hist);
    __syncthreads();
    for (int first = 0; first < h.old; first += kRows) {
      load(first);
      count_digit<F, NR>(key, NR, digit, x.level, hist);
    }
    __syncthreads();
    int c[F::kPer];
#pragma unroll
    for (int i = 0; i < F::kPer; ++i) c[i] = bin_sum(hist, F::kBins - 1 - (F::kPer * (int)threadIdx.x + i));
    next_level<F>(c, digit, waves, found, x);
  }
  int above = 0, ties = 0;
  for (int first = 0, turn = 0; first < h.old; first += kRows, turn ^= 1) {
    load(first);
    // (a round's counts are read while the next one's are written)
    write_rows<F, NR>(h, key, NR, row0, x.level, x.equal, above, ties, parts[turn]);
  }
}

// The long form's workgroups.
constexpr int kThreads = Wide::kThreads, kWaves = Wide::kWaves, kBins = Wide::kBins, kDigits = Wide::kDigits, kPer = Wide::kPer;

// The long form's workspace: per head the level so far, per part the rows above it in the
// parts before, and the histograms [head][part][digit] (counts of at most 32 768 rows).
struct Long {
  Level* level;
  int* before;
  uint16_t* hist;
  int parts;
};

// Launch STEP adds up the histograms of digit STEP - 1 and counts digit STEP, or, the last,
// writes the rows kept.  A part is NR rows a thread.
template <int STEP, int NR>
__global__ __launch_bounds__(kThreads) void evict_part(focus_paged_evict_desc d, Long y) {
  __shared__ __align__(16) int hist[kBins * kCopies];
  __shared__ int waves[kWaves], found[3], pair[kWaves][2];
  const int bg = blockIdx.x / y.parts, part = blockIdx.x % y.parts, tid = threadIdx.x;
  const Head h = head_of(d, bg, STEP == 0 && part == 0);
  if (STEP == kDigits) write_rest<Wide>(d, h, part, y.parts);
  constexpr int kPart = NR * kThreads;
  const int live = (h.old + kPart - 1) / kPart;  // parts that hold rows
  if (h.take == 0 || part >= live) return;
  // a digit's histogram of a part, two bins a thread, the first thread's the last ones
  const int bin0 = kBins - kPer * (tid + 1);
  auto bins = [&](int p, int digit) {
    return reinterpret_cast<uint32_t*>(y.hist + (((int64_t)bg * y.parts + p) * kDigits + digit) * kBins + bin0);
  };
  Level x = {0, h.take, 0};
  int before = 0, before_equal = 0;
  if constexpr (STEP >= 2) {
    x = y.level[2 * bg + STEP % 2];
    before = y.before[(int64_t)bg * y.parts + part];
    if (x.done && STEP < kDigits) {
      if (part == 0 && tid == 0) y.level[2 * bg + (STEP + 1) % 2] = x;
      return;
    }
  }
  uint32_t key[NR];
  int row0;
  {
    float w[NR];
    load_keys<NR>(h.w, h.old, part * kPart, NR, w, row0);
    order_keys<NR>(h, w, row0, NR, key);
  }
  if constexpr (STEP >= 1) {
    if (!x.done) {
      constexpr int kFlight = 8;
      // of all parts, and of those before this one
      int lo = 0, hi = 0, lo_b = 0, hi_b = 0;
      for (int p0 = 0; p0 < live; p0 += kFlight) {
        uint32_t c[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) c[i] = p0 + i < live ? *bins(p0 + i, STEP - 1) : 0;
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
          lo += c[i] & 0xffff, hi += c[i] >> 16;
          if (p0 + i < part) lo_b += c[i] & 0xffff, hi_b += c[i] >> 16;
        }
      }
      const int c[kPer] = {hi, lo};
      const int bucket = next_level<Wide>(c, STEP - 1, waves, found, x);
      const int own = bin0 == bucket ? lo_b : bin0 + 1 == bucket ? hi_b : 0;
      const int up = (bin0 > bucket ? lo_b : 0) + (bin0 + 1 > bucket ? hi_b : 0);
      int total;
      scan<Wide>(up + (x.done ? own : 0), waves, &total);
      before += total;
      if constexpr (STEP == kDigits) {
        scan<Wide>(own, waves, &total);
        before_equal = total;
      } else if (tid == 0) {
        y.before[(int64_t)bg * y.parts + part] = before;
        if (part == 0) y.level[2 * bg + (STEP + 1) % 2] = x;
      }
    }
  }
  if constexpr (STEP == kDigits) {
    write_rows<Wide, NR>(h, key, NR, row0, x.level, x.equal, before, before_equal, pair);
  } else {
    if (x.done) return;
    clear_hist<Wide>(hist);
    __syncthreads();
    count_digit<Wide, NR>(key, NR, STEP, x.level, hist);
    __syncthreads();
    *bins(part, STEP) = (uint32_t)bin_sum(hist, bin0) | (uint32_t)bin_sum(hist, bin0 + 1) << 16;
  }
}

// Neighbouring KV heads that a workgroup of evict_copy takes: their rows lie side by side
// where they go.
inline __host__ __device__ int heads_together(int n_kv_heads) {
  return n_kv_heads % 4 == 0 ? 4 : n_kv_heads % 2 == 0 ? 2 : 1;
}

template <bool STREAM>
__global__ __launch_bounds__(kCopy) void evict_copy(focus_paged_evict_desc d, Copy y) {
  // (the heads' order turns with the rows: those of one sequence would all lie on the same
  // XCDs otherwise)
  const int K = d.cache.n_kv_heads, wide = heads_together(K), item = (blockIdx.x + blockIdx.y) % gridDim.x;
  const int b = item / (K / wide), g0 = item % (K / wide) * wide;
  const int at = threadIdx.x / y.pieces, per = kCopy / (y.pieces * wide);
  if (at < per * wide)
    copy_rows<STREAM>(d, y, b, g0 + at % wide, (int64_t)blockIdx.y * per + at / wide, (int64_t)gridDim.y * per, d.keep_rows,
              threadIdx.x % y.pieces);
  if (blockIdx.y == 0 && g0 == 0 && threadIdx.x == 0) set_length(d, b);
}

__global__ __launch_bounds__(kCopy) void evict_lengths(focus_paged_evict_desc d) {
  const int b = blockIdx.x * kCopy + threadIdx.x;
  if (b < d.cache.batch) set_length(d, b);
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

// Whether two arrays of 4-byte elements have any in common.
bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y ? y - x < (uint64_t)na * 4 : x - y < (uint64_t)nb * 4;
}
int64_t weights_of(const focus_paged_kv& c) { return (int64_t)c.batch * c.n_kv_heads * c.weight_rows; }

// Rows of a table that one workgroup selects from by itself.
constexpr int64_t kShortRows = 32 * kThreads;

// Workgroups a head of the long form; 0 where it is not taken: for short tables, and for
// heads enough for half of the compute units, of which one workgroup each goes through the
// weights (evict_stream) in less time than several pass histograms on.  us, the whole call,
// by parts / by heads, 40 000 rows: 64 heads 46 / 50, 128 69 / 62, 512 247 / 178; 131 072
// rows: 32 heads 48 / 92, 64 71 / 104, 256 183 / 121.
int64_t parts_of(const focus_paged_evict_desc& d, int* rows) {
  const int64_t cap = (int64_t)d.cache.max_pages * d.cache.page_rows, heads = (int64_t)d.cache.batch * d.cache.n_kv_heads;
  if (cap <= kShortRows || heads >= focus::device_cus() / 2) return 0;
  // Rows a thread holds: every workgroup adds up the histograms of all parts of its head, so
  // that few large parts are better as soon as small ones would go around the device more
  // than once, or are more than 32 a head.  8 / 16 / 32, us of the whole call: 8 heads of
  // 131 072 rows 31.6 / 33.8 / 44.4, 32 of them 51 / 47 / 56, 64 of them 90 / 78 / 72; 8 heads
  // of 400 000 rows 52 / 40 / 45, of a million 132 / 70 / 56, one of a million 51 / 43 / 47.
  const int64_t parts = focus::ceil_div(cap, 8 * kThreads), groups = heads * parts, cus = focus::device_cus();
  *rows = groups <= cus && parts <= 32 ? 8 : groups <= 3 * cus ? 16 : 32;
  return focus::ceil_div(cap, *rows * kThreads);
}

// The long form's arrays in the workspace (out may be NULL); returns their bytes.  Two
// levels a head: a launch reads one that its first part's workgroup does not write.
size_t long_form(const focus_paged_evict_desc& d, void* workspace, Long* out) {
  int rows;
  const int64_t parts = parts_of(d, &rows), heads = (int64_t)d.cache.batch * d.cache.n_kv_heads;
  if (parts == 0) return 0;
  const int64_t level = focus::ceil_div(2 * heads * (int64_t)sizeof(Level), 16) * 16;
  const int64_t before = focus::ceil_div(heads * parts * 4, 16) * 16;
  if (out) {
    char* ws = reinterpret_cast<char*>(workspace);
    *out = {reinterpret_cast<Level*>(ws), reinterpret_cast<int*>(ws + level),
            reinterpret_cast<uint16_t*>(ws + level + before), (int)parts};
  }
  return (size_t)(level + before + heads * parts * kDigits * kBins * 2);
}

}  // namespace

extern "C" size_t focus_paged_evict_workspace(const focus_paged_evict_desc* d) {
  if (!d || validate(d) != FOCUS_OK) return 0;
  return long_form(*d, nullptr, nullptr);
}

extern "C" focus_status focus_paged_evict(const focus_paged_evict_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  focus_status st = validate(d);
  if (st != FOCUS_OK) return st;
  if (d->cache.batch == 0) return FOCUS_OK;
  if (!d->cache.weight || (d->keep_rows > 0 && !d->keep)) return FOCUS_E_NULL;
  if ((reinterpret_cast<uintptr_t>(d->keep) & 3u) || (reinterpret_cast<uintptr_t>(d->budgets) & 3u)) return FOCUS_E_ARG;
  int rows = 0;
  const int64_t parts = parts_of(*d, &rows), heads = (int64_t)d->cache.batch * d->cache.n_kv_heads;
  const size_t need = focus_paged_evict_workspace(d);
  if (need > 0 && (!d->workspace || d->workspace_bytes < need)) return FOCUS_E_WORKSPACE;
  if (!focus::aligned16(d->workspace)) return FOCUS_E_ARG;
  // (out.length may be cache.length or budgets, which every head's workgroup reads: it is
  // set by a later launch then, one entry by the thread that read it)
  const bool over_length = overlap(d->out.length, d->cache.batch, d->cache.length, d->cache.batch);
  const bool over_budgets = d->budgets && overlap(d->out.length, d->cache.batch, d->budgets, d->cache.batch);
  if ((over_length && d->out.length != d->cache.length) || (over_budgets && d->out.length != d->budgets) ||
      (d->out.weight && overlap(d->out.weight, weights_of(d->out), d->cache.weight, weights_of(d->cache))))
    return FOCUS_E_ARG;
  // one table of one pool: rows would be copied over others that are still to be copied
  if (d->out.table == d->cache.table && d->out.max_pages > 0 && (d->out.k == d->cache.k || d->out.v == d->cache.v))
    return FOCUS_E_ARG;
  if (heads * std::max<int64_t>(parts, 1) > INT32_MAX / kThreads) return FOCUS_E_SHAPE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int es = (int)focus::elt_bytes(d->cache.dtype), pieces = d->cache.head_dim * es / 16;
  const Copy y = {focus::page_shift(d->cache), focus::page_shift(d->out), pieces, es, !over_length && !over_budgets};
  const dim3 block(kThreads);
  const int64_t cap = (int64_t)d->cache.max_pages * d->cache.page_rows;
  if (parts > 0) {
    const dim3 grid((uint32_t)(heads * parts));
    Long scratch;
    long_form(*d, d->workspace, &scratch);
#define FOCUS_PARTS(NR)                                                      \
  hipLaunchKernelGGL((evict_part<0, NR>), grid, block, 0, s, *d, scratch);   \
  hipLaunchKernelGGL((evict_part<1, NR>), grid, block, 0, s, *d, scratch);   \
  hipLaunchKernelGGL((evict_part<2, NR>), grid, block, 0, s, *d, scratch);   \
  hipLaunchKernelGGL((evict_part<3, NR>), grid, block, 0, s, *d, scratch);
    if (rows == 8) { FOCUS_PARTS(8) } else if (rows == 16) { FOCUS_PARTS(16) } else { FOCUS_PARTS(32) }
#undef FOCUS_PARTS
  } else if (cap > kShortRows) {
    hipLaunchKernelGGL(evict_stream, dim3((uint32_t)heads), block, 0, s, *d);
  } else {
    // A workgroup copies its own head's rows where that is little work, somewhat more where
    // there are heads for every compute unit: a launch less, but a long sequence's rows
    // are copied by one compute unit.  64 x 8 heads, 2 000 rows kept of 4 000 (2 MB a head
    // read and written): 238 us by the heads' own workgroups, 244 by a launch of its own, of
    // uneven lengths 86 and 69; 32 x 32 heads, 500 rows kept of 1 000 (0.5 MB): 131 and 146.
    const int64_t bytes = d->keep_rows * pieces * 64;
    const bool copies = bytes <= (256 << 10) || (bytes <= (512 << 10) && heads >= 2 * focus::device_cus());
    const dim3 grid((uint32_t)heads);
#define FOCUS_SELECT(F, NR)                                                                            \
  if (copies) hipLaunchKernelGGL((evict_select<F, NR, true>), grid, dim3(F::kThreads), 0, s, *d, y);  \
  else hipLaunchKernelGGL((evict_select<F, NR, false>), grid, dim3(F::kThreads), 0, s, *d, y);
    // More heads than compute units go through several of them at a time, by workgroups of
    // 256 threads, whose passes cost less: 1024 x 8 heads of 300 rows, 100 kept, 186 us,
    // with 1024 threads 321; 64 x 8 of 1000, 250 kept, 27 and 34; 512 x 4 of 4000, 200 kept,
    // 53 and 77.  Fewer heads have a compute unit each, and its threads copy as well: 16 x 8
    // of 900, 256 kept, 16.9 and 14.5.
    const bool small = heads > focus::device_cus();
    if (small && cap <= 4 * Small::kThreads) { FOCUS_SELECT(Small, 4) }
    else if (small && cap <= 16 * Small::kThreads) { FOCUS_SELECT(Small, 16) }
    else if (cap <= 4 * Wide::kThreads) { FOCUS_SELECT(Wide, 4) }
    else if (cap <= 16 * Wide::kThreads) { FOCUS_SELECT(Wide, 16) }
    else { FOCUS_SELECT(Wide, 32) }
#undef FOCUS_SELECT
    if (copies) {
      if ((st = focus::launch_status()) != FOCUS_OK || y.lengths) return st;
      hipLaunchKernelGGL(evict_lengths, dim3((uint32_t)focus::ceil_div(d->cache.batch, kCopy)), dim3(kCopy), 0, s, *d);
      return focus::launch_status();
    }
  }
  if ((st = focus::launch_status()) != FOCUS_OK) return st;
  // four rows of a head and thread in flight, one round of them where the grid allows
  const int wide = heads_together(d->cache.n_kv_heads);
  const int64_t blocks = focus::ceil_div(std::max<int64_t>(d->keep_rows, 1), kCopy / (pieces * wide) * 4);
  const dim3 grid((uint32_t)(heads / wide), (uint32_t)std::min<int64_t>(blocks, 4096));
  if ((double)heads * d->keep_rows * pieces * 64 > 512 << 20)
    hipLaunchKernelGGL((evict_copy<true>), grid, dim3(kCopy), 0, s, *d, y);
  else
    hipLaunchKernelGGL((evict_copy<false>), grid, dim3(kCopy), 0, s, *d, y);
  return focus::launch_status();
}
