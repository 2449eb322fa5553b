// Rows stored in a paged cache of 8 bits, a power of two as scale for each block of rows and
// KV head (focus_paged_append).
//
// One wave takes a block of a sequence and a KV head, of k and of v, whose new rows stay in its
// registers (of large blocks, what is past 8 KB of k and of v is read again through the caches):
// the largest magnitude gives the scale, the elements times its inverse are exact and
// rounded once.  Lanes take 16 neighbouring elements each (one 16-byte store).  Which blocks a
// wave takes follows from its rows: it covers a few consecutive ones and takes the blocks whose
// first new row is among them, so that no block has two writers, whatever the lengths of the
// sequences.
//
// HBM bound for many rows: 101 000 rows of 32 heads of 128 (bf16, 2.48 GB) take 445 us, 5.6
// TB/s (two bytes read for each written; this card copies at 5.0, one for one).  With the heads of
// a row far apart among the workgroups 492; with plain stores besides 514; reading the rows twice
// and dividing by the scale 760.  For few, a chain of latencies: one row of each of 64
// sequences 6.1 us (offsets and starts, page table, rows, stores).
#include "paged.h"

#include <algorithm>

namespace {

using focus::u32x4;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kResident = 20;        // workgroups of a compute unit that spans of fewer rows may make
constexpr float kLargest = 448.f;  // of e4m3
constexpr uint32_t kInf = 0x7f800000u;

struct Args {
  focus_paged_append_desc d;
  int shift, scale_shift;  // log2 page_rows, scale_rows
  int span_shift;          // log2 of the rows of a span
  int pieces;              // of 16 elements, in a row of a head
  uint32_t wide;           // waves or workgroups for the heads of a row
  uint32_t inv;            // 2^20 / pieces, rounded up (exact quotients of less than 2^16)
};

// The least e >= -126 with most <= 448 2^e, as the bits of 2^e; most finite.
__device__ inline uint32_t scale_bits(uint32_t most) {
  // most = 1.m 2^x, 448 = 1.75 2^8
  const int x = (int)(most >> 23) - 127, e = x - ((most & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return (uint32_t)(max(e, -126) + 127) << 23;
}

// 16 elements of T: as loaded, and as float32.
template <typename T> struct Piece {
  static constexpr int kLoads = sizeof(T);  // of 16 bytes
  u32x4 w[kLoads];
  __device__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + i * (16 / kLoads)));
  }
  __device__ float at(int k) const {
    if constexpr (sizeof(T) == 2) return k % 2 ? focus::bf16_hi(w[k / 8][k / 2 % 4]) : focus::bf16_lo(w[k / 8][k / 2 % 4]);
    else return __uint_as_float(w[k / 4][k % 4]);
  }
  // Greatest magnitude, as bits of a float32; FINITE: of the finite ones.
  template <bool FINITE> __device__ uint32_t most() const {
    uint32_t m = 0;
    if constexpr (sizeof(T) == 2 && !FINITE) {
      u16x2 x = {0, 0};
#pragma unroll
      for (int k = 0; k < 8; ++k)
        x = __builtin_elementwise_max(x, __builtin_bit_cast(u16x2, w[k / 4][k % 4] & 0x7fff7fffu));
      m = (uint32_t)max(x[0], x[1]) << 16;
    } else {
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const uint32_t x = __float_as_uint(at(k)) & 0x7fffffffu;
        m = max(m, FINITE && x >= kInf ? 0u : x);
      }
    }
    return m;
  }
};

// x times or over a scale, by the power of two that the scale is, or (a user's own) divided
// by it; numbers of at most 448, others NaN, to e4m3.
struct Scaler {
  float to, inv;
  bool exact, finite;
  __device__ float operator()(float x) const {
    x = exact ? x * inv : x / to;
    return finite || fabsf(x) <= kLargest ? x : __uint_as_float(0x7fc00000u);
  }
};
__device__ inline Scaler scaler(float to, bool finite) {
  // (2^e, -126 <= e <= 126, has a normal inverse)
  const uint32_t u = __float_as_uint(to);
  const bool exact = (u & 0x807fffffu) == 0 && u >= 0x00800000u && u <= 0x7e800000u;
  return {to, __uint_as_float(0x7f000000u - u), exact, finite};
}

__device__ inline u32x4 round16(const float (&x)[16]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
    r[i] = (uint32_t)w;
  }
  return r;
}
template <typename T> __device__ inline u32x4 round_piece(const Piece<T>& p, const Scaler& by) {
  float x[16];
  if (by.exact && by.finite) {
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = p.at(k) * by.inv;
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = by(p.at(k));
  }
  return round16(x);
}

// The sequence of row t, the first whose rows end behind it (b = batch if none does), its
// rows [r0, r1) and where they begin in it, by a wave: 64 offsets are looked at together.  (The
// last 64 with the starts beside them: one load's latency less.)
struct Owner {
  int b;
  int64_t r0, r1, start;
};
__device__ Owner owner_of(const focus_paged_append_desc& d, int64_t t) {
  const int batch = d.cache.kv.batch, lane = threadIdx.x % 64;
  if (!d.cu_rows) return {(int)t, t, t + 1, d.start[t]};
  int lo = 0, len = batch;
  while (len > 64) {
    const int step = (len + 63) / 64, at = lo + (lane + 1) * step - 1;  // the last of the lane's part
    const bool upto = at < lo + len && d.cu_rows[at + 1] <= t;
    const int parts = __popcll(__ballot(upto));
    lo += parts * step;
    len = min(step, len - parts * step);
  }
  const bool in = lane < len;
  const int end = in ? d.cu_rows[lo + lane + 1] : INT32_MAX, begin = in ? d.cu_rows[lo + lane] : 0;
  const int start = in ? d.start[lo + lane] : -1;
  const int k = __popcll(__ballot(in && end <= t));
  if (k >= len) return {batch, 0, 0, -1};
  return {lo + k, max(__builtin_amdgcn_readlane(begin, k), 0), min((int64_t)__builtin_amdgcn_readlane(end, k), d.n_rows),
          __builtin_amdgcn_readlane(start, k)};
}

// A block's new rows of one KV head, [t0, t0 + rows) at page + in_page on, of k or v, by GROUP
// threads, which keep HELD pieces each.
template <typename T, int HELD, int GROUP> struct Side {
  const Args& a;
  const T* src;
  int64_t step, to_step;
  uint8_t* dst;
  float* scale;
  int n;                // pieces
  Piece<T> piece[HELD];
  float was;

  __device__ Side(const Args& a, bool is_v, int64_t t0, int rows, int64_t page, int in_page, int g) : a(a) {
    const focus_paged_append_desc& d = a.d;
    const focus_paged_kv& c = d.cache.kv;
    step = is_v ? d.v_row : d.k_row, to_step = c.row_stride;
    src = reinterpret_cast<const T*>(is_v ? d.v : d.k) + t0 * step + g * (is_v ? d.v_head : d.k_head);
    dst = reinterpret_cast<uint8_t*>(is_v ? c.v : c.k) + page * c.page_stride + g * c.head_stride + in_page * to_step;
    scale = (is_v ? d.cache.v_scale : d.cache.k_scale) +
            (page * c.n_kv_heads + g) * (c.page_rows >> a.scale_shift) + (in_page >> a.scale_shift);
    n = rows * a.pieces;
  }
  __device__ static int thread() { return threadIdx.x % GROUP; }
  // Row and first element of piece i.
  __device__ int2 place(int i) const {
    const int r = (int)((uint32_t)i * a.inv >> 20);
    return make_int2(r, (i - r * a.pieces) * 16);
  }
  __device__ const T* from(int i) const {
    const int2 at = place(i);
    return src + at.x * step + at.y;
  }
  __device__ u32x4* to(int i) const {
    const int2 at = place(i);
    return reinterpret_cast<u32x4*>(dst + at.x * to_step + at.y);
  }
  __device__ void load(bool partly) {
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      const int i = thread() + GROUP * j;
#pragma unroll
      for (int k = 0; k < Piece<T>::kLoads; ++k) piece[j].w[k] = u32x4{0, 0, 0, 0};
      if (i < n) piece[j].load(from(i));
    }
    was = partly ? *scale : 0.f;
  }
  template <bool FINITE> __device__ uint32_t most(uint32_t* s_max) const {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < HELD; ++j) m = max(m, piece[j].template most<FINITE>());
    for (int i = thread() + GROUP * HELD; i < n; i += GROUP) {
      Piece<T> p;
      p.load(from(i));
      m = max(m, p.template most<FINITE>());
    }
    m = (uint32_t)focus::wave_max((int)m);
    if (GROUP > 64) {
      if (threadIdx.x % 64 == 0) s_max[threadIdx.x / 64] = m;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = max(m, s_max[w]);
    }
    return m;
  }
  // s_max: two sets of a value of each wave, used by nothing else until the next barrier but one.
  __device__ void store(int in_block, uint32_t* s_max) {
    uint32_t m = most<false>(s_max);
    const bool finite = m < kInf;
    if (!finite) m = most<true>(s_max + kWaves);
    float by = __uint_as_float(scale_bits(m));
    if (in_block > 0) {
      if (was >= by) {
        by = was;
      } else {
        // the rows before the new ones, from their scale to the greater one
        const float f = was / by;
        for (int i = thread(); i < in_block * a.pieces; i += GROUP) {
          const int2 at = place(i);
          u32x4* p = reinterpret_cast<u32x4*>(dst + (at.x - in_block) * to_step + at.y);
          const u32x4 w = *p;
          float x[16];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false);
            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
            x[4 * k] = lo[0] * f, x[4 * k + 1] = lo[1] * f, x[4 * k + 2] = hi[0] * f, x[4 * k + 3] = hi[1] * f;
          }
          *p = round16(x);
        }
      }
    }
    const Scaler scaled = scaler(by, finite);
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      const int i = thread() + GROUP * j;
      if (i < n) __builtin_nontemporal_store(round_piece(piece[j], scaled), to(i));
    }
    for (int i = thread() + GROUP * HELD; i < n; i += GROUP) {
      Piece<T> p;
      p.load(from(i));
      __builtin_nontemporal_store(round_piece(p, scaled), to(i));
    }
    if (thread() == 0) *scale = by;
  }
};

// more: the sequence has further rows behind these.
template <typename T, int HELD, int GROUP>
__device__ void store_block(const Args& a, int64_t t0, int rows, int b, int64_t slot, int g, bool more, uint32_t* s_max) {
  const focus_paged_append_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  const int64_t page = focus::page_of(c, b, (int)slot, a.shift);
  const bool reports = g == 0 && threadIdx.x % GROUP == 0;
  if (page < 0) {
    if (reports) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
    return;
  }
  const int in_block = (int)(slot & (d.cache.scale_rows - 1)), in_page = (int)(slot & (c.page_rows - 1));
  // (both in flight before either is looked at)
  Side<T, HELD, GROUP> k(a, false, t0, rows, page, in_page, g), v(a, true, t0, rows, page, in_page, g);
  k.load(in_block > 0), v.load(in_block > 0);
  k.store(in_block, s_max), v.store(in_block, s_max + 2 * kWaves);
  // The length is raised by the last block, or the last before one that is not stored.  (By all
  // of them: 81 600 rows of one head in 10 200 blocks 128 us, now 21.)
  if (reports) {
    const int64_t next = slot + rows;
    if (!more || next >= (int64_t)c.max_pages * c.page_rows ||
        ((next & (c.page_rows - 1)) == 0 && focus::page_of(c, b, (int)next, a.shift) < 0))
      atomicMax(&c.length[b], (int)next);
  }
}

// GROUP: threads of a block, those of a wave or of the workgroup.  HELD: pieces that a thread
// keeps of k, and of v.
template <typename T, int HELD, int GROUP>
__global__ __launch_bounds__(kThreads) void append_rows(Args a) {
  __shared__ uint32_t s_max[4 * kWaves];
  const focus_paged_append_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  // (neighbours take the heads of the same rows)
  const uint32_t id = GROUP == 64 ? blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : blockIdx.x;
  const uint32_t span = id / a.wide;
  const int g = (int)(id - span * a.wide);
  const bool reports = g == 0 && threadIdx.x % GROUP == 0;
  const int64_t cap = (int64_t)c.max_pages * c.page_rows, in_block = d.cache.scale_rows - 1;
  int64_t t = (int64_t)span << a.span_shift;
  const int64_t end = min(t + (int64_t{1} << a.span_shift), d.n_rows), first = t;
  if (d.cu_rows && t == 0 && reports && (d.cu_rows[0] < 0 || d.cu_rows[c.batch] > d.n_rows))
    focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
  while (t < end) {
    const Owner o = owner_of(d, t);
    if (o.b >= c.batch || o.r1 <= t) return;  // (offsets that do not ascend, too)
    if (t < o.r0 || o.start < 0) {            // rows before the first offset; not served
      t = t < o.r0 ? o.r0 : o.r1;
      continue;
    }
    // from the first block whose first new row is not before this span
    const int64_t to_slot = o.start - o.r0;
    if (t == first && t > o.r0) t = ((t + to_slot + in_block) & ~(int64_t)in_block) - to_slot;
    for (; t < end && t < o.r1; t = ((t + to_slot + in_block + 1) & ~(int64_t)in_block) - to_slot) {
      const int64_t slot = t + to_slot, stop = min(o.r1, ((slot + in_block + 1) & ~(int64_t)in_block) - to_slot);
      if (slot < cap) {
        store_block<T, HELD, GROUP>(a, t, (int)(stop - t), o.b, slot, g, stop < o.r1, s_max);
      } else if (reports) {
        focus::raise_err(d.err, FOCUS_ERR_CAPACITY);
      }
    }
    t = min(t, o.r1);
  }
}

template <typename T> focus_status launch(Args a, hipStream_t s) {
  const focus_paged_append_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  // A wave takes a block that fits its registers, of as many rows as sequences have on average;
  // the fewer it has to keep, the more waves run together.  A larger block takes a workgroup.
  constexpr int kMost = sizeof(T) == 2 ? 4 : 2;
  const int64_t rows = std::min<int64_t>(d.cache.scale_rows, focus::ceil_div(d.n_rows, c.batch));
  const int held = (int)focus::ceil_div(rows * a.pieces, 64);
  const int group = held <= kMost ? kWaves : 1;  // blocks of a workgroup
  const int64_t wide = c.n_kv_heads, most = (int64_t)group * kResident * focus::device_cus();
  // Rows of a span: one (most then find that their block is another's) as long as that makes
  // few of them, else up to as many as a block or a sequence has, on average: short sequences
  // in a span follow one another.  24 calls of 1 to 80 000 rows, workgroups of a compute unit up
  // to which spans are made shorter, geometric mean: 2 16.3 us, 5 16.1, 10 15.6, 20 15.6, 40
  // 15.7, 80 16.1.
  while (a.span_shift < a.scale_shift && (int64_t)c.batch << (a.span_shift + 1) <= d.n_rows &&
         focus::ceil_div(d.n_rows, int64_t{1} << a.span_shift) * wide > most)
    ++a.span_shift;
  // (more than a launch holds: a span of several blocks)
  auto workgroups = [&] { return focus::ceil_div(focus::ceil_div(d.n_rows, int64_t{1} << a.span_shift) * wide, group); };
  while (workgroups() > INT32_MAX / kThreads) ++a.span_shift;
  a.wide = (uint32_t)wide;
  const dim3 grid((uint32_t)workgroups());
  if (held == 1) hipLaunchKernelGGL((append_rows<T, 1, 64>), grid, dim3(kThreads), 0, s, a);
  else if (held == 2) hipLaunchKernelGGL((append_rows<T, 2, 64>), grid, dim3(kThreads), 0, s, a);
  else if (held <= kMost) hipLaunchKernelGGL((append_rows<T, kMost, 64>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((append_rows<T, kMost, kThreads>), grid, dim3(kThreads), 0, s, a);
  return focus::launch_status();
}

focus_status validate(const focus_paged_append_desc* d) {
  const focus_paged_kv& c = d->cache.kv;
  const focus_status st = focus::check_paged8(d->cache);
  if (st != FOCUS_OK) return st;
  const int64_t es = focus::elt_bytes(d->dtype);
  if (es == 0) return FOCUS_E_DTYPE;
  if (d->n_rows < 0) return FOCUS_E_ARG;
  if (d->n_rows > INT32_MAX || (!d->cu_rows && d->n_rows != c.batch)) return FOCUS_E_SHAPE;
  if (c.n_kv_heads > 65535) return FOCUS_E_SHAPE;
  if (c.batch == 0 || d->n_rows == 0) return FOCUS_OK;
  if (!d->start || !d->k || !d->v) return FOCUS_E_NULL;
  if (d->start == c.length) return FOCUS_E_ARG;  // raised while others read it
  for (const void* p : {(const void*)d->cu_rows, (const void*)d->start, (const void*)d->err})
    if (reinterpret_cast<uintptr_t>(p) & 3u) return FOCUS_E_ARG;
  if (!focus::aligned16(d->k) || !focus::aligned16(d->v)) return FOCUS_E_ARG;
  for (int64_t s : {d->k_row, d->k_head, d->v_row, d->v_head})
    if (s < 0 || !focus::pieces16(s, es)) return FOCUS_E_ARG;
  return FOCUS_OK;
}

}  // namespace

extern "C" focus_status focus_paged_append(const focus_paged_append_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  const focus_status st = validate(d);
  const focus_paged_kv& c = d->cache.kv;
  if (st != FOCUS_OK || c.batch == 0 || d->n_rows == 0) return st;
  Args a = {};
  a.d = *d;
  a.shift = focus::page_shift(c), a.scale_shift = __builtin_ctz((unsigned)d->cache.scale_rows);
  a.pieces = c.head_dim / 16, a.inv = ((1 << 20) + a.pieces - 1) / a.pieces;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return d->dtype == FOCUS_BF16 ? launch<__bf16>(a, s) : launch<float>(a, s);
}
