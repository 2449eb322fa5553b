// Rows stored in a paged cache of 8 bits, a power of two as scale for each block of rows and
// KV head (focus_paged_append).
//
// One wave takes a block of a sequence and a KV head, of k and of v (of larger blocks one of
// them, or a workgroup does), whose new rows stay in its registers: the largest magnitude gives
// the scale, the elements times its inverse are exact and rounded once.  Lanes take 32
// neighbouring bytes each: two loads, one store.  (100 000 float32 rows of 8 heads by 64 / 32 / 16
// bytes 270 / 198 / 195 us; 101 000 bf16 rows of 32 by 32 / 16 448 / 464.)  Which blocks a wave takes
// follows from its rows: it covers a few consecutive ones and takes the blocks whose first new
// row is among them, so that no block has two writers, whatever the lengths of the sequences.
//
// HBM bound for many rows: 101 000 rows of 32 heads of 128 (bf16, 2.48 GB) take 445 us, 5.6
// TB/s (two bytes read for each written; this card copies at 5.0, one for one).  With the heads of
// a row far apart among the workgroups 492; with plain stores besides 514; reading the rows twice
// and dividing by the scale 760.  For few, a chain of latencies: one row of each of 64
// sequences 6.1 us (offsets and starts, page table, rows, stores).
#include "paged.h"

#include <algorithm>
#include <type_traits>

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
  int pieces;              // in a row of a head
  uint32_t wide;           // waves or workgroups for the heads of a row
  uint32_t inv;            // 2^20 / pieces, rounded up (exact quotients of up to 1 024 rows of 32 pieces)
};

// The least e >= -126 with most <= 448 2^e, as the bits of 2^e; most finite.
__device__ inline uint32_t scale_bits(uint32_t most) {
  // most = 1.m 2^x, 448 = 1.75 2^8
  const int x = (int)(most >> 23) - 127, e = x - ((most & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return (uint32_t)(max(e, -126) + 127) << 23;
}

// Neighbouring elements that a lane takes together, 32 bytes of T: as loaded, and as float32.
template <typename T> struct Piece {
  static constexpr int kElts = 32 / sizeof(T), kLoads = 2;
  u32x4 w[kLoads];
  __device__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + i * (kElts / kLoads)));
  }
  __device__ void clear() {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) w[i] = u32x4{0, 0, 0, 0};
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
      for (int k = 0; k < kElts / 2; ++k)
        x = __builtin_elementwise_max(x, __builtin_bit_cast(u16x2, w[k / 4][k % 4] & 0x7fff7fffu));
      m = (uint32_t)max(x[0], x[1]) << 16;
    } else {
#pragma unroll
      for (int k = 0; k < kElts; ++k) {
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

__device__ inline uint32_t round4(float x0, float x1, float x2, float x3) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, w, true);
}
// A piece's elements in 8 bits, as they are stored.
template <typename T> struct Narrow {
  static constexpr int kWords = Piece<T>::kElts / 4;
  typedef uint32_t W __attribute__((ext_vector_type(kWords)));
  W w;
  __device__ Narrow(const Piece<T>& p, const Scaler& by) {
    float x[4 * kWords];
    if (by.exact && by.finite) {
#pragma unroll
      for (int k = 0; k < 4 * kWords; ++k) x[k] = p.at(k) * by.inv;
    } else {
#pragma unroll
      for (int k = 0; k < 4 * kWords; ++k) x[k] = by(p.at(k));
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = round4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
  // Numbers that are stored, times f.
  __device__ Narrow(W old, float f) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)old[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)old[i], true);
      w[i] = round4(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
    }
  }
};

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
    return make_int2(r, (i - r * a.pieces) * Piece<T>::kElts);
  }
  __device__ const T* from(int i) const {
    const int2 at = place(i);
    return src + at.x * step + at.y;
  }
  __device__ typename Narrow<T>::W* to(int i) const {
    const int2 at = place(i);
    return reinterpret_cast<typename Narrow<T>::W*>(dst + at.x * to_step + at.y);
  }
  __device__ void load(bool partly) {
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      const int i = thread() + GROUP * j;
      piece[j].clear();
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
  // s_max: two sets of a value of each wave, used by nothing else until the caller's barrier.
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
          auto* p = reinterpret_cast<typename Narrow<T>::W*>(dst + (at.x - in_block) * to_step + at.y);
          *p = Narrow<T>(*p, f).w;
        }
      }
    }
    const Scaler scaled = scaler(by, finite);
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
      const int i = thread() + GROUP * j;
      if (i < n) __builtin_nontemporal_store(Narrow<T>(piece[j], scaled).w, to(i));
    }
    for (int i = thread() + GROUP * HELD; i < n; i += GROUP) {
      Piece<T> p;
      p.load(from(i));
      __builtin_nontemporal_store(Narrow<T>(p, scaled).w, to(i));
    }
    if (thread() == 0) *scale = by;
  }
};

// more: the sequence has further rows behind these.
template <typename T, int HELD, int GROUP, int SIDES>
__device__ void store_block(const Args& a, int64_t t0, int rows, int b, int64_t slot, int g, int side, bool more, uint32_t* s_max) {
  const focus_paged_append_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  const int64_t page = focus::page_of(c, b, (int)slot, a.shift);
  const bool reports = g == 0 && side == 0 && threadIdx.x % GROUP == 0;
  if (page < 0) {
    if (reports) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
    return;
  }
  const int in_block = (int)(slot & (d.cache.scale_rows - 1)), in_page = (int)(slot & (c.page_rows - 1));
  if constexpr (SIDES == 2) {
    static_assert(GROUP == 64, "waves share s_max");
    // (both in flight before either is looked at)
    Side<T, HELD, GROUP> k(a, false, t0, rows, page, in_page, g), v(a, true, t0, rows, page, in_page, g);
    k.load(in_block > 0), v.load(in_block > 0);
    k.store(in_block, s_max), v.store(in_block, s_max);
  } else {
    Side<T, HELD, GROUP> x(a, side, t0, rows, page, in_page, g);
    x.load(in_block > 0);
    x.store(in_block, s_max);
    if (GROUP > 64) __syncthreads();
  }
  // The length is raised by the last block, or the last before one that is not stored.  (By all
  // of them: 81 600 rows of one head in 10 200 blocks 128 us, now 21.)
  if (reports) {
    const int64_t next = slot + rows;
    if (!more || next >= (int64_t)c.max_pages * c.page_rows ||
        ((next & (c.page_rows - 1)) == 0 && focus::page_of(c, b, (int)next, a.shift) < 0))
      atomicMax(&c.length[b], (int)next);
  }
}

// GROUP: threads of a block, those of a wave or of the workgroup, which take SIDES of k and v.
// HELD: pieces that a thread keeps of k, and of v.
template <typename T, int HELD, int GROUP, int SIDES>
__global__ __launch_bounds__(kThreads) void append_rows(Args a) {
  __shared__ uint32_t s_max[2 * kWaves];
  const focus_paged_append_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  // (neighbours take the heads of the same rows)
  const uint32_t id = GROUP == 64 ? blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : blockIdx.x;
  const uint32_t span = id / a.wide;
  const int among = (int)(id - span * a.wide), side = SIDES == 1 && among >= c.n_kv_heads;
  const int g = side ? among - c.n_kv_heads : among;
  const bool reports = g == 0 && side == 0 && threadIdx.x % GROUP == 0;
  const int64_t cap = (int64_t)c.max_pages * c.page_rows, in_block = d.cache.scale_rows - 1;
  int64_t t = (int64_t)span << a.span_shift;
  const int64_t end = min(t + (int64_t{1} << a.span_shift), d.n_rows), first = t;
  while (t < end) {
    const Owner o = owner_of(d, t);
    if (o.b >= c.batch || o.r1 <= t) break;  // (offsets that do not ascend, too)
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
        store_block<T, HELD, GROUP, SIDES>(a, t, (int)(stop - t), o.b, slot, g, side, stop < o.r1, s_max);
      } else if (reports) {
        focus::raise_err(d.err, FOCUS_ERR_CAPACITY);
      }
    }
    t = min(t, o.r1);
  }
  // All offsets are looked at, a few by each span.  (Behind its rows: held from before them, the
  // two numbers left blocks of 8 pieces a lane one wave a SIMD less, 126 us for 121.)
  const int64_t spans = ((d.n_rows - 1) >> a.span_shift) + 1;
  if (!d.cu_rows || g != 0 || side != 0 || span >= spans) return;
  for (int64_t b = (int64_t)span * GROUP + threadIdx.x % GROUP; b < c.batch; b += spans * GROUP) {
    const int from = d.cu_rows[b], to = d.cu_rows[b + 1];
    if (from < 0 || to < from || to > d.n_rows) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
  }
}

template <typename T> focus_status launch(Args a, hipStream_t s) {
  const focus_paged_append_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  // The fewer pieces a lane has to keep, the more waves run together; blocks have as many rows as
  // sequences have on average, at most.  A wave takes k and v of a block together up to 4 pieces (8
  // KB of each), one of them up to 8; larger blocks take a workgroup for each, which keeps 128 KB
  // (what is past that is read again).  100 000 rows of 8 heads of 128 so, and in brackets k and
  // v together by a workgroup of 4 pieces: blocks of 64 119 us (143), of 256 134 (184); of float32
  // 213 (289) and 274 (500).
  constexpr int kBoth = 4, kMost = 8;
  const int64_t rows = std::min<int64_t>(d.cache.scale_rows, focus::ceil_div(d.n_rows, c.batch));
  const int held = (int)focus::ceil_div(rows * a.pieces, 64);
  const int group = held <= kMost ? kWaves : 1;  // waves of a workgroup that take blocks of their own
  const int64_t wide = c.n_kv_heads * (held <= kBoth ? 1 : 2), most = (int64_t)group * kResident * focus::device_cus();
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
  auto append = [&](auto held, auto group, auto sides) {
    hipLaunchKernelGGL((append_rows<T, decltype(held)::value, decltype(group)::value, decltype(sides)::value>), grid,
                       dim3(kThreads), 0, s, a);
  };
  using std::integral_constant;
  constexpr integral_constant<int, 64> wave;
  constexpr integral_constant<int, kThreads> workgroup;
  constexpr integral_constant<int, 1> one;
  constexpr integral_constant<int, 2> two;
  constexpr integral_constant<int, 4> four;
  constexpr integral_constant<int, 8> eight;
  if (held == 1) append(one, wave, two);
  else if (held == 2) append(two, wave, two);
  else if (held <= kBoth) append(four, wave, two);
  else if (held <= kMost) append(eight, wave, one);
  else if (held <= kWaves * 4) append(four, workgroup, one);
  else if (held <= kWaves * 8) append(eight, workgroup, one);
  else append(integral_constant<int, 16>(), workgroup, one);
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
  a.pieces = c.head_dim / (d->dtype == FOCUS_BF16 ? Piece<__bf16>::kElts : Piece<float>::kElts);
  a.inv = ((1 << 20) + a.pieces - 1) / a.pieces;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return d->dtype == FOCUS_BF16 ? launch<__bf16>(a, s) : launch<float>(a, s);
}
