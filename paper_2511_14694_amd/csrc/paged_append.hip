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
// HBM bound for many rows: 101 000 rows of 32 heads of 128 (bf16, 2.48 GB) take 492 us, 5.0
// TB/s, as fast as this card copies; with plain stores 514, reading the rows twice and dividing
// by the scale 760.  For few, a chain of latencies: one row of each of 64 sequences 6.5 us
// (offsets and starts, page table, rows, stores).
#include "paged.h"

namespace {

using focus::u32x4;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kResident = 5;         // workgroups of a compute unit that waves of fewer rows may make
constexpr float kLargest = 448.f;  // of e4m3
constexpr uint32_t kInf = 0x7f800000u;

struct Args {
  focus_paged_append_desc d;
  int shift, scale_shift;  // log2 page_rows, scale_rows
  int span_shift;          // log2 of the rows a wave covers
  int pieces;              // of 16 elements, in a row of a head
  uint32_t wide;           // workgroups for the heads of a row
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

// A block's new rows of one KV head, of k or v: rows [t0, t0 + rows) at page + in_page on.
template <typename T> struct Side {
  static constexpr int kHeld = sizeof(T) == 2 ? 4 : 2;  // pieces that a lane keeps
  const T* src;
  int64_t step, to_step;
  uint8_t* dst;
  float* scale;
  Piece<T> held[kHeld];
  float was;

  __device__ Side(const Args& a, bool is_v, int64_t t0, int64_t page, int in_page, int g) {
    const focus_paged_append_desc& d = a.d;
    const focus_paged_kv& c = d.cache.kv;
    step = is_v ? d.v_row : d.k_row, to_step = c.row_stride;
    src = reinterpret_cast<const T*>(is_v ? d.v : d.k) + t0 * step + (int64_t)g * (is_v ? d.v_head : d.k_head);
    dst = reinterpret_cast<uint8_t*>(is_v ? c.v : c.k) + page * c.page_stride + (int64_t)g * c.head_stride +
          in_page * to_step;
    scale = (is_v ? d.cache.v_scale : d.cache.k_scale) +
            (page * c.n_kv_heads + g) * (c.page_rows >> a.scale_shift) + (in_page >> a.scale_shift);
  }
  // Row and first element of piece i.
  __device__ static int2 place(const Args& a, int i) {
    const int r = (int)((uint32_t)i * a.inv >> 20);
    return make_int2(r, (i - r * a.pieces) * 16);
  }
  __device__ void load(const Args& a, int n, bool partly) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = threadIdx.x % 64 + 64 * j;
      if (i < n) {
        const int2 at = place(a, i);
        held[j].load(src + at.x * step + at.y);
      } else {
#pragma unroll
        for (int k = 0; k < Piece<T>::kLoads; ++k) held[j].w[k] = u32x4{0, 0, 0, 0};
      }
    }
    was = partly ? *scale : 0.f;
  }
  template <bool FINITE> __device__ uint32_t most(const Args& a, int n) const {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) m = max(m, held[j].template most<FINITE>());
    for (int i = threadIdx.x % 64 + 64 * kHeld; i < n; i += 64) {
      const int2 at = place(a, i);
      Piece<T> p;
      p.load(src + at.x * step + at.y);
      m = max(m, p.template most<FINITE>());
    }
    return (uint32_t)focus::wave_max((int)m);
  }
  __device__ void store(const Args& a, int n, int in_block) {
    const int lane = threadIdx.x % 64;
    uint32_t m = most<false>(a, n);
    const bool finite = m < kInf;
    if (!finite) m = most<true>(a, n);
    float to = __uint_as_float(scale_bits(m));
    if (in_block > 0) {
      if (was >= to) {
        to = was;
      } else {
        // (of powers of two, as it is but for the first append to a user's own scales)
        const float f = was / to;
        uint8_t* old = dst - in_block * to_step;
        for (int i = lane; i < in_block * a.pieces; i += 64) {
          const int2 at = place(a, i);
          u32x4* p = reinterpret_cast<u32x4*>(old + at.x * to_step + at.y);
          const u32x4 w = *p;
          float x[16];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
            x[4 * k] = lo[0] * f, x[4 * k + 1] = lo[1] * f, x[4 * k + 2] = hi[0] * f, x[4 * k + 3] = hi[1] * f;
          }
          *p = round16(x);
        }
      }
    }
    const Scaler by = scaler(to, finite);
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = lane + 64 * j;
      if (i < n) {
        const int2 at = place(a, i);
        __builtin_nontemporal_store(round_piece(held[j], by), reinterpret_cast<u32x4*>(dst + at.x * to_step + at.y));
      }
    }
    for (int i = lane + 64 * kHeld; i < n; i += 64) {
      const int2 at = place(a, i);
      Piece<T> p;
      p.load(src + at.x * step + at.y);
      __builtin_nontemporal_store(round_piece(p, by), reinterpret_cast<u32x4*>(dst + at.x * to_step + at.y));
    }
    if (lane == 0) *scale = to;
  }
};

template <typename T>
__device__ void store_block(const Args& a, int64_t t0, int rows, int b, int64_t slot, int g) {
  const focus_paged_append_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  const int64_t page = focus::page_of(c, b, (int)slot, a.shift);
  if (page < 0) {
    if (g == 0 && threadIdx.x % 64 == 0) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
    return;
  }
  const int in_block = (int)(slot & (d.cache.scale_rows - 1)), in_page = (int)(slot & (c.page_rows - 1));
  const int n = rows * a.pieces;
  // (both in flight before either is looked at)
  Side<T> k(a, false, t0, page, in_page, g), v(a, true, t0, page, in_page, g);
  k.load(a, n, in_block > 0), v.load(a, n, in_block > 0);
  k.store(a, n, in_block), v.store(a, n, in_block);
  if (g == 0 && threadIdx.x % 64 == 0) atomicMax(&c.length[b], (int)slot + rows);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void append_rows(Args a) {
  const focus_paged_append_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  // (neighbouring workgroups take the heads of the same rows)
  const uint32_t span = blockIdx.x / a.wide;
  const int g = (int)(blockIdx.x - span * a.wide) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (g >= c.n_kv_heads) return;
  const bool reports = g == 0 && threadIdx.x == 0;
  const int64_t cap = (int64_t)c.max_pages * c.page_rows, in_block = d.cache.scale_rows - 1;
  int64_t t = (int64_t)span << a.span_shift;
  const int64_t end = min(t + (1 << a.span_shift), d.n_rows), first = t;
  if (d.cu_rows && t == 0 && reports && (d.cu_rows[0] < 0 || d.cu_rows[c.batch] > d.n_rows))
    focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
  while (t < end) {
    const Owner o = owner_of(d, t);
    if (o.b >= c.batch || o.r1 <= t) return;  // (offsets that do not ascend, too)
    if (t < o.r0 || o.start < 0) {            // rows before the first offset; not served
      t = t < o.r0 ? o.r0 : o.r1;
      continue;
    }
    // from the first block whose first new row is not before this wave's rows
    const int64_t to_slot = o.start - o.r0;
    if (t == first && t > o.r0) t = ((t + to_slot + in_block) & ~(int64_t)in_block) - to_slot;
    for (; t < end && t < o.r1; t = ((t + to_slot + in_block + 1) & ~(int64_t)in_block) - to_slot) {
      const int64_t slot = t + to_slot, stop = min(o.r1, ((slot + in_block + 1) & ~(int64_t)in_block) - to_slot);
      if (slot < cap) {
        store_block<T>(a, t, (int)(stop - t), o.b, slot, g);
      } else if (reports) {
        focus::raise_err(d.err, FOCUS_ERR_CAPACITY);
      }
    }
    t = min(t, o.r1);
  }
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
  // Rows of a wave: one (most then find that their block is another wave's) as long as that
  // makes few workgroups, else up to as many as a block or a sequence has, on average.  1627
  // rows of 3 heads of 96 in 7 sequences, blocks of 8 (float32): one row 18.7 us, two 12.2,
  // four 13.4, eight 13.6.
  const int64_t wide = focus::ceil_div(c.n_kv_heads, kWaves), most = kResident * focus::device_cus();
  while (a.span_shift < a.scale_shift && (int64_t)c.batch << (a.span_shift + 1) <= d->n_rows &&
         focus::ceil_div(d->n_rows, int64_t{1} << a.span_shift) * wide > most)
    ++a.span_shift;
  const int64_t spans = focus::ceil_div(d->n_rows, int64_t{1} << a.span_shift);
  if (spans > INT32_MAX / kThreads / wide) return FOCUS_E_SHAPE;
  a.wide = (uint32_t)wide;
  const dim3 grid((uint32_t)(spans * wide));
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (d->dtype == FOCUS_BF16) hipLaunchKernelGGL(append_rows<__bf16>, grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(append_rows<float>, grid, dim3(kThreads), 0, s, a);
  return focus::launch_status();
}
