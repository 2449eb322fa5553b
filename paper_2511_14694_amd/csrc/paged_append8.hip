// Rows stored in a paged cache of 8 bits, a power of two as scale for each block of rows and
// KV head (focus_paged_append8).
//
// One wave takes a block of a sequence, a KV head and k or v: the largest magnitude of the
// new rows gives the scale, the elements times its inverse are exact and rounded once.  Lanes
// take 16 neighbouring elements each (one 16-byte store).  Which blocks a wave takes follows
// from its rows: it covers a few consecutive ones and takes the blocks whose first new row
// is among them, so that no block has two writers, whatever the lengths of the sequences.
#include "paged.h"

namespace {

using focus::u32x4;

constexpr int kThreads = 256, kWaves = 4;
constexpr float kLargest = 448.f;  // of e4m3
constexpr uint32_t kInf = 0x7f800000u;

struct Args {
  focus_paged_append8_desc d;
  int shift, scale_shift;  // log2 page_rows, scale_rows
  int span_shift;          // log2 of the rows a wave covers
  int pieces;              // of 16 elements, in a row of a head
  uint32_t inv;            // 2^20 / pieces, rounded up (exact quotients of less than 2^16)
};

// The least e >= -126 with most <= 448 2^e, as the bits of 2^e; most finite.
__device__ inline uint32_t scale_bits(uint32_t most) {
  // most = 1.m 2^x, 448 = 1.75 2^8
  const int x = (int)(most >> 23) - 127, e = x - ((most & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return (uint32_t)(max(e, -126) + 127) << 23;
}

// 16 elements as float32.
template <typename T> __device__ inline void load16(const T* p, float (&x)[16]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p + 8 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[8 * i + 2 * k] = focus::bf16_lo(w[k]), x[8 * i + 2 * k + 1] = focus::bf16_hi(w[k]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p + 4 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[4 * i + k] = __uint_as_float(w[k]);
    }
  }
}

__device__ inline uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// 16 numbers of at most 448 (or NaN) to e4m3.
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

// Index of the first of cu[1 .. n] greater than t (n if none is), by a wave: 64 of them are
// looked at together.
__device__ int sequence_of(const int32_t* cu, int n, int64_t t) {
  const int lane = threadIdx.x % 64;
  int lo = 0, len = n;
  while (len > 0) {
    const int step = (len + 63) / 64, at = lo + (lane + 1) * step - 1;  // the last of the lane's part
    const bool upto = at < lo + len && cu[at + 1] <= t;
    const int parts = __popcll(__ballot(upto));
    lo += parts * step;
    len = min(step - 1, len - parts * step);
  }
  return lo;
}

template <typename T>
__device__ void store_block(const Args& a, int64_t t0, int rows, int b, int64_t slot, int g, bool is_v) {
  const focus_paged_append8_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  const int lane = threadIdx.x % 64;
  const int64_t page = focus::page_of(c, b, (int)slot, a.shift);
  if (page < 0) {
    if (g == 0 && !is_v && lane == 0) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
    return;
  }
  const T* src = reinterpret_cast<const T*>(is_v ? d.v : d.k) + t0 * (is_v ? d.v_row : d.k_row) +
                 (int64_t)g * (is_v ? d.v_head : d.k_head);
  const int64_t step = is_v ? d.v_row : d.k_row;
  const int in_block = (int)(slot & (d.cache.scale_rows - 1)), in_page = (int)(slot & (c.page_rows - 1));
  uint8_t* dst = reinterpret_cast<uint8_t*>(is_v ? c.v : c.k) + page * c.page_stride + (int64_t)g * c.head_stride;
  float* scale = (is_v ? d.cache.v_scale : d.cache.k_scale) +
                 (page * c.n_kv_heads + g) * (c.page_rows >> a.scale_shift) + (in_page >> a.scale_shift);
  const int n = rows * a.pieces;
  uint32_t most = 0, any = 0;  // greatest finite magnitude, and any
  for (int i = lane; i < n; i += 64) {
    const int r = (int)((uint32_t)i * a.inv >> 20), e = (i - r * a.pieces) * 16;
    float x[16];
    load16(src + r * step + e, x);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const uint32_t m = magnitude(x[k]);
      any = max(any, m);
      most = max(most, m < kInf ? m : 0u);
    }
  }
  most = (uint32_t)focus::wave_max((int)most);
  any = (uint32_t)focus::wave_max((int)any);
  float to = __uint_as_float(scale_bits(most));
  if (in_block > 0) {
    const float was = *scale;
    if (was >= to) {
      to = was;
    } else {
      const float f = was / to;
      uint8_t* old = dst + (int64_t)(in_page - in_block) * c.row_stride;
      for (int i = lane; i < in_block * a.pieces; i += 64) {
        const int r = (int)((uint32_t)i * a.inv >> 20), e = (i - r * a.pieces) * 16;
        u32x4* at = reinterpret_cast<u32x4*>(old + r * c.row_stride + e);
        const u32x4 w = *at;
        float x[16];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
          x[4 * k] = lo[0] * f, x[4 * k + 1] = lo[1] * f, x[4 * k + 2] = hi[0] * f, x[4 * k + 3] = hi[1] * f;
        }
        *at = round16(x);
      }
    }
  }
  for (int i = lane; i < n; i += 64) {
    const int r = (int)((uint32_t)i * a.inv >> 20), e = (i - r * a.pieces) * 16;
    float x[16];
    load16(src + r * step + e, x);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      x[k] /= to;
      if (any >= kInf && !(fabsf(x[k]) <= kLargest)) x[k] = __uint_as_float(0x7fc00000u);
    }
    *reinterpret_cast<u32x4*>(dst + (int64_t)(in_page + r) * c.row_stride + e) = round16(x);
  }
  if (lane == 0) {
    *scale = to;
    if (g == 0 && !is_v) atomicMax(&c.length[b], (int)slot + rows);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void append_rows(Args a) {
  const focus_paged_append8_desc& d = a.d;
  const focus_paged_kv& c = d.cache.kv;
  const int unit = blockIdx.y * kWaves + threadIdx.x / 64;  // k of all heads, then v
  if (unit >= 2 * c.n_kv_heads) return;
  const bool is_v = unit >= c.n_kv_heads, reports = unit == 0 && threadIdx.x == 0;
  const int g = is_v ? unit - c.n_kv_heads : unit;
  const int64_t cap = (int64_t)c.max_pages * c.page_rows;
  int64_t t = (int64_t)blockIdx.x << a.span_shift;
  const int64_t end = min(t + (1 << a.span_shift), d.n_rows), first = t;
  if (d.cu_rows && t == 0 && reports && (d.cu_rows[0] < 0 || d.cu_rows[c.batch] > d.n_rows))
    focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
  while (t < end) {
    int b = (int)t;
    int64_t r0 = t, r1 = t + 1;  // the sequence's rows
    if (d.cu_rows) {
      b = sequence_of(d.cu_rows, c.batch, t);
      if (b >= c.batch) return;
      r0 = max(d.cu_rows[b], 0), r1 = min((int64_t)d.cu_rows[b + 1], d.n_rows);
      if (t < r0) {              // rows before the first offset
        t = r0;
        continue;
      }
      if (r1 <= t) return;       // (offsets that do not ascend)
    }
    const int64_t start = d.start[b];
    if (start < 0) {
      t = r1;
      continue;
    }
    const int64_t slot = start + (t - r0), next = t + d.cache.scale_rows - (slot & (d.cache.scale_rows - 1));
    const int64_t stop = min(r1, next);
    // (a block whose first new row lies before this wave's rows is another wave's)
    if (t > first || t == r0 || (slot & (d.cache.scale_rows - 1)) == 0) {
      if (slot >= cap) {
        if (reports) focus::raise_err(d.err, FOCUS_ERR_CAPACITY);
      } else {
        store_block<T>(a, t, (int)(stop - t), b, slot, g, is_v);
      }
    }
    t = stop;
  }
}

focus_status validate(const focus_paged_append8_desc* d) {
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

extern "C" focus_status focus_paged_append8(const focus_paged_append8_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  const focus_status st = validate(d);
  const focus_paged_kv& c = d->cache.kv;
  if (st != FOCUS_OK || c.batch == 0 || d->n_rows == 0) return st;
  Args a = {};
  a.d = *d;
  a.shift = focus::page_shift(c), a.scale_shift = __builtin_ctz((unsigned)d->cache.scale_rows);
  a.pieces = c.head_dim / 16, a.inv = ((1 << 20) + a.pieces - 1) / a.pieces;
  // rows of a wave: as many as a block has, fewer where sequences have fewer
  while (a.span_shift < a.scale_shift && (int64_t)c.batch << (a.span_shift + 1) <= d->n_rows) ++a.span_shift;
  const dim3 grid((uint32_t)focus::ceil_div(d->n_rows, int64_t{1} << a.span_shift),
                  (uint32_t)focus::ceil_div(2 * c.n_kv_heads, kWaves));
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (d->dtype == FOCUS_BF16) hipLaunchKernelGGL(append_rows<__bf16>, grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(append_rows<float>, grid, dim3(kThreads), 0, s, a);
  return focus::launch_status();
}
