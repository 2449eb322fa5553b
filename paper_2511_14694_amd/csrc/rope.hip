// Rotary positions (focus_rope_turns, focus_rope).
//
// Every pair of a head's first rot_dim elements turns by pos * turns[i] revolutions.
// A float32 angle would be off by 0.06 rad at a million positions, so the product and
// its fraction are float64 (the fraction is then exact); what is left of it after
// taking out whole quarter turns is a float32 of at most 1/8, whose sine and cosine
// carry float32's relative accuracy.
//
// A workgroup takes a few rows.  The sines and cosines of its rows are computed once, in
// LDS, and serve every head.  A thread then takes pieces of 16 bytes (for half pairs two of
// them, half the turned part apart), always the same ones of a head, with 128 bytes in
// flight: the first are loaded before the angles are computed.  q, k and v are taken one
// after another, so that a step's addresses are a scalar and an offset that a thread keeps.
//
// HBM bound: 101 000 rows of 32 + 32 heads of 128 in bf16, k and v into pages, take 973 us
// (5.1 TB/s read and written; torch's copy of the same q reaches 4.3); without the cache
// 623 us (5.3 TB/s).  The first form, a workgroup a row and a thread a pair, took 2160.  How the threads
// share heads and rows is worked out by the host: with the divisions in the kernel one row
// took 5.4 us from launch to launch, now 4.5, and 2000 rows 17.4, now 14.1.
#include "paged.h"

#include <math.h>

#include <type_traits>

namespace {

using focus::u32x4;
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kMaxRot = 256;

struct Store {
  focus_paged_kv c;
  int shift;
  bool on;
};

// Slot of row t in the cache: the element offset of its head 0, or -1 and in `bit` why.
__device__ int64_t slot_of(const focus_rope_desc& d, const Store& st, int64_t t, int32_t& bit) {
  const int slot = d.row_slot[t], b = d.row_seq[t];
  bit = 0;
  if (slot < 0) return -1;
  if (b < 0 || b >= st.c.batch) {
    bit = FOCUS_ERR_BOUNDS;
    return -1;
  }
  if (slot >= (int64_t)st.c.max_pages * st.c.page_rows) {
    bit = FOCUS_ERR_CAPACITY;
    return -1;
  }
  const int64_t p = focus::page_of(st.c, b, slot, st.shift);
  if (p < 0) {
    bit = FOCUS_ERR_BOUNDS;
    return -1;
  }
  return focus::row_at(st.c, p, slot, 0);
}

// N elements of a head in registers: one access of 4, 8 or 16 bytes (as wide as a head's
// turned part is whole pieces of), or a single bf16.
template <typename T, int N> struct Piece {
  static constexpr bool kHalfWord = N * sizeof(T) == 2;
  static constexpr int kWords = kHalfWord ? 1 : N * sizeof(T) / 4;
  using V = typename std::conditional<kWords == 4, u32x4, typename std::conditional<kWords == 2, u32x2, uint32_t>::type>::type;
  V w;
  __device__ uint32_t word(int i) const {
    if constexpr (kWords == 1) return w;
    else return w[i];
  }
  __device__ void set(int i, uint32_t x) {
    if constexpr (kWords == 1) w = x;
    else w[i] = x;
  }
  __device__ void load(const T* p) {
    if constexpr (kHalfWord) w = *reinterpret_cast<const uint16_t*>(p);
    else w = *reinterpret_cast<const V*>(p);
  }
  __device__ void store(T* p) const {
    if constexpr (kHalfWord) *reinterpret_cast<uint16_t*>(p) = (uint16_t)w;
    else *reinterpret_cast<V*>(p) = w;
  }
  __device__ void unpack(float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 2) x[i] = i % 2 ? focus::bf16_hi(word(i / 2)) : focus::bf16_lo(word(i / 2));
      else x[i] = __uint_as_float(word(i));
    }
  }
  __device__ void pack(const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 4) set(i, __float_as_uint(x[i]));
      else if (i % 2 == 0) set(i / 2, focus::pack_bf16x2(x[i], i + 1 < N ? x[i + 1] : 0.f));
    }
  }
};

constexpr int kMaxRows = 8;

// Rows of one tensor: where they come from and go to.
template <typename T> struct Rows {
  const T* src;
  int64_t row, head;
  T* dst;               // or NULL
  int64_t drow, dhead;
  T* page;              // the cache's pool, or NULL
  int heads;
  bool turn;
};

// How the threads of a workgroup share a tensor's rows (host: no division at a kernel's
// start, where a single row's latency lies).
struct Walk {
  int per, chunks;   // rows of a step; steps of a row
  uint32_t by_heads; // 65536 / heads, rounded up: lane / heads = lane * by_heads >> 16
};
struct Units {
  int turned, units, lanes;  // turned units of a head; all; heads a workgroup takes at a time
  uint32_t by_units;         // 65536 / units, rounded up
  Walk q, kv;
};

template <typename T, int N, bool HALF>
__global__ __launch_bounds__(kThreads) void rope_rows(focus_rope_desc d, Store st, Units sh, int rows) {
  using P = Piece<T, N>;
  constexpr int kFlight = HALF && P::kWords == 4 ? 4 : 8;
  __shared__ float2 cs[kMaxRows][kMaxRot / 2];
  __shared__ int64_t s_slot[kMaxRows];
  const int64_t t0 = (int64_t)blockIdx.x * rows;
  const int tid = threadIdx.x, R = d.rot_dim, half = R / 2;
  const int here = (int)min((int64_t)rows, d.n_rows - t0);
  // units of a head: turned pieces (pairs of pieces), then the others
  const int turned = sh.turned, lanes = sh.lanes, lane = tid * sh.by_units >> 16, u = tid - lane * sh.units;
  const bool pair = HALF && u < turned;
  const int e = !HALF || u < turned ? u * N : R + (u - turned) * N;

  P lo[kFlight], hi[kFlight];
  // a step takes `lanes` heads of a row, or all heads of several rows
  struct At {
    int row, h;           // the thread's first row and head
    int load_row, load_h; // the next step to load: its first row, and heads before it
    int store_row, store_h;
  };
  auto start = [&](const Rows<T>& x, const Walk& w) {
    At at = {};
    at.row = w.chunks > 1 ? 0 : lane * w.by_heads >> 16;
    at.h = lane - at.row * x.heads;
    if (lane >= lanes || at.row >= w.per) at.row = here;
    return at;
  };
  // the step after (row, h)
  auto next = [&](const Rows<T>& x, const Walk& w, int& row, int& h) {
    h += lanes;
    if (h >= x.heads) h = 0, row += w.per;
  };
  auto load = [&](const Rows<T>& x, const Walk& w, At& at) {
    const T* from = x.src + (t0 + at.row) * x.row + at.h * x.head + e;
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      if (at.load_row + at.row < here && at.load_h + at.h < x.heads) {
        const T* p = from + (int64_t)at.load_row * x.row + (int64_t)at.load_h * x.head;
        lo[i].load(p);
        if (pair) hi[i].load(p + half);
      }
      next(x, w, at.load_row, at.load_h);
    }
  };
  auto store = [&](const Rows<T>& x, const Walk& w, At& at) {
    T* to = x.dst ? x.dst + (t0 + at.row) * x.drow + at.h * x.dhead + e : nullptr;
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const int row = at.store_row + at.row, h = at.store_h + at.h;
      if (row < here && h < x.heads) {
        if (x.turn && u < turned) {
          const float2* a = cs[row] + (HALF ? e : e / 2);
          float y[N], z[N];
          lo[i].unpack(y);
          if constexpr (HALF) {
            hi[i].unpack(z);
#pragma unroll
            for (int k = 0; k < N; ++k) {
              const float v = y[k] * a[k].x - z[k] * a[k].y;
              z[k] = y[k] * a[k].y + z[k] * a[k].x;
              y[k] = v;
            }
            hi[i].pack(z);
          } else {
#pragma unroll
            for (int k = 0; k < N; k += 2) {
              const float v = y[k] * a[k / 2].x - y[k + 1] * a[k / 2].y;
              y[k + 1] = y[k] * a[k / 2].y + y[k + 1] * a[k / 2].x;
              y[k] = v;
            }
          }
          lo[i].pack(y);
        }
        if (x.dst) {
          T* p = to + (int64_t)at.store_row * x.drow + (int64_t)at.store_h * x.dhead;
          lo[i].store(p);
          if (pair) hi[i].store(p + half);
        }
        if (x.page && s_slot[row] >= 0) {
          T* p = x.page + s_slot[row] + h * st.c.head_stride + e;
          lo[i].store(p);
          if (pair) hi[i].store(p + half);
        }
      }
      next(x, w, at.store_row, at.store_h);
    }
  };

  const Rows<T> q = {reinterpret_cast<const T*>(d.q), d.q_row, d.q_head, reinterpret_cast<T*>(d.q_out), d.qo_row,
                     d.qo_head, nullptr, d.n_heads, true};
  const Rows<T> k = {reinterpret_cast<const T*>(d.k), d.k_row, d.k_head, reinterpret_cast<T*>(d.k_out), d.ko_row,
                     d.ko_head, st.on ? reinterpret_cast<T*>(st.c.k) : nullptr, d.n_kv_heads, true};
  const Rows<T>& first = d.q ? q : k;
  const Walk& w0 = d.q ? sh.q : sh.kv;
  At at = start(first, w0);
  load(first, w0, at);

  for (int i = tid; i < here * half; i += kThreads) {
    const int row = here == 1 ? 0 : i / half, p = i - row * half;
    double f = (double)d.pos[t0 + row] * d.turns[p];
    f -= rint(f);
    const double quarter = rint(4.0 * f);
    float s, c;
    sincospif(2.f * (float)(f - 0.25 * quarter), &s, &c);
    const int n = (int)quarter & 3;
    float2 r = n == 0 ? make_float2(c, s) : n == 1 ? make_float2(-s, c) : n == 2 ? make_float2(-c, -s) : make_float2(s, -c);
    cs[row][p] = make_float2(r.x * d.amplitude, (d.inverse ? -r.y : r.y) * d.amplitude);
  }
  if (st.on && tid < here) {
    const int64_t t = t0 + tid;
    int32_t bit;
    const int64_t slot = slot_of(d, st, t, bit);
    s_slot[tid] = slot;
    if (bit) focus::raise_err(d.err, bit);
    // The length is raised by the last row of a run of ascending ones (the next row is
    // then stored, and raises it further): a prefill's rows would otherwise queue at one
    // address (101 000 of them for 0.5 ms).
    if (slot >= 0) {
      const int to = d.row_slot[t], b = d.row_seq[t];
      bool last = true;
      if (t + 1 < d.n_rows && d.row_seq[t + 1] == b && d.row_slot[t + 1] > to) last = slot_of(d, st, t + 1, bit) < 0;
      if (last) atomicMax(st.c.length + b, to + 1);
    }
  }
  __syncthreads();
  if (st.on && st.c.weight)
    for (int i = tid; i < here * d.n_kv_heads; i += kThreads) {
      const int row = here == 1 ? 0 : i / d.n_kv_heads, h = i - row * d.n_kv_heads;
      if (s_slot[row] >= 0)
        st.c.weight[((int64_t)d.row_seq[t0 + row] * d.n_kv_heads + h) * st.c.weight_rows + d.row_slot[t0 + row]] = 0.f;
    }

  auto rest = [&](const Rows<T>& x, const Walk& w) {
    for (bool loaded = true; at.store_row < here; loaded = false) {
      if (!loaded) load(x, w, at);
      store(x, w, at);
    }
  };
  rest(first, w0);
  if (d.q && d.k) {
    at = start(k, sh.kv);
    load(k, sh.kv, at);
    rest(k, sh.kv);
  }
  if (st.on) {
    const Rows<T> v = {reinterpret_cast<const T*>(d.v), d.v_row, d.v_head, nullptr, 0, 0, reinterpret_cast<T*>(st.c.v),
                       d.n_kv_heads, false};
    at = start(v, sh.kv);
    load(v, sh.kv, at);
    rest(v, sh.kv);
  }
}

// Rows a workgroup takes: several where there are enough of them for every compute
// unit, so that a thread has pieces to keep in flight.
int rows_per_group(int64_t n_rows) {
  const int64_t r = n_rows / (8 * focus::device_cus());
  return (int)(r < 1 ? 1 : r > kMaxRows ? kMaxRows : r);
}

Walk walk(int heads, int lanes) {
  if (heads <= 0) return {1, 1, 0};
  return {lanes >= heads ? lanes / heads : 1, (heads + lanes - 1) / lanes, (uint32_t)((65536 + heads - 1) / heads)};
}

template <typename T, int N, bool HALF>
void launch_rows(const focus_rope_desc& d, const Store& st, hipStream_t s) {
  Units sh;
  sh.turned = (HALF ? d.rot_dim / 2 : d.rot_dim) / N;
  sh.units = sh.turned + (d.head_dim - d.rot_dim) / N;
  sh.lanes = kThreads / sh.units;
  sh.by_units = (uint32_t)((65536 + sh.units - 1) / sh.units);  // exact: thread numbers are below 256
  sh.q = walk(d.q ? d.n_heads : 0, sh.lanes);
  sh.kv = walk(d.k ? d.n_kv_heads : 0, sh.lanes);
  const int rows = rows_per_group(d.n_rows);
  hipLaunchKernelGGL((rope_rows<T, N, HALF>), dim3((uint32_t)focus::ceil_div(d.n_rows, rows)), dim3(kThreads), 0, s, d, st,
                     sh, rows);
}

// The widest pieces that the turned part is whole ones of.  9000 rows of 64 + 8 heads of 80
// elements in bf16, 40 of them turned in halves: pieces of 8 bytes 39 us, single elements
// 92.  (float32 gains nothing by 8 bytes over 4: 20 000 rows of 24 heads of 128, 136 and 130.)
template <typename T>
void launch(const focus_rope_desc& d, const Store& st, hipStream_t s) {
  constexpr int N = 16 / sizeof(T);
  const int part = d.pairs == FOCUS_ROPE_HALF ? d.rot_dim / 2 : d.rot_dim;
  if (d.pairs == FOCUS_ROPE_HALF) {
    if (part % N == 0) launch_rows<T, N, true>(d, st, s);
    else if (sizeof(T) == 2 && part % 4 == 0) launch_rows<T, 4, true>(d, st, s);
    else launch_rows<T, 1, true>(d, st, s);
  } else {
    if (part % N == 0) launch_rows<T, N, false>(d, st, s);
    else launch_rows<T, 2, false>(d, st, s);
  }
}

bool strides_ok(int64_t row, int64_t head, int64_t es) {
  return row >= 0 && head >= 0 && focus::pieces16(row, es) && focus::pieces16(head, es);
}

}  // namespace

extern "C" focus_status focus_rope_turns(const focus_rope_scaling* s, double* turns) {
  if (!s || !turns) return FOCUS_E_NULL;
  const int R = s->rot_dim;
  if (R < 2 || R > kMaxRot || (R & 1) || !(s->theta > 1.0) || !isfinite(s->theta)) return FOCUS_E_ARG;
  if (s->kind < FOCUS_ROPE_NONE || s->kind > FOCUS_ROPE_BANDS) return FOCUS_E_ARG;
  if (s->kind != FOCUS_ROPE_NONE && (!(s->factor >= 1.0) || !isfinite(s->factor))) return FOCUS_E_ARG;
  if (s->kind == FOCUS_ROPE_BASE && R < 4) return FOCUS_E_ARG;
  if (s->kind == FOCUS_ROPE_BANDS &&
      (!(s->context > 0.0) || !isfinite(s->context) || !(s->low >= 0.0) || !(s->high > s->low) || !isfinite(s->high)))
    return FOCUS_E_ARG;
  const double theta = s->kind == FOCUS_ROPE_BASE ? s->theta * pow(s->factor, R / (R - 2.0)) : s->theta;
  for (int i = 0; i < R / 2; ++i) {
    double f = pow(theta, -2.0 * i / R) / (2.0 * M_PI);
    if (s->kind == FOCUS_ROPE_LINEAR) f /= s->factor;
    if (s->kind == FOCUS_ROPE_BANDS) {
      double g = (s->context * f - s->low) / (s->high - s->low);
      g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
      f *= (1.0 - g) / s->factor + g;
    }
    turns[i] = f;
  }
  return FOCUS_OK;
}

extern "C" focus_status focus_rope(const focus_rope_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  const int64_t es = focus::elt_bytes(d->dtype);
  if (es == 0) return FOCUS_E_DTYPE;
  if (d->n_rows < 0 || d->head_dim <= 0 || d->rot_dim < 0 || (d->rot_dim & 1) || d->rot_dim > d->head_dim ||
      (d->pairs != FOCUS_ROPE_INTERLEAVED && d->pairs != FOCUS_ROPE_HALF) || !isfinite(d->amplitude) ||
      (d->q && d->n_heads <= 0) || ((d->k || d->v) && d->n_kv_heads <= 0))
    return FOCUS_E_ARG;
  if (d->head_dim > 256 || !focus::pieces16(d->head_dim, es)) return FOCUS_E_UNSUPPORTED;
  Store st = {};
  if (d->cache) {
    const focus_status s = focus::check_paged(*d->cache);
    if (s != FOCUS_OK) return s;
    if (d->cache->dtype != d->dtype || d->cache->head_dim != d->head_dim || d->cache->n_kv_heads != d->n_kv_heads)
      return FOCUS_E_SHAPE;
    if (d->inverse) return FOCUS_E_ARG;
  }
  if ((d->k_out && !d->k) || (d->v && !d->cache) || (d->cache && d->n_rows > 0 && (!d->k || !d->v))) return FOCUS_E_NULL;
  if (d->n_rows == 0 || (!d->q && !d->k)) return FOCUS_OK;
  if (!d->pos || (d->rot_dim > 0 && !d->turns) || (d->q && !d->q_out) || (d->k && !d->k_out && !d->cache) ||
      (d->cache && (!d->row_seq || !d->row_slot)))
    return FOCUS_E_NULL;
  if (!focus::aligned16(d->q) || !focus::aligned16(d->q_out) || !focus::aligned16(d->k) ||
      !focus::aligned16(d->k_out) || !focus::aligned16(d->v) || (reinterpret_cast<uintptr_t>(d->pos) & 3u) ||
      (reinterpret_cast<uintptr_t>(d->turns) & 7u) || (reinterpret_cast<uintptr_t>(d->row_seq) & 3u) ||
      (reinterpret_cast<uintptr_t>(d->row_slot) & 3u))
    return FOCUS_E_ARG;
  if ((d->q && (!strides_ok(d->q_row, d->q_head, es) || !strides_ok(d->qo_row, d->qo_head, es))) ||
      (d->k && !strides_ok(d->k_row, d->k_head, es)) || (d->k_out && !strides_ok(d->ko_row, d->ko_head, es)) ||
      (d->v && !strides_ok(d->v_row, d->v_head, es)))
    return FOCUS_E_ARG;
  if ((d->q && !focus::disjoint_rows<2>(d->head_dim, {d->qo_row, d->qo_head}, {d->n_rows, d->n_heads})) ||
      (d->k_out && !focus::disjoint_rows<2>(d->head_dim, {d->ko_row, d->ko_head}, {d->n_rows, d->n_kv_heads})))
    return FOCUS_E_ARG;
  if (d->n_rows > INT32_MAX / kThreads) return FOCUS_E_SHAPE;
  if (d->cache) {
    st.c = *d->cache;
    st.shift = focus::page_shift(st.c);
    st.on = true;
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (d->dtype == FOCUS_BF16)
    launch<__bf16>(*d, st, s);
  else
    launch<float>(*d, st, s);
  return focus::launch_status();
}
