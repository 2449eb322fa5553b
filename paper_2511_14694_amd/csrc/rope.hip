// Rotary positions (focus_rope_turns, focus_rope).
//
// Every pair of a head's first rot_dim elements turns by pos * turns[i] revolutions.
// A float32 angle would be off by 0.06 rad at a million positions, so the product and
// its fraction are float64 (the fraction is then exact); what is left of it after
// taking out whole quarter turns is a float32 of at most 1/8, whose sine and cosine
// carry float32's relative accuracy.
//
// One workgroup per row: the sines and cosines of a row are computed once, in LDS, and
// serve every head.
#include "paged.h"

#include <math.h>

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRot = 256;

struct Store {
  focus_paged_kv c;
  int shift;
  bool on;
};

// Slot of row t in the cache: the page's element offset for head 0, or -1.
__device__ int64_t slot_of(const focus_rope_desc& d, const Store& st, int64_t t, bool first) {
  const int slot = d.row_slot[t], b = d.row_seq[t];
  if (slot < 0) return -1;
  if (b < 0 || b >= st.c.batch) {
    if (first) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
    return -1;
  }
  if (slot >= (int64_t)st.c.max_pages * st.c.page_rows) {
    if (first) focus::raise_err(d.err, FOCUS_ERR_CAPACITY);
    return -1;
  }
  const int64_t p = focus::page_of(st.c, b, slot, st.shift);
  if (p < 0) {
    if (first) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
    return -1;
  }
  return focus::row_at(st.c, p, slot, 0);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rope_rows(focus_rope_desc d, Store st) {
  __shared__ float2 cs[kMaxRot / 2];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, R = d.rot_dim, D = d.head_dim, half = R / 2;
  for (int i = tid; i < half; i += kThreads) {
    double f = (double)d.pos[t] * d.turns[i];
    f -= rint(f);
    const double q = rint(4.0 * f);
    const float x = (float)(f - 0.25 * q);
    float s, c;
    sincospif(2.f * x, &s, &c);
    const int k = (int)q & 3;  // quarter turns
    float2 r = k == 0 ? make_float2(c, s) : k == 1 ? make_float2(-s, c) : k == 2 ? make_float2(-c, -s) : make_float2(s, -c);
    if (d.inverse) r.y = -r.y;
    cs[i] = make_float2(r.x * d.amplitude, r.y * d.amplitude);
  }
  __syncthreads();
  const int64_t slot = st.on ? slot_of(d, st, t, tid == 0) : -1;
  const int H = d.q ? d.n_heads : 0, K = d.k ? d.n_kv_heads : 0;
  const int units = half + (D - R);  // pairs, then single elements
  for (int64_t u = tid; u < (int64_t)(H + K) * units; u += kThreads) {
    const int h = (int)(u / units), i = (int)(u % units);
    const bool is_q = h < H;
    const int hh = is_q ? h : h - H;
    const T* src = reinterpret_cast<const T*>(is_q ? d.q : d.k) + t * (is_q ? d.q_row : d.k_row) +
                   hh * (is_q ? d.q_head : d.k_head);
    T* dst = reinterpret_cast<T*>(is_q ? d.q_out : d.k_out);
    if (dst) dst += t * (is_q ? d.qo_row : d.ko_row) + hh * (is_q ? d.qo_head : d.ko_head);
    T* page = !is_q && slot >= 0 ? reinterpret_cast<T*>(st.c.k) + slot + hh * st.c.head_stride : nullptr;
    if (i < half) {
      const int a = d.pairs == FOCUS_ROPE_HALF ? i : 2 * i, b = d.pairs == FOCUS_ROPE_HALF ? i + half : 2 * i + 1;
      const float x = (float)src[a], y = (float)src[b];
      const T xo = (T)(x * cs[i].x - y * cs[i].y), yo = (T)(x * cs[i].y + y * cs[i].x);
      if (dst) dst[a] = xo, dst[b] = yo;
      if (page) page[a] = xo, page[b] = yo;
    } else {
      const int e = R + i - half;
      const T x = src[e];
      if (dst) dst[e] = x;
      if (page) page[e] = x;
    }
  }
  if (slot < 0) return;
  for (int u = tid; u < K * D; u += kThreads) {
    const int h = u / D, e = u % D;
    reinterpret_cast<T*>(st.c.v)[slot + h * st.c.head_stride + e] =
        reinterpret_cast<const T*>(d.v)[t * d.v_row + h * d.v_head + e];
  }
  if (st.c.weight)
    for (int h = tid; h < K; h += kThreads)
      st.c.weight[((int64_t)d.row_seq[t] * K + h) * st.c.weight_rows + d.row_slot[t]] = 0.f;
  if (tid == 0) atomicMax(st.c.length + d.row_seq[t], d.row_slot[t] + 1);
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
  const dim3 grid((uint32_t)d->n_rows), block(kThreads);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (d->dtype == FOCUS_BF16)
    hipLaunchKernelGGL((rope_rows<__bf16>), grid, block, 0, s, *d, st);
  else
    hipLaunchKernelGGL((rope_rows<float>), grid, block, 0, s, *d, st);
  return focus::launch_status();
}
