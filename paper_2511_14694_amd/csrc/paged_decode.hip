// Attention of one new token over a paged K/V cache (focus_paged_decode).
//
//   paged_attend   one workgroup per (sequence, head): four waves take the rows in
//                  turn, each with a running maximum and sum, joined through LDS
//   paged_weights  where weights are accumulated: per cached row and KV head, the
//                  softmax weights of the group's heads from the stored scores
#include "paged.h"

#include <math.h>

namespace {

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kMinit = -1.0e30f;
constexpr int kThreads = 256, kWaves = 4;

struct Plan {
  int64_t scores, cap;  // float offset and rows of the stored scores
  size_t bytes;
};

Plan make_plan(const focus_paged_decode_desc* d) {
  Plan p = {};
  p.cap = (int64_t)d->cache.max_pages * d->cache.page_rows;
  if (d->accumulate) {
    const int64_t heads = (int64_t)d->cache.batch * d->n_heads;
    p.scores = heads;  // the log-sum-exps (log2) come first
    p.bytes = (size_t)(heads + heads * p.cap) * sizeof(float);
  }
  return p;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void paged_attend(focus_paged_decode_desc d, float sc, int shift, float* ws,
                                                         int64_t scores, int64_t cap) {
  constexpr int E = D / 64;
  __shared__ float red_m[kWaves], red_l[kWaves], red_o[kWaves][D];
  const focus_paged_kv& c = d.cache;
  const int H = d.n_heads, b = blockIdx.x / H, h = blockIdx.x % H, g = h / (H / c.n_kv_heads);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int n = focus::paged_length(c, b);
  if (threadIdx.x == 0 && h == 0 && n != c.length[b]) focus::raise_err(d.err, FOCUS_ERR_CAPACITY);
  const T* q = reinterpret_cast<const T*>(d.q) + b * d.q_row + h * d.q_head + lane * E;
  float x[E], o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = (float)q[e] * sc, o[e] = 0.f;
  float m = kMinit, l = 0.f;
  for (int r = wave; r < n; r += kWaves) {
    const int64_t p = focus::page_of(c, b, r, shift);
    float s = 0.f;
    if (p < 0) {
      if (lane == 0) focus::raise_err(d.err, FOCUS_ERR_BOUNDS);
      s = -INFINITY;
    } else {
      const int64_t at = focus::row_at(c, p, r, g) + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) s = fmaf(x[e], (float)reinterpret_cast<const T*>(c.k)[at + e], s);
#pragma unroll
      for (int i = 32; i >= 1; i >>= 1) s += __shfl_xor(s, i);
      const float m_new = fmaxf(m, s), alpha = exp2f(m - m_new), w = exp2f(s - m_new);
      l = fmaf(l, alpha, w);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(w, (float)reinterpret_cast<const T*>(c.v)[at + e], o[e] * alpha);
      m = m_new;
    }
    if (d.accumulate && lane == 0) ws[scores + ((int64_t)b * H + h) * cap + r] = s;
  }
  if (lane == 0) red_m[wave] = m, red_l[wave] = l;
#pragma unroll
  for (int e = 0; e < E; ++e) red_o[wave][lane * E + e] = o[e];
  __syncthreads();
  float M = kMinit, L = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) M = fmaxf(M, red_m[w]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) L += red_l[w] * exp2f(red_m[w] - M);
  if (threadIdx.x < D) {
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) y = fmaf(red_o[w][threadIdx.x], exp2f(red_m[w] - M), y);
    reinterpret_cast<T*>(d.o)[((int64_t)b * H + h) * D + threadIdx.x] = (T)(L == 0.f ? 0.f : y / L);
  }
  if (threadIdx.x == 0) {
    const float e = L == 0.f ? -INFINITY : M + log2f(L);
    if (d.lse) d.lse[(int64_t)b * H + h] = e * kLn2;
    if (d.accumulate) ws[(int64_t)b * H + h] = e;
  }
}

__global__ __launch_bounds__(kThreads) void paged_weights(focus_paged_decode_desc d, const float* ws, int64_t scores,
                                                          int64_t cap) {
  const focus_paged_kv& c = d.cache;
  const int H = d.n_heads, K = c.n_kv_heads, G = H / K;
  const int b = blockIdx.x / K, g = blockIdx.x % K, n = focus::paged_length(c, b);
  float* w = c.weight + ((int64_t)b * K + g) * c.weight_rows;
  for (int r = blockIdx.y * kThreads + threadIdx.x; r < n; r += gridDim.y * kThreads) {
    float x = 0.f;
    for (int h = g * G; h < (g + 1) * G; ++h) {
      const float s = ws[scores + ((int64_t)b * H + h) * cap + r];
      if (s != -INFINITY) x += exp2f(s - ws[(int64_t)b * H + h]);
    }
    w[r] = d.weight_decay == 0.f ? x : fmaf(d.weight_decay, w[r], x);
  }
}

focus_status validate(const focus_paged_decode_desc* d) {
  const focus_paged_kv& c = d->cache;
  const focus_status st = focus::check_paged(c);
  if (st != FOCUS_OK) return st;
  if (c.head_dim != 64 && c.head_dim != 128) return FOCUS_E_UNSUPPORTED;
  if (d->n_heads <= 0 || d->split_keys < 0 || d->split_keys % 128 || !(d->softmax_scale == d->softmax_scale) ||
      !isfinite(d->weight_decay))
    return FOCUS_E_ARG;
  if (d->n_heads % c.n_kv_heads) return FOCUS_E_SHAPE;
  if ((int64_t)c.batch * d->n_heads > INT32_MAX / kThreads) return FOCUS_E_SHAPE;
  const int64_t es = focus::elt_bytes(c.dtype);
  if (d->q_row < 0 || d->q_head < 0 || !focus::pieces16(d->q_row, es) || !focus::pieces16(d->q_head, es))
    return FOCUS_E_ARG;
  return FOCUS_OK;
}

}  // namespace

extern "C" size_t focus_paged_decode_workspace(const focus_paged_decode_desc* d) {
  if (!d || validate(d) != FOCUS_OK) return 0;
  return make_plan(d).bytes;
}

extern "C" focus_status focus_paged_decode(const focus_paged_decode_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  focus_status st = validate(d);
  if (st != FOCUS_OK) return st;
  const focus_paged_kv& c = d->cache;
  if (c.batch == 0) return FOCUS_OK;
  if (!d->q || !d->o || (d->accumulate && !c.weight)) return FOCUS_E_NULL;
  if (!focus::aligned16(d->q) || !focus::aligned16(d->o) || (reinterpret_cast<uintptr_t>(d->lse) & 3u)) return FOCUS_E_ARG;
  const Plan p = make_plan(d);
  if (p.bytes && (!d->workspace || d->workspace_bytes < p.bytes)) return FOCUS_E_WORKSPACE;
  if (!focus::aligned16(d->workspace)) return FOCUS_E_ARG;
  const float scale = d->softmax_scale > 0.f ? d->softmax_scale : 1.0f / sqrtf((float)c.head_dim);
  const float sc = scale * kLog2e;
  const int shift = focus::page_shift(c);
  float* ws = reinterpret_cast<float*>(d->workspace);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 grid((uint32_t)(c.batch * d->n_heads)), block(kThreads);
#define FOCUS_LAUNCH(T, D) hipLaunchKernelGGL((paged_attend<T, D>), grid, block, 0, s, *d, sc, shift, ws, p.scores, p.cap)
  if (c.dtype == FOCUS_BF16) {
    if (c.head_dim == 128) FOCUS_LAUNCH(__bf16, 128); else FOCUS_LAUNCH(__bf16, 64);
  } else {
    if (c.head_dim == 128) FOCUS_LAUNCH(float, 128); else FOCUS_LAUNCH(float, 64);
  }
#undef FOCUS_LAUNCH
  if ((st = focus::launch_status()) != FOCUS_OK || !d->accumulate) return st;
  const int64_t y = focus::ceil_div(p.cap > 0 ? p.cap : 1, kThreads * 4);
  hipLaunchKernelGGL(paged_weights, dim3((uint32_t)(c.batch * c.n_kv_heads), (uint32_t)(y > 64 ? 64 : y)), block, 0, s, *d,
                     ws, p.scores, p.cap);
  return focus::launch_status();
}
