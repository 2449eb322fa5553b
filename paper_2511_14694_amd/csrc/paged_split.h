// How the rows of a batch of paged sequences are split into chunks, one workgroup each (and
// KV head, or neighbouring ones), and the partials of a sequence's chunks joined: shared by
// the attention kernels over paged caches.
#pragma once

#include "paged.h"

#include <math.h>

namespace focus {

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kMinit = -3.40282347e38f; // the least finite score still counts
constexpr int kSplitGrid = 32768;  // workgroups in a grid's second and third dimension
constexpr int kWave = 128;         // sequences whose lengths a wave holds, two a lane
constexpr int kPlan = 1024;        // threads of a planning workgroup

// What the device knows of the split.
struct Split {
  int split_keys;       // rows of a chunk, or 0: chosen
  int unit_shift;       // log2 of what chunks are multiples of
  int target;           // chunks resident at a time
  float each;           // cost of a chunk by itself, in rows read
  int64_t cap;          // rows of a sequence's table
  bool single;          // a sequence is one chunk
  int64_t slots;        // upper bound of the chunks of all sequences
  int4* info;           // [batch] {first slot, chunks, rows, rows of a chunk}
  int* owner;           // [slots] sequence (-1: none); null unless planned by paged_plan
};

// Rows of a chunk when they are to be chosen, for `target` chunks resident at a time: the
// least estimate of the time among
//   the rows of the whole batch spread over `target` chunks, rounded up to units, or over
//   half or twice as many;
//   the least size at which the chunks of all sequences are resident at once (up to kWave
//   sequences; it needs 16 steps of a search);
//   no split at all.
// The estimate, in rows a resident workgroup streams while all of them do: what there is
// to read, and for each chunk `each` rows' worth of beginning and end and its partials
// written and read, over the target; where not all are resident at once kLate of the
// longest more, which may begin late; at least the longest at kAlone times the rate, as
// fast as one gets when the others have ended.  us, before twice as many were tried (100 rows
// where 72 are now, all of the longest more) / now: 64 sequences of 4096 rows, 5 KV heads, 152 / 120;
// 48 with 7 heads 152 / 121; 16 of 10 000, 32 heads, 417 / 409; 200 of 1000 to 2000, 8 heads,
// 272 / 246; 400 of 600 to 1200, 4 heads, 165 / 184; over 104 such batches 0.8 % less.
constexpr float kLate = 0.3f, kAlone = 1.1f;

__device__ inline float estimate(const Split& a, uint32_t units, int chunks, int rows, int longest) {
  const float even = ((float)units * (1 << a.unit_shift) + a.each * (float)chunks) / (float)a.target;
  const float last = (float)min(rows, longest);
  return fmaxf(chunks > a.target ? even + kLate * last : even, last / kAlone);
}

// Sum and maximum of f(rows) over the sequences: of a wave, two sequences a lane, or of
// paged_plan's workgroup.  The results are the same in all threads.
struct OverWave {
  int n0, n1;  // rows of the lane's sequences; -1 for none
  template <typename F> __device__ uint32_t total(F f) const {
    return (uint32_t)__builtin_amdgcn_readlane(wave_scan((int)(f(n0) + f(n1))), 63);
  }
  template <typename F> __device__ uint32_t most(F f) const { return (uint32_t)wave_max((int)max(f(n0), f(n1))); }
};
struct OverGroup {
  const focus_paged_kv& c;
  int* s_part;  // one per wave
  template <typename F> __device__ uint32_t total(F f) const {
    uint32_t x = 0;
    for (int b = threadIdx.x; b < c.batch; b += kPlan) x += f(paged_length(c, b));
    return join(wave_scan((int)x), [](int x, int y) { return x + y; });
  }
  template <typename F> __device__ uint32_t most(F f) const {
    uint32_t x = 0;
    for (int b = threadIdx.x; b < c.batch; b += kPlan) x = max(x, f(paged_length(c, b)));
    return join(wave_max((int)x), [](int x, int y) { return max(x, y); });
  }
  template <typename Op> __device__ uint32_t join(int x, Op op) const {
    __syncthreads();
    if (threadIdx.x % 64 == 63) s_part[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int w = 0; w < kPlan / 64; ++w) x = op(x, s_part[w]);
    return (uint32_t)x;
  }
};

// (Counted in units: the host has checked that all tables together hold fewer than 2^31.)
template <typename Over> __device__ int chunk_rows(const Split& a, int batch, const Over& over) {
  const int shift = a.unit_shift, unit = 1 << shift;
  const uint32_t target = (uint32_t)a.target;
  // units of a sequence; its chunks of so many units
  auto units_of = [&](int n) { return (uint32_t)(max(n, 0) + unit - 1) >> shift; };
  auto chunks = [&](uint32_t units) {
    return over.total([&](int n) { return n < 0 ? 0u : max(1u, (units_of(n) + units - 1) / units); });
  };
  const uint32_t total = over.total(units_of);
  if (total + batch <= target) return unit;
  const uint32_t one = (total + target - 1) / target, two = min(2 * one, 1u << 30 >> shift);
  const uint32_t whole = max(1u, over.most(units_of));
  if (one >= whole) return (int)(whole << shift);
  const int longest = (int)(whole << shift);
  const uint32_t count1 = chunks(one), count2 = chunks(two);
  uint32_t units = one;
  float best = estimate(a, total, count1, one << shift, longest);
  auto better = [&](uint32_t count, uint32_t with) {
    const float e = estimate(a, total, count, with << shift, longest);
    if (e < best) best = e, units = with;
  };
  better(count2, two);
  const uint32_t half = (one + 1) / 2;
  better(chunks(half), half);
  if (count1 > target && batch <= kWave && (uint32_t)batch <= target) {
    uint32_t lo = one, hi = whole;  // too many chunks at lo, few enough at hi
    for (int k = 0; k < 16 && hi - lo > 1; ++k) {
      const uint32_t mid = (lo + hi) / 2;
      const bool many = chunks(mid) > target;
      lo = many ? mid : lo, hi = many ? hi : mid;
    }
    better(chunks(hi), hi);
  }
  better(batch, whole);
  return (int)(units << shift);
}

// The chunk of slot i (chunks 0: none), in scalar registers: all of a wave's lanes ask for
// the same.
__device__ inline int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
struct Chunk {
  int b, c, n, slot0, chunks, rows;
};
__device__ __forceinline__ Chunk find_chunk(const Split& a, const focus_paged_kv& c, int i) {
  int b = 0, n = 0, slot0 = i, chunks = 0, rows = (int)a.cap;
  if (a.single) {
    if (i < c.batch) b = i, n = paged_length(c, i), chunks = 1;
  } else if (a.owner) {
    const int own = i < a.slots ? scalar(a.owner[i]) : -1;
    if (own >= 0) {
      const int4 info = a.info[own];
      b = own, slot0 = info.x, chunks = info.y, n = info.z, rows = info.w;
    }
  } else {
    const int two = threadIdx.x % 64 * 2;
    const int n0 = two < c.batch ? paged_length(c, two) : -1;
    const int n1 = two + 1 < c.batch ? paged_length(c, two + 1) : -1;
    rows = scalar(a.split_keys ? a.split_keys : chunk_rows(a, c.batch, OverWave{n0, n1}));
    auto chunks_of = [&](int n) { return n < 0 ? 0 : max(1, (n - 1) / rows + 1); };
    const int own0 = chunks_of(n0), own1 = chunks_of(n1), upto = wave_scan(own0 + own1);
    if (i < __builtin_amdgcn_readlane(upto, 63)) {
      const int lane = __ffsll((unsigned long long)__ballot(i < upto)) - 1;
      const int end = __builtin_amdgcn_readlane(upto, lane), last = __builtin_amdgcn_readlane(own1, lane);
      const bool second = i >= end - last;
      b = 2 * lane + second;
      n = __builtin_amdgcn_readlane(second ? n1 : n0, lane);
      chunks = __builtin_amdgcn_readlane(second ? own1 : own0, lane);
      slot0 = end - last - (second ? 0 : chunks);
    }
  }
  slot0 = scalar(slot0);
  return {scalar(b), i - slot0, scalar(n), slot0, scalar(chunks), scalar(rows)};
}

// The chunks of more than kWave sequences, by one workgroup of kPlan threads.  (With every
// wave going through all lengths by itself 4096 sequences of 200 to 400 rows, 8 KV heads of
// 128, took 1570 us, now 900; of 128 sequences the launch would cost as much as it saves.)
__device__ __forceinline__ void plan_chunks(const Split& a, const focus_paged_kv& c) {
  __shared__ int s_part[kPlan / 64];
  const int tid = threadIdx.x;
  const int rows = a.split_keys ? a.split_keys : chunk_rows(a, c.batch, OverGroup{c, s_part});
  int before = 0;
  for (int b0 = 0; b0 < c.batch; b0 += kPlan) {
    const int b = b0 + tid, n = b < c.batch ? paged_length(c, b) : 0;
    const int own = b < c.batch ? max(1, (n - 1) / rows + 1) : 0, upto = wave_scan(own);
    __syncthreads();  // the last round's sums are read
    if (tid % 64 == 63) s_part[tid / 64] = upto;
    __syncthreads();
    int slot = before + upto - own;
#pragma unroll
    for (int w = 0; w < kPlan / 64; ++w) {
      if (w < tid / 64) slot += s_part[w];
      before += s_part[w];
    }
    if (b < c.batch) a.info[b] = make_int4(slot, own, n, rows);
    for (int k = 0; k < own && slot + k < a.slots; ++k) a.owner[slot + k] = b;
  }
  for (int64_t i = before + tid; i < a.slots; i += kPlan) a.owner[i] = -1;
}

// Maximum over the lanes 16 and 32 apart.
__device__ inline float max_column(float x) {
  const uint32_t u = __float_as_uint(x);
  auto y = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])));
  y = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// log of a softmax's sum, from its maximum score (unscaled) and its sum; sc: the scale in
// log2 units.
__device__ inline float lse_of(float sc, float2 ml) {
  return ml.y == 0.f ? -INFINITY : fmaf(ml.x, sc, log2f(ml.y)) * kLn2;
}

// Maximum and sum over a sequence's chunks of column h of `columns`, by one wave.
__device__ inline float2 joined(const float2* ml, float sc, const int4& info, int columns, int h) {
  const int lane = threadIdx.x % 64;
  float M = kMinit, L = 0.f;
  for (int i = lane; i < info.y; i += 64) {
    const float2 y = ml[(int64_t)(info.x + i) * columns + h];
    const float m = fmaxf(M, y.x);
    L = L * __builtin_amdgcn_exp2f((M - m) * sc) + y.y * __builtin_amdgcn_exp2f((y.x - m) * sc);
    M = m;
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) {
    const float m2 = __shfl_xor(M, k), l2 = __shfl_xor(L, k), m = fmaxf(M, m2);
    L = L * __builtin_amdgcn_exp2f((M - m) * sc) + l2 * __builtin_amdgcn_exp2f((m2 - m) * sc);
    M = m;
  }
  return make_float2(M, L);
}

}  // namespace focus
