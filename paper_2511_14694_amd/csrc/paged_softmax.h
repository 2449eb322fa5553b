// What the attention kernels over paged caches share: constants of the online softmax, a column's
// maximum, the log-sum-exp.
#pragma once

#include "paged.h"

#include <math.h>

namespace focus {

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kMinit = -3.40282347e38f; // the least finite score still counts
constexpr int kWave = 128;         // sequences whose lengths a wave holds, two a lane

// x, the same in all lanes, in a scalar register.
__device__ inline int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

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

}  // namespace focus
