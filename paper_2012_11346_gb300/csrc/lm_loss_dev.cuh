// Device helpers shared by the vocabulary loss kernels.
#pragma once
#include <math.h>

#include "common.cuh"

namespace slim {
namespace lm {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ long long load_target(const void* t, int i64, long long i) {
  return i64 ? static_cast<const long long*>(t)[i] : static_cast<const int*>(t)[i];
}

// Part of a row's logits (its target's left out) as sum = sum_v 2^(z_v log2 e -
// base), base the largest exponent among them (-inf and 0: none).
struct LogSum {
  float base = -INFINITY, sum = 0.0f;
  __device__ __forceinline__ void add(float b, float s) {
    const float to = fmaxf(base, b), ref = to == -INFINITY ? 0.0f : to;
    sum = sum * exp2f(base - ref) + s * exp2f(b - ref);
    base = to;
  }
};

// A row's loss and log-sum from its other words' weight and its target's logit
// (read where there is one).  loss = log1p(rest / target) keeps its digits
// where the target outweighs the rest.  Returns whether the row counts.
__device__ __forceinline__ bool finish_loss(const LogSum& a, long long target, long long ignore,
                                            int V, const float* zt, float& loss, float& lse) {
  // a base of some tens and a logarithm, joined in fp64 so that only the result
  // is rounded
  const double rest64 = ((double)a.base + (double)log2f(a.sum)) * 0.69314718055994531;
  const float rest = (float)rest64;
  loss = 0.0f;
  lse = rest;
  if (target == ignore) return false;
  if (target < 0 || target >= V) {
    loss = __int_as_float(0x7fffffff);
    return true;
  }
  const float z = *zt, d = (float)(rest64 - (double)z);
  if (rest == -INFINITY && z > -INFINITY) {  // the target is all there is
    lse = z;
  } else {
    const float small = log1pf(expf(-fabsf(d)));
    loss = d > 0.0f ? d + small : small;
    lse = d > 0.0f ? rest + small : z + small;
    if (d != d) lse = loss = d;
  }
  return true;
}

}  // namespace lm
}  // namespace slim
