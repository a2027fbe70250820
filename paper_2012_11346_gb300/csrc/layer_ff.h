// The gated feed-forward's activations, and its form for a few rows
// (layer_ff_rows.cu).
#pragma once
#include <math.h>

#include <type_traits>

#include "../../include/slim_layer.h"
#include "common.cuh"
#include "tc_common.cuh"

namespace slim {
namespace layer {

// sigmoid(y), and with REST 1 - sigmoid(y), each to its own digits.  FAST: within some
// units of 2^-22 of either, for results that are rounded to bf16.
template <bool FAST, bool REST>
__device__ __forceinline__ void sigmoids(float y, float& s, float& rest) {
  if (FAST) {
    // from -88 on e^-y is infinite, and s = 0 right; rest takes it as the largest number
    float e = tc::ex2_approx(-1.44269504f * y);
    if (REST) e = fminf(e, 3.0e38f);
    s = __fdividef(1.0f, 1.0f + e);
    if (REST) rest = e > 1e37f ? 1.0f : e * s;
    if (y != y) s = rest = y;
    return;
  }
  const float e = expf(-fabsf(y)), big = 1.0f / (1.0f + e), small = e * big;
  s = y >= 0.0f ? big : small;
  rest = y >= 0.0f ? small : big;
  if (y != y) s = rest = y;
}

// a = act(g), and with GRAD its derivative da.
template <int ACT, bool FAST, bool GRAD>
__device__ __forceinline__ void activate(float g, float& a, float& da) {
  if (ACT == SLIM_ACT_RELU) {
    a = g > 0.0f ? g : g != g ? g : 0.0f;
    if (GRAD) da = g > 0.0f ? 1.0f : 0.0f;
  } else if (ACT == SLIM_ACT_GELU) {
    // g Phi(g): the complementary error function keeps the digits of the lower tail
    const float phi = 0.5f * erfcf(-0.70710678f * g);
    a = g * phi;
    if (GRAD) da = fmaf(g * 0.39894228f, FAST ? __expf(-0.5f * g * g) : expf(-0.5f * g * g), phi);
  } else {
    // g sigmoid(y), or sigmoid(g) alone
    constexpr float k = 1.5957691216f, m = 0.044715f;  // 2 sqrt(2 / pi)
    float y = g, t = 0.0f;
    if (ACT == SLIM_ACT_GELU_TANH) {
      t = fminf(fmaxf(g, -30.0f), 30.0f);  // sigmoid has long come to its end
      y = k * t * fmaf(m * t, t, 1.0f);
    }
    float s, rest;
    sigmoids<FAST, GRAD>(y, s, rest);
    a = ACT == SLIM_ACT_SIGMOID ? s : g * s;
    if (GRAD) {
      if (ACT == SLIM_ACT_SIGMOID)
        da = s * rest;
      else if (ACT == SLIM_ACT_SILU)
        da = s * fmaf(g, rest, 1.0f);
      else
        da = s * fmaf(t * rest, k * fmaf(3.0f * m * t, t, 1.0f), 1.0f);
    }
  }
}

// Calls go(act) with the activation as a constant.
template <typename Go>
__host__ __device__ __forceinline__ void with_act(int act, Go go) {
  switch (act) {
    case SLIM_ACT_SILU: go(std::integral_constant<int, SLIM_ACT_SILU>()); break;
    case SLIM_ACT_GELU: go(std::integral_constant<int, SLIM_ACT_GELU>()); break;
    case SLIM_ACT_GELU_TANH: go(std::integral_constant<int, SLIM_ACT_GELU_TANH>()); break;
    case SLIM_ACT_RELU: go(std::integral_constant<int, SLIM_ACT_RELU>()); break;
    default: go(std::integral_constant<int, SLIM_ACT_SIGMOID>()); break;
  }
}

// Whether a forward of these sizes takes the form for a few rows.
bool ff_rows_fit(long long N, int D, int F, slim_dtype dtype);
// Arguments as in slim_gated_ff_fwd, already checked.  Nothing waits: no workspace.
slim_status ff_rows_fwd(const void* x, const void* w, int N, int D, int F, slim_dtype dtype,
                        slim_act act, void* h, cudaStream_t s);

}  // namespace layer
}  // namespace slim
