// Device side of mixattn_set_layer_scores: with s = scale * q . k of a query at position i and a
// key at position j,
//   a = cap * tanh(s / cap)      (cap > 0; else a = s)
//   b = a - slope_h * (i - j)    (when the layer is biased)
// and the kernels' base-2 softmax runs on b * log2(e).
#pragma once

#include "internal.h"

namespace mixattn {

// tanh on |x| <= 1: x times a polynomial of degree 5 in x^2, fitted to tanh(x) / x by weighted
// least squares until the relative error was level (5.9e-7; 6.9e-7 as evaluated in fp32, about six
// fp32 roundings, and three orders below the bf16 rounding of the weights that follow).
// (tanh_coefficient is declared with ScoreShape.)
__device__ __forceinline__ float tanh_poly(float x) {   // |x| <= 1
  const float u = x * x;
  float p = fmaf(tanh_coefficient(5), u, tanh_coefficient(4));
  p = fmaf(p, u, tanh_coefficient(3));
  p = fmaf(p, u, tanh_coefficient(2));
  p = fmaf(p, u, tanh_coefficient(1));
  p = fmaf(p, u, tanh_coefficient(0));
  return p * x;
}
// 1 - 2 / (1 + e^2|x|) with the sign of x: two special-function operations, an absolute error of
// about 2^-23, so it serves where |tanh| is not small.  e^2|x| = inf gives 1; NaN stays NaN.
__device__ __forceinline__ float tanh_exp(float x) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(x) * 2.885390081777927f));   // 2 log2(e)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.f));
  return copysignf(fmaf(-2.f, r, 1.f), x);
}
// raw products -> capped base-2 scores
__device__ __forceinline__ void cap_scores(float (&s)[4], const ScoreShape& sh) {
  float x[4], top = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = s[e] * sh.pre;
    s[e] = tanh_poly(x[e]) * sh.post;
    top = fmaxf(top, fabsf(x[e]));
  }
  if (top > 1.f) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (fabsf(x[e]) > 1.f) s[e] = tanh_exp(x[e]) * sh.post;
  }
}
__device__ __forceinline__ float shaped_score_exact(float raw, const ScoreShape& sh, float bias) {   // fp32 mode
  float y = raw * sh.pre;
  if (sh.post > 0.f) y = tanhf(y) * sh.post;
  return y + bias;
}

}  // namespace mixattn
