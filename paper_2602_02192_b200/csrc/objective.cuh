// One token of the clipped objective with truncated importance sampling, for the forward calls and the gradient.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace echo {

struct GrpoRule {
  float eps_clip, C, beta;
  double log_hi, log_lo;       // log(1 + eps), log(1 - eps) (-inf if eps >= 1)
};
struct GrpoToken {
  float w, term, slope;        // the token counts w term, with slope w slope
};

__device__ __forceinline__ float grpo_clip(const GrpoRule &a, float rho) {
  return ptx::min_nan(ptx::max_nan(rho, 1.0f - a.eps_clip), 1.0f + a.eps_clip);
}
// The clipped term's slope is rho A where the minimum is the unclipped side (A > 0: rho <= 1 + eps; A < 0: rho >= 1 - eps),
// else 0; which side it is goes by the exact difference ln - lo, since the slope jumps there.
__device__ __forceinline__ bool grpo_flat(const GrpoRule &a, float A, float ln, float lo) {
  const double x = static_cast<double>(ln) - static_cast<double>(lo);
  return A > 0.f ? x > a.log_hi : x < a.log_lo;
}

// The token where a ratio exp(x) or the estimate's exp(d) is large.  Either may overflow beside a weight w = exp(lo - ls)
// < C that underflows: their products are exp(ln - ls) and exp(d + lo - ls), ordinary numbers.  (From 40 on: below, a
// product with a weight under fp32's normal numbers is under 1e-20.  The estimate's - 1 is nothing beside its exp(d).)
constexpr float kGrpoFar = 40.0f;
static __device__ __noinline__ GrpoToken grpo_token_far(const GrpoRule a, GrpoToken near, float A, float ln, float lo,
                                                        float ls, float lr) {
  const float x = ln - lo, d = a.beta > 0.f ? lr - ln : 0.f, w = near.w;
  // (lo = -inf beside an ln that is not: the ratio is infinite, and w = 0 times it is undefined)
  const bool far_ratio = w < a.C && x > kGrpoFar && lo > -INFINITY, far_kl = w < a.C && d > kGrpoFar;
  if (!far_ratio && !far_kl) return near;
  const float rho = A == 0.f && x > kGrpoFar ? 1.0f : expf(x);
  const float unclipped = far_ratio && A != 0.f ? static_cast<float>(exp(static_cast<double>(ln) - ls)) * A : w * (rho * A);
  GrpoToken t{1.0f, w * ptx::min_nan(rho * A, grpo_clip(a, rho) * A), grpo_flat(a, A, ln, lo) ? 0.f : unclipped};
  if (far_ratio) t.term = ptx::min_nan(unclipped, w * (grpo_clip(a, rho) * A));
  if (a.beta > 0.f) {
    float w_k = w * expm1f(d);
    if (far_kl) w_k = static_cast<float>(exp((static_cast<double>(lr) - ln) + (static_cast<double>(lo) - ls)));
    t.term -= a.beta * (w_k - w * d);
    t.slope = fmaf(a.beta, w_k, t.slope);
  }
  return t;
}

// w (min(rho A, clip(rho) A) - beta k) and w times the bracket's slope in ln; rho = exp(ln - lo), w = min(exp(lo - ls), C),
// k = exp(d) - d - 1 with d = lr - ln (beta = 0: no such term, lr is not used).  NaN in any of the log-probabilities, or in
// a difference of infinite ones, makes both NaN.
__device__ __forceinline__ GrpoToken grpo_token(const GrpoRule &a, float A, float ln, float lo, float ls, float lr) {
  float rho = expf(ln - lo), far = ln - lo;
  if (A == 0.f && rho == INFINITY) rho = 1.0f;         // a zero advantage weighs nothing: no inf * 0
  GrpoToken t{ptx::min_nan(expf(lo - ls), a.C), ptx::min_nan(rho * A, grpo_clip(a, rho) * A),
              grpo_flat(a, A, ln, lo) ? 0.f : rho * A};
  if (a.beta > 0.f) {
    const float d = lr - ln, k = expm1f(d);
    t.term -= a.beta * (k - d);
    t.slope = fmaf(a.beta, k, t.slope);
    far = fmaxf(far, d);
  }
  if (far > kGrpoFar) t = grpo_token_far(a, t, A, ln, lo, ls, lr);
  return t;
}

}  // namespace echo
