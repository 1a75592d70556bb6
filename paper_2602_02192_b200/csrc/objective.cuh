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
constexpr float kGrpoFar = 40.0f;      // (below it a product with a weight under fp32's normal numbers is under 1e-20)

// A ratio exp(x) that may overflow beside a weight w = exp(lo - ls) < C that may underflow: their product is exp(ln - ls),
// an ordinary number.  The same for the estimate's exp(d) (whose - 1 is nothing beside it).
static __device__ __noinline__ GrpoToken grpo_token_far(float A, float ln, float lo, float ls, float lr, float d, float w,
                                                        float policy, float slope, bool flat, float clipped, bool far_ratio,
                                                        bool far_kl, float beta) {
  GrpoToken t{1.0f, w * policy, w * slope};
  if (far_ratio) {
    const float both = A == 0.f ? 0.f : static_cast<float>(exp(static_cast<double>(ln) - ls)) * A;
    t.term = ptx::min_nan(both, w * (clipped * A));
    t.slope = flat ? 0.f : both;
  }
  if (far_kl) {
    const float e = static_cast<float>(exp((static_cast<double>(lr) - ln) + (static_cast<double>(lo) - ls)));
    t.term -= beta * (e - w * d);
    t.slope = fmaf(beta, e, t.slope);
  } else if (beta > 0.f) {
    const float k = expm1f(d);
    t.term -= w * (beta * (k - d));
    t.slope = fmaf(w, beta * k, t.slope);
  }
  return t;
}

// w (min(rho A, clip(rho) A) - beta k) and w times the bracket's slope in ln; rho = exp(ln - lo), w = min(exp(lo - ls), C),
// k = exp(d) - d - 1 with d = lr - ln (beta = 0: no such term, lr is not used).  The clipped term's slope is rho A where
// the minimum is the unclipped side (A > 0: rho <= 1 + eps; A < 0: rho >= 1 - eps), else 0; which side it is goes by the
// exact difference ln - lo, since the slope jumps there.  NaN in any of the log-probabilities, or in a difference of
// infinite ones, makes both NaN.
__device__ __forceinline__ GrpoToken grpo_token(const GrpoRule &a, float A, float ln, float lo, float ls, float lr) {
  float rho = expf(ln - lo);
  if (A == 0.f && rho == INFINITY) rho = 1.0f;         // a zero advantage weighs nothing: no inf * 0
  const float w = ptx::min_nan(expf(lo - ls), a.C);
  const float clipped = ptx::min_nan(ptx::max_nan(rho, 1.0f - a.eps_clip), 1.0f + a.eps_clip);
  const double x = static_cast<double>(ln) - static_cast<double>(lo);
  const bool flat = A > 0.f ? x > a.log_hi : x < a.log_lo;
  float term = ptx::min_nan(rho * A, clipped * A);
  float slope = flat ? 0.f : rho * A;
  const bool kl = a.beta > 0.f;
  const float d = kl ? lr - ln : 0.f;
  // (lo = -inf beside an ln that is not: the ratio is infinite, and w = 0 times it is undefined)
  const bool far_ratio = w < a.C && ln - lo > kGrpoFar && lo > -INFINITY, far_kl = w < a.C && d > kGrpoFar;
  if (far_ratio || far_kl) return grpo_token_far(A, ln, lo, ls, lr, d, w, term, slope, flat, clipped, far_ratio, far_kl, a.beta);
  if (kl) {
    const float k = expm1f(d);
    term -= a.beta * (k - d);
    slope = fmaf(a.beta, k, slope);
  }
  return {w, term, slope};
}

}  // namespace echo
