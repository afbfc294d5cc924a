// Capped scores, cap tanh(x / cap) of x = softmax_scale q.k, in the exp2 domain.
//
// Near caps, up to kNearCap:  cap - 2 cap / (1 + e^(2 x / cap)), one exponential and one reciprocal.  It cancels where x is small beside the cap: a score is off by about
// 4 2^-24 of the cap, whatever it is itself, so at most by 2^-16 (less than the rounding of the weights, 2^-9 or 2^-17).
// Far caps, above it: x (1 + u^2 P(u^2)), u = x / cap, up to |u| = 1/2, with the terms of tanh's series up to u^14 (the next one is 9e-9); beyond, cap (1 - 2 / (1 + e^(2 u))),
// whose error is a few units of the score there.  Right at any cap: what is small against it stays as it is.
#pragma once

#include <math.h>

#include <algorithm>

#include "common.h"

namespace eco {

constexpr float kNearCap = 64.f;
enum { kNoCap, kNear, kFar };

struct Cap {
  int kind;
  float scale_log2e;  // of the scores
  float in;           // near: 2 x / cap = in (q.k), in the exp2 domain;  far: u = in x
  float log2e;        // the cap in the exp2 domain
};
// (clamped: factors that leave fp32 would make 0 times them NaN)
inline Cap make_cap(float softcap, float scale_log2e) {
  const auto held = [](double x) { return (float)std::min(x, 3.4028234663852886e38); };
  const double cap = (double)softcap * 1.4426950408889634;
  if (!(softcap > 0.f)) return {kNoCap, scale_log2e, 0.f, 0.f};
  if (softcap <= kNearCap) return {kNear, scale_log2e, held(2.0 * scale_log2e / softcap), (float)cap};
  return {kFar, scale_log2e, held(1.0 / cap), held(cap)};
}

#if defined(__HIPCC__)
// Near caps: -1 / (1 + e^(2 x / cap)) of a product q.k; times twice the cap, and the cap added, it is the score.
__device__ __forceinline__ float near_cap(float qk, const Cap& cap) { return __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(qk * cap.in)); }
// Far caps: the score of a product q.k.  (One behind the other: all of a step's side by side would take the registers of others.)
__device__ __forceinline__ float far_cap(float qk, const Cap& cap) {
  const float x = qk * cap.scale_log2e, u = x * cap.in, u2 = u * u;
  float p = -929569.f / 638512875.f;
  p = __builtin_fmaf(p, u2, 21844.f / 6081075);
  p = __builtin_fmaf(p, u2, -1382.f / 155925);
  p = __builtin_fmaf(p, u2, 62.f / 2835);
  p = __builtin_fmaf(p, u2, -17.f / 315);
  p = __builtin_fmaf(p, u2, 2.f / 15);
  p = __builtin_fmaf(p, u2, -1.f / 3);
  float all = cap.log2e * __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u * (2.f * kLog2e))), 1.f), few = __builtin_fmaf(x * u2, p, x);
  asm volatile("" : "+v"(all), "+v"(few));  // (a select, and no branch per score)
  return fabsf(u) > 0.5f ? all : few;
}
#endif

}  // namespace eco
