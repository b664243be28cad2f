// Shared by the output head's kernels (lm_head.cu, lm_head_tc.cuh): statistics of a strip of logits, the gradient of a logit, outputs.
#pragma once

#include "lm_common.cuh"

namespace cocodc_lm_impl {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kMostScale = 1e30f;
// Logits are taken in base 2 (times scale log2 e).  A strip of a row's logits leaves its largest one and the sum of 2^(z - largest): (m, s).
struct Stats { float m, s; };
__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.f : m; }   // nothing but -Inf: the sum is then 0
__device__ __forceinline__ Stats join(Stats a, Stats b) {
  const float m = fmaxf(a.m, b.m), k = shift_of(m);
  return Stats{m, a.s * fast_exp2(a.m - k) + b.s * fast_exp2(b.m - k)};
}

struct HeadArgs {
  long long T, V;
  int width;
  long long strips;
  float scale2;                                      // scale * log2 e
  const void* targets;
  int targets64;
  float2* stats;                                     // [strip][T]
  float* picked;                                     // [T]: the target's logit, base 2
};
__device__ __forceinline__ long long raw_target(const void* targets, int is64, long long t) {
  return is64 ? static_cast<const long long*>(targets)[t] : (long long)static_cast<const int*>(targets)[t];
}

struct DzArgs {
  long long T, V;
  float scale2;
  const void* targets;
  int targets64;
  const float *lse, *dlogp, *dlse, *factor;          // factor NULL: 1
  long long v0, v1;                                  // the piece
  void* dz;                                          // [T][pitch]
  long long pitch;
  int* status;
};
// What a row's dz needs: p's factor, what the target gets on top, and lse in base 2.
struct RowOf { float slope, hit, lse2; long long y; };
__device__ __forceinline__ RowOf row_of(const DzArgs& a, long long t) {
  RowOf r{0.f, 0.f, 0.f, -1};
  const float f = a.factor ? a.factor[0] : 1.f;
  if (a.targets) r.y = token_at(a.targets, a.targets64, t, a.V, a.status);
  const float up = r.y >= 0 ? a.dlogp[t] * f : 0.f, dl = a.dlse ? a.dlse[t] * f : 0.f, lse = a.lse[t];
  if ((up == 0.f && dl == 0.f) || lse == -INFINITY) {               // nothing: whatever p is, it counts for nothing
    r.y = -1;
    r.lse2 = INFINITY;
    return r;
  }
  r.slope = dl - up;
  r.hit = up;
  r.lse2 = lse == INFINITY ? __uint_as_float(0x7fc00000u) : lse * kLog2e;
  return r;
}
__device__ __forceinline__ float dz_of(const RowOf& r, float z2, bool target) {
  if (r.lse2 == INFINITY) return 0.f;
  return fmaf(fast_exp2(z2 - r.lse2), r.slope, target ? r.hit : 0.f);
}

// Where a product goes: fp32 sums that other pieces of the vocabulary share, or the output.
struct Out {
  void* out;
  int type, accumulate;
  long long ld;
  float* sums;                                       // [rows][cols], or NULL
  int add, last;                                     // add what the sums hold; the sums are complete and go to the output
  const float* factor;
  float scale;
};
// What the products are multiplied by at the end, in two steps where one number would leave fp32's range (and 0 times it be NaN).
struct Back {
  float one, two = 1.f;
  __device__ __forceinline__ explicit Back(const Out& o) : one(o.factor ? o.factor[1] * o.scale : o.scale) {
    if (!(one >= 0x1p-126f && one < INFINITY)) {
      one = o.factor ? o.factor[1] : 1.f;
      two = o.scale;
    }
  }
  __device__ __forceinline__ float operator()(float v) const { return v * one * two; }
};

}  // namespace cocodc_lm_impl
