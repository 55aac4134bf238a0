// Sums of a softmax with a running maximum.  Shared by the kernels on logits; not part of the public interface.
#pragma once
#include <cfloat>

#include "qa_rows.h"

#if defined(__HIPCC__)

namespace qa {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kFar = -1e4f;                      // 2^kFar is 0

// With m the largest logit so far: s = sum of 2^t and w = sum of 2^t t, t = (x - m) log2 e.  Then log p = (x - m) -
// log s and entropy = log s - ln2 w / s; both terms of the entropy are >= 0, nothing cancels.
// m is -FLT_MAX at least, so that -infinity has t = -infinity and adds nothing; in the product t is kFar at least.
struct Sums { float m, s, w; };
__device__ __forceinline__ Sums no_sums() { return {-FLT_MAX, 0.0f, 0.0f}; }

// The same sums against another maximum.
__device__ __forceinline__ void raise(Sums& a, float m) {
  const float t = fmaxf((a.m - m) * kLog2e, kFar), f = __builtin_amdgcn_exp2f(t);
  a.w = (a.w + a.s * t) * f;
  a.s *= f;
  a.m = m;
}
}  // namespace qa

#endif  // __HIPCC__
