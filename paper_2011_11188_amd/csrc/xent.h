// Pieces of the last layer's cross entropy shared by its kernels.
#pragma once

#include "common.h"

namespace mdnn {

// A maximum m and the sum of exp(z - m) over some logits z of a row.  m is
// -Inf where there is no logit above it (none at all, or classes masked by a
// bias of -Inf): such a pair adds nothing, and differences are then taken from
// 0 so that they are no NaN.
struct Pair {
  float m, s;
};
__device__ __forceinline__ float pair_ref(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ Pair join(Pair a, Pair b) {
  const float m = fmaxf(a.m, b.m), ref = pair_ref(m);
  return {m, a.s * __expf(a.m - ref) + b.s * __expf(b.m - ref)};
}

}  // namespace mdnn
