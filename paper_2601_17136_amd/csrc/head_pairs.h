// A target's pairs (class, teacher's logit) as the class head's kernels read them.
#pragma once
#include <cfloat>

#include "kkm_internal.h"

namespace kkm {

// The target is softmax(scale t) over a row's pairs.  A pair's key is t, with its
// sign turned where the scale is negative, and its weight exp(|scale| (key -
// largest key)): no product overflows before the difference is taken, so logits
// near the type's lowest value and a scale of 0 have the weights of the formula.
// A pair of a negative id or a logit of -inf is none, whatever the scale.
__device__ inline float pair_key(const int32_t* __restrict__ ids, const float* __restrict__ logits, int64_t at,
                                 float scale, int classes, int& id, bool& bad) {
  id = ids[at];
  const float t = id < 0 ? -INFINITY : logits ? logits[at] : 0.f;
  if (t == -INFINITY) id = -1;
  if (id >= classes) {
    id = -1;
    bad = true;
  }
  return id < 0 ? -INFINITY : scale < 0.f ? -t : t;
}

__device__ inline float pair_weight(float key, float largest, float scale) {
  const float gap = key - largest;
  return expf(fabsf(scale) * (gap == -INFINITY ? -FLT_MAX : gap));
}

}  // namespace kkm
