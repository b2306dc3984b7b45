// Shared device code of the kernels for attention with changed scores: what a row sees.
#pragma once
#include "attend_common.hpp"

namespace dk {
namespace mfma {

// What a row sees: positions from .. last.
struct RowRange {
  int32_t pos, from, last;
};
__device__ __forceinline__ RowRange row_range(const ScoreParams& sp, const int32_t* first, const DkEntry& e, int tok) {
  RowRange r;
  r.pos = e.n + tok;
  r.last = max(r.pos, e.pad[0] - 1);
  r.from = sp.has_first ? first[e.tok0 + tok] : 0;
  if (sp.window > 0) r.from = max(r.from, r.pos - sp.window + 1);
  return r;
}

// What the non-finite elements of V that a row sees make of a sum of the finite ones, by their numbers.
__device__ __forceinline__ float with_non_finite(float sum, float nans, float plus, float minus) {
  if (nans > 0.f || (plus > 0.f && minus > 0.f)) return __uint_as_float(0x7fc00000u);
  return plus > 0.f ? INFINITY : minus > 0.f ? -INFINITY : sum;
}

}  // namespace mfma
}  // namespace dk
