// Inverse frequencies of rotary positions, scaled for contexts longer than the trained one (host, in double).
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/deltakv.h"

extern "C" int32_t dk_rotary_freqs(int32_t rotary_dim, double base, int32_t scaling, const double* params, float* inv_freq_out,
                                   float* amplitude_out) {
  if (rotary_dim < 0 || rotary_dim % 2 || !(base > 0.0) || !std::isfinite(base) || (rotary_dim > 0 && !inv_freq_out))
    return DK_ERR_INVALID;
  if (scaling < DK_ROTARY_PLAIN || scaling > DK_ROTARY_RAMP) return DK_ERR_UNSUPPORTED;
  const double pi2 = 6.283185307179586;
  double factor = 1.0, low = 0.0, high = 0.0, length = 0.0;
  if (scaling != DK_ROTARY_PLAIN) {
    if (!params || !(params[0] > 0.0) || !std::isfinite(params[0])) return DK_ERR_INVALID;
    factor = params[0];
  }
  if (scaling == DK_ROTARY_BASE) {
    if (rotary_dim <= 2) return DK_ERR_INVALID;
    base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
  }
  double from = 0.0, to = 0.0;
  if (scaling == DK_ROTARY_BANDS || scaling == DK_ROTARY_RAMP) {
    low = params[1];
    high = params[2];
    length = params[3];
    if (!(low > 0.0) || !(high >= low) || !(length > 0.0) || !std::isfinite(high) || !std::isfinite(length)) return DK_ERR_INVALID;
    if (scaling == DK_ROTARY_BANDS && high == low) return DK_ERR_INVALID;
    if (scaling == DK_ROTARY_RAMP) {
      if (base == 1.0) return DK_ERR_INVALID;
      // the pair that turns `times` times within the length: length * base^(-2 i / rotary_dim) = 2 pi times
      const auto pair_of = [&](double times) { return rotary_dim * std::log(length / (times * pi2)) / (2.0 * std::log(base)); };
      const double last = std::max(0, rotary_dim - 1);
      from = std::min(std::max(std::floor(pair_of(high)), 0.0), last);
      to = std::min(std::max(std::ceil(pair_of(low)), 0.0), last);
    }
  }
  for (int32_t i = 0; i < rotary_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rotary_dim);
    double kept = 1.0;  // the share that stays as it is
    if (scaling == DK_ROTARY_LINEAR) kept = 0.0;
    if (scaling == DK_ROTARY_BANDS) kept = std::min(std::max((length * f / pi2 - low) / (high - low), 0.0), 1.0);
    if (scaling == DK_ROTARY_RAMP) kept = to > from ? 1.0 - std::min(std::max((i - from) / (to - from), 0.0), 1.0) : (i > from ? 0.0 : 1.0);
    inv_freq_out[i] = (float)(kept * f + (1.0 - kept) * f / factor);
  }
  if (amplitude_out) *amplitude_out = scaling == DK_ROTARY_RAMP && factor > 1.0 ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return DK_OK;
}
