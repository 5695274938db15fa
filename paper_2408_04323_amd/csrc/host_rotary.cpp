// Frequencies of the rotations by position, scaled for contexts longer than a model was trained with (host code only).
#include <cmath>

#include "internal.h"

using namespace scoot;

namespace {
constexpr double kPi = 3.14159265358979323846;
bool positive(double x) { return x > 0.0 && std::isfinite(x); }
double within01(double x) { return x < 0.0 ? 0.0 : x > 1.0 ? 1.0 : x; }
}  // namespace

extern "C" int scoot_rotary_frequencies(int dim, double base, int scaling, double factor, double length, double low, double high,
                                        double* freqs, double* magnitude) {
  clear_error();
  if (dim < 2 || dim > 1024 || dim % 2 != 0) return fail_static(SCOOT_ERR_INVALID_ARG, "rotary: dim must be even, in 2..1024");
  if (!(base > 1.0) || !std::isfinite(base)) return fail_static(SCOOT_ERR_INVALID_ARG, "rotary: base must be above 1 and finite");
  if (!freqs || !magnitude) return fail_static(SCOOT_ERR_INVALID_ARG, "rotary: null output");
  if (scaling < SCOOT_ROTARY_NONE || scaling > SCOOT_ROTARY_BANDS) return fail_static(SCOOT_ERR_INVALID_ARG, "rotary: unknown scaling");
  if (scaling != SCOOT_ROTARY_NONE && (!(factor >= 1.0) || !std::isfinite(factor)))
    return fail_static(SCOOT_ERR_INVALID_ARG, "rotary: factor must be at least 1 and finite");
  const bool blends = scaling == SCOOT_ROTARY_RAMP || scaling == SCOOT_ROTARY_BANDS;
  if (blends && (!positive(length) || !positive(low) || !positive(high) || !(low < high)))
    return fail_static(SCOOT_ERR_INVALID_ARG, "rotary: length, low and high must be positive, and low below high");
  if (scaling == SCOOT_ROTARY_BASE && dim == 2) return fail_static(SCOOT_ERR_INVALID_ARG, "rotary: base scaling needs more than one pair");
  const int pairs = dim / 2;
  if (scaling == SCOOT_ROTARY_BASE) base *= std::pow(factor, (double)dim / (dim - 2));
  // Pairs that make `turns` turns over the length: base^(-2 i / dim) length = 2 pi turns.
  const auto pair_of = [&](double turns) { return dim * std::log(length / (2.0 * kPi * turns)) / (2.0 * std::log(base)); };
  double first = 0.0, last = 1.0;
  if (scaling == SCOOT_ROTARY_RAMP) {
    first = std::fmax(std::floor(pair_of(high)), 0.0);
    last = std::fmin(std::ceil(pair_of(low)), dim - 1.0);
    if (!(last > first)) last = first + 0.001;
  }
  for (int i = 0; i < pairs; ++i) {
    const double f = std::pow(base, -2.0 * i / dim);
    double keep = 1.0;  // how much of the pair stays as it is; the rest goes `factor` times slower
    if (scaling == SCOOT_ROTARY_LINEAR) keep = 0.0;
    if (scaling == SCOOT_ROTARY_RAMP) keep = 1.0 - within01((i - first) / (last - first));
    if (scaling == SCOOT_ROTARY_BANDS) keep = within01((length * f / (2.0 * kPi) - low) / (high - low));
    freqs[i] = scaling == SCOOT_ROTARY_BASE ? f : keep * f + (1.0 - keep) * f / factor;
  }
  *magnitude = scaling == SCOOT_ROTARY_RAMP ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return SCOOT_OK;
}
