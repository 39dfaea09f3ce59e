// Rotary frequencies and the cos / sin tables, in double precision on the host.
//
// Pair i of a head with `rot` turned dims turns by w_i = theta^(-2 i / rot) a
// position, and with scaling for contexts `factor` times longer than the
// original_len tokens the model was trained on by
//   linear:  w_i / factor
//   banded:  w_i where the pair turns more than high_freq times in original_len
//            tokens, w_i / factor where it turns less than low_freq times, and in
//            between a blend that is linear in the number of turns
//   ramp:    a blend of the same two that is linear in the pair's index, between
//            the pairs that would turn beta_fast and beta_slow times in
//            original_len tokens (rounded outwards); cos and sin are scaled by
//            attn_factor, 0.1 ln(factor) + 1 if that is 0 (YaRN, arXiv 2309.00071)
#include <cmath>

#include "internal.h"

namespace sidp {

static bool finite_positive(float v) { return v > 0.f && std::isfinite(v); }

bool rope_frequencies(const sidp_rope& r, int head_dim, double* freqs, double* scale) {
  if (r.layout != SIDP_ROPE_HALF && r.layout != SIDP_ROPE_INTERLEAVED) return false;
  if (r.rotary_dim < 16 || r.rotary_dim > head_dim || r.rotary_dim % 16) return false;
  if (!(r.theta > 1.f) || !std::isfinite(r.theta)) return false;
  const double two_pi = 2.0 * std::acos(-1.0), theta = r.theta, rot = r.rotary_dim, orig = r.original_len;
  const int pairs = r.rotary_dim / 2;
  for (int i = 0; i < pairs; i++) freqs[i] = std::pow(theta, -2.0 * (double)i / rot);
  *scale = 1.0;
  if (r.scaling == SIDP_ROPE_SCALE_NONE) return true;
  if (!finite_positive(r.factor)) return false;
  const double factor = r.factor;
  if (r.scaling == SIDP_ROPE_SCALE_LINEAR) {
    for (int i = 0; i < pairs; i++) freqs[i] /= factor;
    return true;
  }
  if (r.original_len < 1) return false;
  if (r.scaling == SIDP_ROPE_SCALE_LLAMA3) {
    if (!finite_positive(r.low_freq) || !finite_positive(r.high_freq) || !(r.high_freq > r.low_freq)) return false;
    const double low = r.low_freq, high = r.high_freq;
    for (int i = 0; i < pairs; i++) {
      const double turns = orig * freqs[i] / two_pi;
      const double keep = std::min(1.0, std::max(0.0, (turns - low) / (high - low)));
      freqs[i] = keep * freqs[i] + (1.0 - keep) * (freqs[i] / factor);
    }
    return true;
  }
  if (r.scaling == SIDP_ROPE_SCALE_YARN) {
    if (!finite_positive(r.beta_slow) || !finite_positive(r.beta_fast) || !(r.beta_fast > r.beta_slow)) return false;
    if (!(r.attn_factor >= 0.f) || !std::isfinite(r.attn_factor) || (r.attn_factor == 0.f && factor < 1.0)) return false;
    // the (fractional) index of the pair that turns n times in original_len tokens
    auto pair_at = [&](double n) { return rot * std::log(orig / (n * two_pi)) / (2.0 * std::log(theta)); };
    const double lo = std::max(std::floor(pair_at(r.beta_fast)), 0.0);
    const double hi = std::min(std::ceil(pair_at(r.beta_slow)), rot - 1.0);
    const double width = hi > lo ? hi - lo : 0.001;
    for (int i = 0; i < pairs; i++) {
      const double stretch = std::min(1.0, std::max(0.0, ((double)i - lo) / width));
      freqs[i] = stretch * (freqs[i] / factor) + (1.0 - stretch) * freqs[i];
    }
    *scale = r.attn_factor > 0.f ? (double)r.attn_factor : 0.1 * std::log(factor) + 1.0;
    return true;
  }
  return false;
}

void rope_tables(const double* freqs, int pairs, double scale, int positions, int head_dim, float* cos, float* sin) {
  const size_t half = (size_t)head_dim / 2;
  for (int p = 0; p < positions; p++)
    for (size_t i = 0; i < half; i++) {
      const double a = (int)i < pairs ? (double)p * freqs[i] : 0.0;
      cos[(size_t)p * half + i] = (int)i < pairs ? (float)(std::cos(a) * scale) : 0.f;
      sin[(size_t)p * half + i] = (int)i < pairs ? (float)(std::sin(a) * scale) : 0.f;
    }
}

}  // namespace sidp
