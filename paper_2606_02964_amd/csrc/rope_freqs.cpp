// rope_freqs.cpp -- frequency tables of rotary positions (msa_rope_freqs): host
// arithmetic in 64 bits, once per model.
#include <cmath>
#include <string>

#include "errors.h"
#include "msa_rope.h"

namespace {

msa_status refuse(const std::string& what) {
  msa::set_last_error("msa_rope_freqs: " + what);
  return MSA_ERR_INVALID_ARG;
}

bool positive(double x) { return std::isfinite(x) && x > 0.0; }

}  // namespace

extern "C" msa_status msa_rope_freqs(const msa_rope_scaling* scaling, int32_t rotary_dim, double* inv_freq,
                                     float* amplitude) {
  if (!scaling || !inv_freq) return refuse("scaling and inv_freq must be non-null");
  const msa_rope_scaling& s = *scaling;
  const double kTwoPi = 6.283185307179586476925;
  if (rotary_dim < 2 || rotary_dim % 2 != 0) return refuse("rotary_dim must be even and >= 2");
  if (s.reserved != 0) return refuse("reserved must be zero");
  if (s.kind < MSA_ROPE_SCALE_NONE || s.kind > MSA_ROPE_SCALE_PAIRS) return refuse("unknown kind");
  if (!positive(s.base)) return refuse("base must be finite and > 0");
  if (s.kind != MSA_ROPE_SCALE_NONE && !positive(s.factor)) return refuse("factor must be finite and > 0");
  if (s.kind == MSA_ROPE_SCALE_BASE && rotary_dim == 2) return refuse("kind BASE needs rotary_dim > 2");
  const bool mixed = s.kind == MSA_ROPE_SCALE_TURNS || s.kind == MSA_ROPE_SCALE_PAIRS;
  if (mixed && !positive(s.original_len)) return refuse("original_len must be finite and > 0");
  if (mixed && !(s.low >= 0.0 && s.low < s.high && std::isfinite(s.high))) return refuse("0 <= low < high is needed");
  if (s.kind == MSA_ROPE_SCALE_PAIRS && !(s.base > 1.0 && s.low > 0.0)) return refuse("kind PAIRS needs base > 1 and low > 0");
  const double R = rotary_dim;
  const double base = s.kind == MSA_ROPE_SCALE_BASE ? s.base * std::pow(s.factor, R / (R - 2.0)) : s.base;
  // (kind PAIRS) the pair, in fractions, that makes `turns` turns: original_len * base^(-2 i / R) = 2 pi turns
  auto pair_of = [&](double turns) { return R * std::log(s.original_len / (kTwoPi * turns)) / (2.0 * std::log(s.base)); };
  double from = 0.0, to = 0.0;
  if (s.kind == MSA_ROPE_SCALE_PAIRS) {
    from = std::fmax(std::floor(pair_of(s.high)), 0.0);
    to = std::fmin(std::ceil(pair_of(s.low)), R - 1.0);
    if (to <= from) to = from + 0.001;  // (a step)
  }
  for (int32_t i = 0; i < rotary_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / R);
    double keep = 1.0;  // share of f that is not divided
    if (s.kind == MSA_ROPE_SCALE_LINEAR) keep = 0.0;
    if (s.kind == MSA_ROPE_SCALE_TURNS) keep = (s.original_len * f / kTwoPi - s.low) / (s.high - s.low);
    if (s.kind == MSA_ROPE_SCALE_PAIRS) keep = 1.0 - (i - from) / (to - from);
    keep = std::fmin(std::fmax(keep, 0.0), 1.0);
    inv_freq[i] = keep == 1.0 ? f : keep * f + (1.0 - keep) * (f / s.factor);
  }
  // (contexts that are not stretched keep their scores: the logarithm would lower them, below factor e^-10 past 0)
  const bool raised = s.kind == MSA_ROPE_SCALE_PAIRS && s.factor > 1.0;
  if (amplitude) *amplitude = raised ? (float)(0.1 * std::log(s.factor) + 1.0) : 1.0f;
  return MSA_OK;
}
