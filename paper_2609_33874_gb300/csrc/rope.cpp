// What the rotation by position needs of a model (jet_rope): the frequencies as fractions
// of a turn. An angle p f is needed modulo a turn only, and p times f / (2 pi) in units of
// 2^-64 turns wraps in 64 bits by itself: no position loses digits to a large angle. What is left
// are the digits of the quotient f / (2 pi) in doubles, 2^-52 of itself.
#include <cmath>
#include <cstring>

#include "jet.h"

extern "C" jet_status jet_rope_init(int32_t rot, int32_t style, double theta, const double* freq,
                                    int32_t norm, float eps, jet_rope* out) {
  if (!out) return JET_ERR_ARG;
  if (style != JET_ROPE_HALVES && style != JET_ROPE_PAIRS) return JET_ERR_ARG;
  if (norm != 0 && norm != 1) return JET_ERR_ARG;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return JET_ERR_ARG;
  if (rot < 0 || rot > 256 || rot % 8 != 0) return JET_ERR_SHAPE;
  if (!freq && !(theta > 0.0 && std::isfinite(theta))) return JET_ERR_ARG;
  jet_rope r;
  std::memset(&r, 0, sizeof(r));
  r.rot = rot;
  r.style = style;
  r.norm = norm;
  r.eps = eps;
  for (int i = 0; i < rot / 2; ++i) {
    const double f = freq ? freq[i] : std::pow(theta, -2.0 * i / rot);
    if (!std::isfinite(f)) return JET_ERR_ARG;
    // the fraction of its magnitude, to all 64 digits; a backward one is its complement (1 - t in
    // doubles would keep 54 binary digits of a small t)
    const double t = std::fmod(std::fabs(f) / 6.283185307179586476925286766559, 1.0);
    const uint64_t turn = static_cast<uint64_t>(std::ldexp(t, 64));  // t < 1
    r.turn[i] = f < 0.0 ? uint64_t(0) - turn : turn;
  }
  *out = r;
  return JET_OK;
}
