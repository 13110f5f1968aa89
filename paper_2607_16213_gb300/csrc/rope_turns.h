// Frequencies of a rotary embedding as 64-bit fractions of a turn a position: plain host C++.
//
// The kernel multiplies a fraction by a 32-bit position, so its 64 bits have to be right for the angle to be: a frequency from pow
// and a division in 53 bits left the angle 2^-25 turns off at position 2^31.  So all of it is done in pairs of doubles (the rounded
// result and what it is short of: about 100 bits), with exp by its series and log as its inverse by Newton's method.
#pragma once

#include <cmath>
#include <cstdint>

#include "../../include/selkv.h"

namespace selkv {

struct Wide {
  double hi, lo;
};
inline Wide wide_sum(double a, double b) {  // a + b without error
  const double s = a + b, t = s - a;
  return {s, (a - (s - t)) + (b - t)};
}
inline Wide operator+(Wide a, Wide b) {
  const Wide s = wide_sum(a.hi, b.hi), t = wide_sum(a.lo, b.lo);
  const Wide u = wide_sum(s.hi, s.lo + t.hi);
  return wide_sum(u.hi, u.lo + t.lo);
}
inline Wide operator-(Wide a) { return {-a.hi, -a.lo}; }
inline Wide operator-(Wide a, Wide b) { return a + -b; }
inline Wide operator*(Wide a, Wide b) {
  const double p = a.hi * b.hi;
  return wide_sum(p, std::fma(a.hi, b.hi, -p) + std::fma(a.hi, b.lo, a.lo * b.hi));
}
inline Wide operator/(Wide a, Wide b) {
  const double q0 = a.hi / b.hi;
  const Wide r0 = a - b * Wide{q0, 0.0};
  const double q1 = r0.hi / b.hi;
  const Wide r1 = r0 - b * Wide{q1, 0.0};
  return wide_sum(q0, q1) + Wide{r1.hi / b.hi, 0.0};
}
inline bool operator<(Wide a, Wide b) { return a.hi < b.hi || (a.hi == b.hi && a.lo < b.lo); }
inline Wide wide_scale(Wide a, int e) { return {std::ldexp(a.hi, e), std::ldexp(a.lo, e)}; }
inline Wide wide_floor(Wide a) {
  const double f = std::floor(a.hi);
  return f == a.hi ? wide_sum(f, std::floor(a.lo)) : Wide{f, 0.0};
}

constexpr Wide kWideLn2{0.6931471805599453, 2.3190468138462996e-17};
constexpr Wide kWideTwoPi{6.283185307179586, 2.4492935982947064e-16};

inline Wide wide_exp(Wide x) {
  const double k = std::nearbyint(x.hi / kWideLn2.hi);
  const Wide r = wide_scale(x - kWideLn2 * Wide{k, 0.0}, -8);  // below 2^-9: ten terms leave 2^-110
  Wide e{1.0, 0.0};
  for (int n = 10; n > 0; --n) e = Wide{1.0, 0.0} + r * e / Wide{(double)n, 0.0};
  for (int i = 0; i < 8; ++i) e = e * e;
  return wide_scale(e, (int)k);
}
inline Wide wide_log(double x) {
  int e = 0;
  const double m = std::frexp(x, &e);
  Wide y{std::log(m), 0.0};
  for (int i = 0; i < 2; ++i) y = y + (wide_exp(-y) * Wide{m, 0.0} - Wide{1.0, 0.0});
  return y + kWideLn2 * Wide{(double)e, 0.0};
}

// The pairs' turns a position, modulo one and in units of 2^-64, into turns[0 .. rot / 2 - 1] (rounded; right to that where a pair
// turns less than 2^19 times a position); false where one is no number.  w_f is the power of w_1: 63 products leave 2^-88.
inline bool rope_turns(int rot, double theta, const selkv_rope_scaling* s, uint64_t* turns) {
  const int kind = s != nullptr ? s->kind : SELKV_ROPE_SCALE_NONE;
  const Wide none{0.0, 0.0}, all{1.0, 0.0}, log_theta = wide_log(theta);
  const Wide step = wide_exp(-(Wide{2.0, 0.0} / Wide{(double)rot, 0.0} * log_theta));
  double i0 = 0.0, i1 = 0.0;
  if (kind == SELKV_ROPE_SCALE_RAMP) {
    const Wide log_span = wide_log((double)s->original) - wide_log(kWideTwoPi.hi) - Wide{kWideTwoPi.lo / kWideTwoPi.hi, 0.0};
    // the pair that turns n times over the original context
    auto pair_of = [&](double n) { return Wide{(double)rot, 0.0} * (log_span - wide_log(n)) / (log_theta + log_theta); };
    i0 = std::fmax(0.0, wide_floor(pair_of(s->high)).hi);
    i1 = std::fmin(rot - 1.0, -wide_floor(-pair_of(s->low)).hi);
  }
  Wide w = all;
  for (int f = 0; f < rot / 2; ++f, w = w * step) {
    Wide t = w / kWideTwoPi;
    if (kind != SELKV_ROPE_SCALE_NONE) {
      Wide keep = none;
      if (kind == SELKV_ROPE_SCALE_WAVELENGTH)
        keep = (t * Wide{(double)s->original, 0.0} - Wide{s->low, 0.0}) / (Wide{s->high, 0.0} - Wide{s->low, 0.0});
      else if (kind == SELKV_ROPE_SCALE_RAMP)
        keep = all - Wide{f - i0, 0.0} / Wide{std::fmax(i1 - i0, 0.001), 0.0};
      keep = keep < none ? none : all < keep ? all : keep;
      t = keep * t + (all - keep) * t / Wide{s->factor, 0.0};
    }
    if (!std::isfinite(t.hi) || !std::isfinite(t.lo)) return false;
    t = t - wide_floor(t);
    const double high = std::ldexp(t.hi, 64), whole = std::floor(high);
    const double rest = std::floor((high - whole) + std::ldexp(t.lo, 64) + 0.5);  // (a few thousand at most)
    turns[f] = (whole < 0x1p64 ? (uint64_t)whole : 0u) + (uint64_t)(int64_t)rest;
  }
  return true;
}

}  // namespace selkv
