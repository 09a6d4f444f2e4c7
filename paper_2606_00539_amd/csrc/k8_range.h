// The powers of two by which K8's Gram matrix and polynomial are multiplied in fp16,
// chosen so that neither passes its largest value, 65,504 (host code).
#pragma once

#include <math.h>

#include <algorithm>

namespace gnmr {

constexpr int kHeldX = 12;             // X is held times 2^12: |X| < 65504 / 2^12
constexpr double kMostSigma = 15.9;    // so its singular values have to stay below this

// p(s) = a + b s + c s^2, which a step multiplies a singular value of square s by.
struct StepPolynomial {
  double a, b, c;
  double at(double s) const { return a + s * (b + s * c); }
  // the largest |p| over [0, s]
  double most(double s) const {
    double m = std::max(fabs(at(0.0)), fabs(at(s)));
    const double v = c == 0.0 ? -1.0 : -b / (2.0 * c);
    if (v > 0.0 && v < s) m = std::max(m, fabs(at(v)));
    return m;
  }
  // the largest |x p(x^2)| over [0, top]: where its derivative a + 3 b s + 5 c s^2 is 0, or at top
  double most_image(double top) const {
    double m = top * fabs(at(top * top));
    auto root = [&](double s) {
      if (s > 0.0 && s < top * top) m = std::max(m, sqrt(s) * fabs(at(s)));
    };
    if (c != 0.0) {
      const double d = 9.0 * b * b - 20.0 * a * c;
      if (d >= 0.0) {
        root((-3.0 * b + sqrt(d)) / (10.0 * c));
        root((-3.0 * b - sqrt(d)) / (10.0 * c));
      }
    } else if (b != 0.0) {
      root(-a / (3.0 * b));
    }
    return m;
  }
};

struct HeldExponents {
  int a, p;     // A is held times 2^a, P times 2^p
  int growth;   // a step multiplies no singular value by more than 2^growth
};

// An update starts with singular values in [0, 1], since its Frobenius norm is at most 1.  Each
// step maps the interval that they can lie in to another, whose largest A = s and |P| are taken;
// 2% are left for the roundings.  Beyond kMostSigma X itself is out of range.  The usual
// coefficients leave both at 2^12: singular values to 1.2 and |P| to 3.4445.
inline HeldExponents held_exponents(float a, float b, float c, int steps) {
  constexpr double kMostHalf = 65504.0, kSlack = 1.02;
  const StepPolynomial p{a, b, c};
  double top = 1.0, most_a = 0.0, most_p = 0.0;
  for (int i = 0; i < steps; ++i) {
    most_a = std::max(most_a, top * top);
    most_p = std::max(most_p, p.most(top * top));
    top = std::min(kMostSigma, kSlack * p.most_image(top));
  }
  auto exponent = [&](double most) {
    const double e = floor(log2(kMostHalf / (kSlack * std::max(most, 1e-30))));
    return int(std::max(-120.0, std::min(double(kHeldX), e)));
  };
  const int growth = most_p > 0.0 ? int(std::max(0.0, ceil(log2(kSlack * most_p)))) : 0;
  return HeldExponents{exponent(most_a), exponent(most_p), growth};
}

}  // namespace gnmr
