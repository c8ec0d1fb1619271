// Host arithmetic in numbers of two doubles, hi + lo with |lo| at most half a unit of hi: some 100 significant bits, the same on
// every machine with IEEE doubles.  Error-free sums and products as by Knuth and Dekker; e^x by halving the argument nine
// times and a power series, ln x by one Newton step on it.
#pragma once

#include <cmath>

namespace pad {

struct Wide {
  double hi = 0, lo = 0;
  Wide() = default;
  Wide(double h) : hi(h) {}
  Wide(double h, double l) : hi(h), lo(l) {}
};

inline Wide wide_sum(double a, double b) {
  const double s = a + b, t = s - a;
  return {s, (a - (s - t)) + (b - t)};
}
inline Wide operator-(const Wide& a) { return {-a.hi, -a.lo}; }
inline Wide operator+(const Wide& a, const Wide& b) {
  const Wide h = wide_sum(a.hi, b.hi), l = wide_sum(a.lo, b.lo);
  const Wide s = wide_sum(h.hi, h.lo + l.hi);
  return wide_sum(s.hi, s.lo + l.lo);
}
inline Wide operator-(const Wide& a, const Wide& b) { return a + -b; }
inline Wide operator*(const Wide& a, const Wide& b) {
  const volatile double product = a.hi * b.hi;  // (rounded, whatever a compiler would fuse it with)
  const double p = product, e = std::fma(a.hi, b.hi, -p);
  return wide_sum(p, e + (a.hi * b.lo + a.lo * b.hi));
}
inline Wide operator/(const Wide& a, const Wide& b) {
  const double q = a.hi / b.hi;
  const Wide r = a - b * q;
  const double q2 = r.hi / b.hi;
  return wide_sum(q, q2) + (r - b * q2).hi / b.hi;
}
inline bool operator<(const Wide& a, const Wide& b) { return a.hi < b.hi || (a.hi == b.hi && a.lo < b.lo); }
inline Wide wide_floor(const Wide& a) {
  const double f = std::floor(a.hi);
  return f == a.hi ? wide_sum(f, std::floor(a.lo)) : Wide(f);
}

inline Wide wide_two_pi() { return {6.283185307179586, 2.4492935982947064e-16}; }

inline Wide wide_exp(const Wide& x) {
  if (!(std::fabs(x.hi) < 800)) return x.hi < 0 ? Wide(0) : Wide(HUGE_VAL);
  const Wide ln2(0.6931471805599453, 2.3190468138462996e-17);
  const double k = std::nearbyint(x.hi / ln2.hi);
  Wide r = x - ln2 * k;
  r = {std::ldexp(r.hi, -9), std::ldexp(r.lo, -9)};
  Wide term = 1, sum = 1;
  for (int i = 1; i <= 11; ++i) {  // (|r| < 2^-10: what follows is below 2^-140)
    term = term * r / (double)i;
    sum = sum + term;
  }
  for (int i = 0; i < 9; ++i) sum = sum * sum;
  return {std::ldexp(sum.hi, (int)k), std::ldexp(sum.lo, (int)k)};
}
// x > 0
inline Wide wide_log(const Wide& x) {
  const Wide y = std::log(x.hi);
  return y + (x * wide_exp(-y) - 1);
}

}  // namespace pad
