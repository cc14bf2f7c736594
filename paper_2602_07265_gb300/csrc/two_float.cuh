// Numbers held as the unevaluated sum of two fp32 values (about 48 bits), for the few
// places where fp32 does not decide and fp64 units are scarce.
//
// Sums are Knuth's two-sum, products use the fused multiply-add's exact residual
// (Dekker, "A floating-point technique for extending the available precision", 1971).
// exp reduces by multiples of ln 2 and takes the Taylor series, whose terms from the sixth on
// need fp32 only: r^6 / 720 is below 2^-18 for |r| <= ln 2 / 2.
#pragma once

#include <cmath>
#include <cstring>

#ifdef __CUDACC__
#define XS_HD __host__ __device__ __forceinline__
#else
#define XS_HD inline
#endif

namespace xs {

struct Two {
  float hi, lo;   // |lo| <= half an ulp of hi
};

// a + b with |a| >= |b| or a == 0.
XS_HD Two quick_two(float a, float b) {
  const float s = a + b;
  return Two{s, b - (s - a)};
}
XS_HD Two two_sum(float a, float b) {
  const float s = a + b, v = s - a;
  return Two{s, (a - (s - v)) + (b - v)};
}
XS_HD Two operator+(Two a, Two b) {
  const Two s = two_sum(a.hi, b.hi), t = two_sum(a.lo, b.lo);
  const Two u = quick_two(s.hi, s.lo + t.hi);
  return quick_two(u.hi, u.lo + t.lo);
}
XS_HD Two operator+(Two a, float b) {
  const Two s = two_sum(a.hi, b);
  return quick_two(s.hi, s.lo + a.lo);
}
XS_HD Two operator*(Two a, Two b) {
  const float p = a.hi * b.hi, e = fmaf(a.hi, b.hi, -p);
  return quick_two(p, fmaf(a.hi, b.lo, fmaf(a.lo, b.hi, e)));
}
// 1 / b within 2 ulp for 2^-100 < b < 2^100 (on the device without the division's branches, so that
// several values' chains run side by side).
XS_HD float near_reciprocal(float b) {
#ifdef __CUDA_ARCH__
  const float r = __fdividef(1.f, b);
  return fmaf(r, fmaf(-b, r, 1.f), r);
#else
  return 1.f / b;
#endif
}
// a / b for such b: the quotient's residual is exact but for its own rounding.
XS_HD Two operator/(Two a, Two b) {
  const float r = near_reciprocal(b.hi), q = a.hi * r;
  return quick_two(q, (fmaf(-q, b.hi, a.hi) + fmaf(-q, b.lo, a.lo)) * r);
}

// 2^k for -126 <= k <= 127.
XS_HD float power_of_two(int k) {
  const unsigned bits = static_cast<unsigned>(k + 127) << 23;
#ifdef __CUDA_ARCH__
  return __uint_as_float(bits);
#else
  float v;
  memcpy(&v, &bits, 4);
  return v;
#endif
}

// e^x for x <= 0, within 2^-40 of its value and 2^-148 (the parts may be subnormal: the latter is the larger
// from x = -75 down); 0 below -100.
XS_HD Two two_exp(float x) {
  const bool none = !(x > -100.f);
  x = none ? 0.f : x;
  const float n = rintf(x * 1.44269504f);
  // ln 2 = 0.693145751953125 (15 bits, so that n times it is exact) + the rest as two fp32.
  const float r0 = fmaf(n, -0.693145751953125f, x);   // exact
  const float m = 0x1.7f7d1cp-20f, ml = 5.497923e-14f;
  const float p = n * m, pe = fmaf(n, m, -p);
  const Two r = two_sum(r0, -p) + (-(pe + n * ml));
  // Terms 6 .. 11.
  const float t = r.hi;
  float h = 1.f / 39916800.f;
  h = fmaf(h, t, 1.f / 3628800.f);
  h = fmaf(h, t, 1.f / 362880.f);
  h = fmaf(h, t, 1.f / 40320.f);
  h = fmaf(h, t, 1.f / 5040.f);
  h = fmaf(h, t, 1.f / 720.f);
  Two s = Two{h, 0.f} * r + Two{8.33333377e-03f, -4.34617203e-10f};   // 1 / 120
  s = s * r + Two{4.16666679e-02f, -1.24176344e-09f};                 // 1 / 24
  s = s * r + Two{1.66666672e-01f, -4.96705377e-09f};                 // 1 / 6
  s = s * r + 0.5f;
  s = s * r + 1.f;
  s = s * r + 1.f;
  // In two steps: 2^k may be below the least normal number.
  const int k = static_cast<int>(n), half = k / 2;
  const float p0 = none ? 0.f : power_of_two(half), p1 = power_of_two(k - half);
  return Two{s.hi * p0 * p1, s.lo * p0 * p1};
}

// e^(l - m) as a pair, for l and m of any size with l <= m; within 1.5 x 2^-40 of its value and 2^-148, 0 below -100.
XS_HD Two two_exp_diff(float l, float m) {
  // The exponential of the difference's upper part times that of the lower: 1 + r + r^2 / 2 for r up to 2^-18.
  const Two d = two_sum(l, -m);
  const float r = d.hi > -100.f ? d.lo : 0.f;
  return two_exp(fminf(d.hi, 0.f)) * quick_two(1.f, fmaf(0.5f * r, r, r));
}

// 1 / (1 + e^-x), within 2^-38 of its value and 2^-147; 0 for x below -100.
XS_HD Two two_sigmoid(float x) {
  const Two e = two_exp(-fabsf(x)), one = Two{1.f, 0.f};
  return (x >= 0.f ? one : e) / (e + 1.f);
}

}  // namespace xs
