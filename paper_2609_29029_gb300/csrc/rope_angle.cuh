// Cosine and sine of a position times a frequency, without double arithmetic on the device.
//
// A GB300 SM retires about two double operations a cycle, and a rotation of few heads has more angles than
// that hides (4,091 rows of 16 pairs: 14.5 us, 5.1 of them the bytes').  So the angle is taken as a fraction of a turn in
// 64-bit fixed point: the host gives f = 2^64 w / 2 pi (mod 2^64), and p f mod 2^64 is the fraction at any int32
// position p, exact but for f's own rounding to the nearest (of which p takes p pi 2^-64, below p 2^-62, into the
// angle), with its quadrant in the top bits.  What is left, |x| <= pi / 4,
// goes through the Taylor polynomials of sine and cosine, whose leading steps run on unevaluated sums of two fp32
// values (Dekker's and Knuth's error-free sum and product): about 100 fp32 operations, good to 2^-34.
#pragma once

#include <algorithm>

#include "rift_common.cuh"

namespace rift {

#ifdef __CUDA_ARCH__
__device__ __forceinline__ float rn_mul(float a, float b) { return __fmul_rn(a, b); }
__device__ __forceinline__ float rn_add(float a, float b) { return __fadd_rn(a, b); }
#else
inline float rn_mul(float a, float b) {
  volatile float p = a * b;  // volatile: no contraction into a fused operation
  return p;
}
inline float rn_add(float a, float b) {
  volatile float s = a + b;
  return s;
}
#endif

struct Float2Sum {  // the value hi + lo
  float hi, lo;
};
__host__ __device__ __forceinline__ Float2Sum fs_mul(Float2Sum a, Float2Sum b) {
  const float p = rn_mul(a.hi, b.hi);
  return {p, fmaf(a.hi, b.lo, fmaf(a.lo, b.hi, fmaf(a.hi, b.hi, -p)))};
}
// c - a, |c| >= |a|.
__host__ __device__ __forceinline__ Float2Sum fs_from(Float2Sum c, Float2Sum a) {
  const float s = rn_add(c.hi, -a.hi);
  return {s, rn_add(rn_add(rn_add(c.hi, -s), -a.hi), rn_add(c.lo, -a.lo))};
}

// (cos, sin) of 2 pi turns / 2^64, times `amplitude`, each rounded once to fp32.
__host__ __device__ __forceinline__ float2 cos_sin_of_turns(uint64_t turns, Float2Sum amplitude) {
  const uint64_t quadrant = (turns + (1ull << 61)) >> 62;
  const long long r = (long long)(turns - (quadrant << 62));  // |r| <= 2^61
  const float a = (float)r, b = (float)(r - (long long)a);
  // x = r 2 pi / 2^64
  const Float2Sum k = {0x1.921fb6p-62f, -0x1.777a5cp-87f};
  Float2Sum x = {rn_mul(a, k.hi), 0.f};
  x.lo = fmaf(a, k.lo, fmaf(b, k.hi, fmaf(a, k.hi, -x.hi)));
  const Float2Sum z = fs_mul(x, x);
  // sin x = x - x z (1/6 - z (1/120 - z (1/5040 - z (1/9! - z / 11!))))
  float t = fmaf(z.hi, -1.f / 39916800.f, 1.f / 362880.f);
  t = fmaf(-z.hi, t, 1.f / 5040.f);
  Float2Sum q = fs_from({0x1.111112p-7f, -0x1.ddddep-32f}, fs_mul(z, {t, 0.f}));
  q = fs_from({0x1.555556p-3f, -0x1.555556p-28f}, fs_mul(z, q));
  const Float2Sum s = fs_from(x, fs_mul(fs_mul(x, z), q));
  // cos x = 1 - z (1/2 - z (1/24 - z (1/720 - z (1/8! - z (1/10! - z / 12!)))))
  t = fmaf(z.hi, -1.f / 479001600.f, 1.f / 3628800.f);
  t = fmaf(-z.hi, t, 1.f / 40320.f);
  t = fmaf(-z.hi, t, 1.f / 720.f);
  q = fs_from({0x1.555556p-5f, -0x1.555556p-30f}, fs_mul(z, {t, 0.f}));
  q = fs_from({0.5f, 0.f}, fs_mul(z, q));
  const Float2Sum c = fs_from({1.f, 0.f}, fs_mul(z, q));
  const Float2Sum& u = quadrant & 1 ? s : c;
  const Float2Sum& v = quadrant & 1 ? c : s;
  auto times = [&](const Float2Sum& x) {
    const float p = rn_mul(x.hi, amplitude.hi);
    return rn_add(p, fmaf(x.hi, amplitude.lo, fmaf(x.lo, amplitude.hi, fmaf(x.hi, amplitude.hi, -p))));
  };
  const float cosine = times(u), sine = times(v);
  return make_float2((quadrant + 1) & 2 ? -cosine : cosine, quadrant & 2 ? -sine : sine);
}

// 2^64 w / 2 pi modulo 2^64 for 0 <= w <= 2^31 (host), to the nearest integer: w's product with 1 / 2 pi as an unevaluated
// sum of two doubles, p + e.  Whole turns leave p, whole units of 2^-64 turns what is left of it (both exactly), and only
// the rest, with e, is rounded.
inline uint64_t turns_of(double w) {
  const double inv = 0.15915494309189535, rest = -9.839338337591243e-18;
  const double p = w * inv, e = (std::fma(w, inv, -p) + w * rest) * 0x1p64;
  const double fraction = (p - std::floor(p)) * 0x1p64, units = std::floor(fraction);
  return (uint64_t)units + (uint64_t)(long long)std::floor(e + (fraction - units) + 0.5);
}

// w_j of a rotation's pairs j < rot_dim / 2 (host).  theta^(-2j / rot_dim) is a product of two powers, each rounded once: a
// call has 16 to 24 of them to take, not 64 to 128.  The exponents' rounding is |ln theta| 2^-53 of w together, the powers'
// (an ulp each) and the product's 5 2^-53 more, the factor's one.
inline void rope_frequencies(const rift_rope_spec& s, double* w) {
  double fine[8], coarse = 1.0;
  for (int i = 0; i < 8; ++i) fine[i] = i == 0 ? 1.0 : std::pow(s.theta, -2.0 * i / s.rot_dim);
  for (int j = 0; j < s.rot_dim / 2; ++j) {
    if (j % 8 == 0 && j > 0) coarse = std::pow(s.theta, -2.0 * j / s.rot_dim);
    w[j] = coarse * fine[j % 8];
    if (s.scaling == RIFT_ROPE_LINEAR) w[j] /= s.factor;
    if (s.scaling == RIFT_ROPE_PARTS) {
      const double turns = s.orig_len * w[j] / 6.283185307179586;
      const double g = std::min(1.0, std::max(0.0, (turns - s.low) / (s.high - s.low)));
      w[j] *= g + (1.0 - g) / s.factor;
    }
  }
}

}  // namespace rift
