// expfix.cuh - softmax weights as 64-bit fixed-point integers.
//
// weight(z) = 2^46 * exp((z - max) / T) as an odd integer: off by at most 2^-46 of the
// largest weight and 2^-29.9 of itself; 0 below 2^-45.  (The roundings of f, 5 * 2^-25 at worst,
// are 2^-31.2 of the weight, the cubic's three 2^-30.8, the rest below 2^-35.  Of 56 million pairs
// the worst was off by 2^-30.9, the mean square 2^-33.7.)  Integers add up to the same sum in any order, so
// thousands of threads may sum them as they come and every comparison of sums (does this
// prefix hold p of the mass? does the running sum pass u times the total?) is exact; with
// 32-bit floating-point sums one draw in a few hundred lands within a rounding of a border
// between two ids (25 of 11232 in sampling.cu's kernel).  131072 weights stay below 2^63 + 2^17.
//
// exp by a table of 2^(i/256) and a cubic for the rest (the table-driven scheme of
// P. T. P. Tang, ACM TOMS 15 (1989)): 256 y = 256 (z - max) log2(e) / T = n + f with a whole
// n and |f| <= 1, where 2^(f/256) - 1 is below 2^-8, so that 24 bits of it are 32
// of the weight.  Some 30 instructions, none of them 64-bit floating point (2 a clock and SM here).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace memspec {

constexpr int kExpSteps = 256;
constexpr int kExpBits = 62;       // table entries: 2^62 * 2^(i/256)
constexpr int kWeightBits = 46;    // weight of the maximum: 2^46

struct ExpTable {
  unsigned long long v[kExpSteps];
};
// 2^(1/256) by eight square roots (Newton), its powers by products: 2^-45 at worst.
constexpr double newton_sqrt(double x) {
  double r = x;
  for (int i = 0; i < 60; ++i) r = 0.5 * (r + x / r);
  return r;
}
constexpr ExpTable make_exp_table() {
  ExpTable t{};
  double base = 2.0;
  for (int i = 0; i < 8; ++i) base = newton_sqrt(base);
  double x = 1.0;
  for (int i = 0; i < kExpSteps; ++i) {
    t.v[i] = static_cast<unsigned long long>(x * 4611686018427387904.0);   // 2^62
    x *= base;
  }
  return t;
}

// The table in device memory (kernels copy it to shared memory).
__device__ __forceinline__ const unsigned long long* exp_table() {
  static __device__ const ExpTable t = make_exp_table();
  return t.v;
}

// What weights need of a row: the maximum, and c = log2(e) / T.
struct WeightScale {
  float max;
  float scale;              // above T = 2^64: 2^-64, of logits and T alike, else 1
  float hi256, lo256;       // 256 c / scale in two floats
  bool near;                // 256 z c stays below 2^22 for the z that have weight: then also
  float f_max;              // 256 max c = n_max + f_max
  int n_max;
  float z_deep;             // and a logit without weight
  __device__ __forceinline__ float c() const { return hi256 * scale / kExpSteps; }   // for estimates
};
constexpr float kRound = 12582912.f;          // 1.5 * 2^23: x + kRound has round(x) in its low bits
constexpr int kRoundBits = 0x4B400000;
constexpr float kLowest = 1e-30f;             // temperatures above 0 count as this at least: 1 / T and
                                              // its lower part are normal numbers
constexpr int kNoWeight = -45 * kExpSteps;    // n at and below which the weight is 0
// Above T = 2^64 differences of logits that count may pass the largest float (infinities count
// as it, and masks may be of its negative) and c's lower part falls below the smallest one:
// logits and T are taken 2^-64 fold (exactly, but for logits below 2^-62, whose differences are
// no part of such a T), always the long way.
__device__ __forceinline__ float logit_scale(float temperature) {
  return temperature > 18446744073709551616.f ? 5.42101086e-20f : 1.f;
}
__device__ __forceinline__ WeightScale weight_scale(float row_max, float temperature) {
  // T from kLowest to inf (which weighs all alike).  A quotient and its remainder's in 32 bits:
  // 64-bit arithmetic by every thread of a CTA is 2 us.
  constexpr float kHi = 1.44269504f, kLo = 1.92596299e-8f;   // log2(e)
  WeightScale s;
  s.max = row_max;
  s.scale = logit_scale(temperature);
  const float T = temperature * s.scale;
  const float hi = __fdiv_rn(kHi, T), lo = hi > 0.f ? __fdiv_rn(fmaf(-hi, T, kHi) + kLo, T) : 0.f;
  s.hi256 = hi * kExpSteps;
  s.lo256 = lo * kExpSteps;
  s.near = s.scale == 1.f && fabsf(row_max) * s.hi256 < 4e6f;
  const float big = fmaf(row_max, s.hi256, kRound);
  s.n_max = __float_as_int(big) - kRoundBits;
  s.f_max = fmaf(row_max, s.lo256, fmaf(row_max, s.hi256, kRound - big));
  s.z_deep = row_max - 47.f / hi;
  return s;
}

// The whole part n of 256 (z - max) c and the rest f, z finite or -inf and z <= s.max;
// n <= kNoWeight: no weight.  n grows with z (each step is monotonic).
__device__ __forceinline__ int place_near(float z, const WeightScale& s, float& f) {
  // 256 z c less 256 max c, part by part
  z = fmaxf(z, s.z_deep);
  const float big = fmaf(z, s.hi256, kRound);
  f = fmaf(z, s.lo256, fmaf(z, s.hi256, kRound - big)) - s.f_max;
  return __float_as_int(big) - (kRoundBits + s.n_max);
}
__device__ __forceinline__ int place_far(float z, const WeightScale& s, float& f) {
  // the difference first: max - z = d + e exactly (two-sum)
  const float top = s.max * s.scale;
  z *= s.scale;
  const float d = top - z;
  const float b = d - top;
  const float e = (top - (d - b)) - (z + b);
  const float yh = d * s.hi256;
  const float yl = fmaf(d, s.hi256, -yh) + fmaf(d, s.lo256, e * s.hi256);
  const float big = kRound - yh;
  f = ((kRound - big) - yh) - yl;
  return yh < 46.f * kExpSteps ? __float_as_int(big) - kRoundBits : 2 * kNoWeight;
}
__device__ __forceinline__ int weight_place(float z, const WeightScale& s, float& f) {
  return s.near ? place_near(z, s, f) : place_far(z, s, f);
}
// Several at once: one branch, and their arithmetic interleaves.
template <int N>
__device__ __forceinline__ void weight_places(const float (&z)[N], const WeightScale& s, int (&n)[N], float (&f)[N]) {
  if (s.near) {
#pragma unroll
    for (int q = 0; q < N; ++q) n[q] = place_near(z[q], s, f[q]);
  } else {
#pragma unroll
    for (int q = 0; q < N; ++q) n[q] = place_far(z[q], s, f[q]);
  }
}
__device__ __forceinline__ unsigned long long weight_at(int n, float f, const unsigned long long* table) {
  constexpr double kLn = 0.693147180559945 / kExpSteps, kScale = 549755813888.0;   // 2^39
  // 2^39 (2^(f/256) - 1), the parenthesis below 0.0028
  const float p = fmaf(fmaf(f, static_cast<float>(kScale * kLn * kLn * kLn / 6), static_cast<float>(kScale * kLn * kLn / 2)),
                       f, static_cast<float>(kScale * kLn)) * f;
  const unsigned long long t = table[n & (kExpSteps - 1)];          // [2^62, 2^63)
  // t times that: its upper half times p, in units of 2^25
  const long long r = static_cast<long long>(__mulhi(static_cast<int>(t >> 32), __float2int_rn(p)));
  const unsigned long long w = t + static_cast<unsigned long long>(r * (1ll << 25));
  // 2 floor(x / 2) + 1 is x in the mean, so that truncation adds no drift to a long sum
  return n > kNoWeight ? (w >> (kExpBits - kWeightBits - (n >> 8))) | 1u : 0;
}
__device__ __forceinline__ unsigned long long weight(float z, const WeightScale& s, const unsigned long long* table) {
  float f;
  const int n = weight_place(z, s, f);
  return weight_at(n, f, table);
}

// The float order of logits as unsigned keys (-0 as +0).
__device__ __forceinline__ uint32_t logit_key(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  return __uint_as_float(k ^ ((k & 0x80000000u) ? 0x80000000u : 0xFFFFFFFFu));
}

// floor(f 2^64) of f in [0, 1), exact down to 2^-64; f >= 1: 2^64 - 1; f <= 0 or NaN: 0.
__device__ __forceinline__ unsigned long long fraction64(float f) {
  if (!(f > 0.f)) return 0;
  if (f >= 1.f) return ~0ull;
  const uint32_t b = __float_as_uint(f);
  const int ex = static_cast<int>(b >> 23);               // f = m 2^(ex - 150)
  const unsigned long long m = ex ? (b & 0x7FFFFFu) | 0x800000u : b & 0x7FFFFFu;
  const int sh = (ex ? ex : 1) - 150 + 64;
  return sh >= 0 ? m << sh : (sh > -64 ? m >> -sh : 0);
}

}  // namespace memspec
