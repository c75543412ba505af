// Scores of rows (any storage format) as ordered keys, and their weights in fp64.
#pragma once

#include "common.h"

namespace gs {
namespace {

struct ScoreF32 {
  typedef float elem;
  static constexpr uint32_t kNone = 0xff800000u;      // -infinity
  static __device__ __forceinline__ float get(float x) { return x; }
};
template <typename H>
struct ScoreHalf {
  typedef uint16_t elem;
  static constexpr uint32_t kNone = H::kNone;         // -infinity, twice
  static __device__ __forceinline__ float get(uint16_t x) { return H::lo(x); }
  static __device__ __forceinline__ float get_of(uint32_t word, int which) { return which ? H::hi(word) : H::lo(word); }
};

// 0: left out (-infinity or NaN); otherwise larger keys for larger scores, one key for both zeros
__device__ __forceinline__ uint32_t key_of(float s) {
  if (!(s > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(s == 0.0f ? 0.0f : s);
  return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float score_of(uint32_t key) {
  return __uint_as_float((key >> 31) ? (key & 0x7fffffffu) : ~key);
}

// exp((s - top) / temperature) as 2^(n / 64) 2^r, r within 1/128: a table of 64 powers in LDS and the series of 2^r to r^5
// (the next term is below 2^-54).  Half the instructions of exp(), which would bound the passes that weigh every score: about
// 2^-51 (1 + |exponent|) of relative error, most of it the exponent's own rounding, as with exp().
constexpr int kPowers = 64;
struct Weigh {
  double top, rate;                            // log2(e) / temperature
  const double* powers;                        // 2^(j / 64)
  __device__ __forceinline__ Weigh(float top_, float temperature, const double* powers_)
      : top((double)top_), rate(fmax(1.4426950408889634074 / (double)temperature, 0x1p-900)), powers(powers_) {}
  __device__ __forceinline__ double operator()(float s) const {     // without branches: they would split every wave
    // infinities: NaN for the greatest, which fmin takes to 0, -infinity for the others
    const double y = fmax(fmin(((double)s - top) * rate, 0.0), -2000.0);
    const double t = fma(y, (double)kPowers, 0x1.8p52);              // its last bits: the nearest whole number
    const double r = fma(t - 0x1.8p52, -1.0 / kPowers, y);
    const int n = __double2loint(t);
    const double power = powers[n & (kPowers - 1)];
    constexpr double l = 0.69314718055994530942, l2 = l * l, l3 = l2 * l, l4 = l2 * l2, l5 = l4 * l;
    double q = fma(r, l5 / 120, l4 / 24);
    q = fma(r, q, l3 / 6);
    q = fma(r, q, l2 / 2);
    q = fma(r, q, l) * r;
    return ldexp(fma(power, q, power), n >> 6);
  }
};
// by the first wave; a barrier follows before the first use
__device__ __forceinline__ void fill_powers(double* powers) {
  static_assert(kPowers == 64, "one per lane");
  if (threadIdx.x < kPowers) powers[threadIdx.x] = exp2((double)threadIdx.x / kPowers);
}

}  // namespace
}  // namespace gs
