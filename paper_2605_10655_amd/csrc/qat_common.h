// qat_common.h -- what the kernels of the quantised linear layer share: types,
// 8-bit groups, activations.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bcjr {
namespace qlin {

enum : int { kF32 = 0, kBF16 = 1, kF16 = 2 };
enum : int { kActNone = 0, kActSilu = 1, kActGelu = 2, kActGeluTanh = 3 };

using bf16 = __bf16;
using f16 = _Float16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <class T>
struct Vec;  // 16 bytes of T
template <>
struct Vec<bf16> {
  typedef bf16 type __attribute__((ext_vector_type(8)));
};
template <>
struct Vec<f16> {
  typedef f16 type __attribute__((ext_vector_type(8)));
};
template <>
struct Vec<float> {
  typedef float type __attribute__((ext_vector_type(4)));
};
template <class T>
constexpr int kPer16 = 16 / (int)sizeof(T);  // values of T in 16 bytes

// ---------------------------------------------------------------- 8-bit groups
// A group is 32 rows (tokens) of one column, with a power of two 2^e as its
// scale: the smallest with amax <= 127 * 2^e.  q * 2^e is then exact in bf16
// and, with e bounded below by the type's smallest step, in fp16, so the
// matrix instructions of the backward pass read the checkpoint's values
// unrounded.  Where the scale would carry code 64 past the type's largest
// value the code stops at 63.
constexpr int kRows = 32;

struct Q8 {
  float inv;   // 2^-e
  float top;   // largest code
  int e;
};

__device__ __forceinline__ bool finite_bits(float v) {
  return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u;
}

// emin, emax: -24, 10 for fp16 (its smallest step; 64 * 2^10 is past its
// largest value), -126, 122 otherwise
__device__ __forceinline__ Q8 q8_of(float amax, int emin, int emax) {
  // amax = m 2^p: e = p - 6 where m <= 127 / 64, else p - 5 (the addition
  // carries into the exponent exactly there)
  int e = (int)((__float_as_uint(amax) + 0x1ffffu) >> 23) - 133;
  e = e < emin ? emin : e;
  Q8 q;
  q.e = e;
  q.inv = __uint_as_float((uint32_t)(127 - e) << 23);
  q.top = e >= emax ? 63.f : 127.f;
  return q;
}

__device__ __forceinline__ int q8_code(float v, const Q8& q) {
  if (!finite_bits(v)) return -128;
  return (int)fminf(fmaxf(rintf(v * q.inv), -q.top), q.top);
}

// Whether a group whose largest magnitude has these bits is finite and below
// the codes' cut at 63: then no value needs a bound of its own, as |v| <= 127 *
// 2^e.
__device__ __forceinline__ bool q8_plain(uint32_t top, int emax) {
  return top < 0x7f800000u && (int)((top + 0x1ffffu) >> 23) - 133 < emax;
}

// Four codes of such a group: v / 2^e is exact, and added to 1.5 * 2^23 it is
// rounded half to even into the low bits.
__device__ __forceinline__ uint32_t q8_codes4(float a, float b, float c, float d, float inv) {
  const float m = 12582912.f;
  const uint32_t x = __float_as_uint(__builtin_fmaf(a, inv, m)), y = __float_as_uint(__builtin_fmaf(b, inv, m));
  const uint32_t z = __float_as_uint(__builtin_fmaf(c, inv, m)), w = __float_as_uint(__builtin_fmaf(d, inv, m));
  // bytes 0 of both operands side by side, then the two halves
  const uint32_t lo = __builtin_amdgcn_perm(y, x, 0x0c0c0400u), hi = __builtin_amdgcn_perm(w, z, 0x04000c0cu);
  return lo | hi;
}

// the scale's bf16 bits; negative where the group holds a non-finite value
__device__ __forceinline__ uint16_t q8_scale_bits(const Q8& q, bool bad) {
  return (uint16_t)(((uint32_t)(q.e + 127) << 7) | (bad ? 0x8000u : 0u));
}

// value of a code, given the scale's bits
__device__ __forceinline__ float q8_value(int code, uint16_t sbits) {
  const float s = __uint_as_float((uint32_t)(sbits & 0x7fffu) << 16);
  return code == -128 ? __uint_as_float(0x7fc00000u) : (float)code * s;
}

template <class T>
constexpr int kEmin = sizeof(T) == 2 && !__is_same(T, bf16) ? -24 : -126;
template <class T>
constexpr int kEmax = sizeof(T) == 2 && !__is_same(T, bf16) ? 10 : 122;

// ---------------------------------------------------------------- activations
// 1 / (1 + e^-z) by the exponential and reciprocal instructions (a step off
// each); 0 and 1 far out
__device__ __forceinline__ float logistic(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}

// The normal distribution's Phi(z), and e = exp(-z^2 / 2): Phi(-|z|) = erfc(|z|
// / sqrt 2) / 2 by the polynomial of Abramowitz & Stegun 7.1.26 (erf within
// 1.5e-7), without a branch.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * 0.70710678118654752f * fabsf(z));
  e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
  const float q = 0.5f * e * t *
                  (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
  return z < 0.f ? q : 1.f - q;
}

__device__ __forceinline__ float act_value(float z, int act) {
  if (act == kActSilu) return z * logistic(z);
  if (act == kActGelu) {
    float e;
    return z * normal_cdf(z, e);
  }
  if (act == kActGeluTanh) {
    // 0.5 (1 + tanh u) = 1 / (1 + e^(-2u))
    const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
    return z * logistic(2.f * u);
  }
  return z;
}

__device__ __forceinline__ float act_slope(float z, int act) {
  // far out the slope is 0 or 1; a NaN stays one
  z = z > 1e4f ? 1e4f : z;
  z = z < -1e4f ? -1e4f : z;
  if (act == kActSilu) {
    const float p = logistic(z);
    return p * (1.f + z * (1.f - p));
  }
  if (act == kActGelu) {
    float e;
    const float p = normal_cdf(z, e);
    return p + z * e * 0.39894228040143268f;
  }
  if (act == kActGeluTanh) {
    const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
    const float s = logistic(2.f * u);
    return s + 2.f * z * s * (1.f - s) * 0.79788456080286536f * (1.f + 0.134145f * z * z);
  }
  return 1.f;
}

// scale * c in fp32: kept from being fused with what follows (a conversion to
// fp16, a sum), so that every type and kernel rounds the same product
__device__ __forceinline__ float scaled(float scale, float c) {
  float p = scale * c;
  asm("" : "+v"(p));
  return p;
}

}  // namespace qlin
}  // namespace bcjr
