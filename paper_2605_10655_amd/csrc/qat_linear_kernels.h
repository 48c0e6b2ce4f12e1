// qat_linear_kernels.h -- kernels of the quantised linear layer: the product
// with bias, activation and residual in its epilogue, the 8-bit checkpoints of
// activations and their use in the backward pass, and trellis-coded weights.
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

// One thread per group: 32 rows of one column, read coalesced over the
// columns, 32 codes written as 32 contiguous bytes.
template <class T>
__global__ void act8_store_kernel(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ldx,
                                  int8_t* __restrict__ codes, uint16_t* __restrict__ scales) {
  const int64_t c = (int64_t)blockIdx.y * blockDim.x + threadIdx.x;
  const int64_t g = blockIdx.x;
  if (c >= cols) return;
  float v[kRows];
  float amax = 0.f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int64_t r = g * kRows + i;
    v[i] = r < rows ? (float)x[r * ldx + c] : 0.f;
    if (finite_bits(v[i]))
      amax = fmaxf(amax, fabsf(v[i]));
    else
      bad = true;
  }
  const Q8 q = q8_of(amax, kEmin<T>, kEmax<T>);
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w[i] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[i] |= (uint32_t)(q8_code(v[4 * i + j], q) & 255) << (8 * j);
  }
  const int64_t at = g * cols + c;
  u32x4* o = reinterpret_cast<u32x4*>(codes + at * kRows);
  o[0] = u32x4{w[0], w[1], w[2], w[3]};
  o[1] = u32x4{w[4], w[5], w[6], w[7]};
  scales[at] = q8_scale_bits(q, bad);
}

template <class T>
__global__ void act8_load_kernel(const int8_t* __restrict__ codes, const uint16_t* __restrict__ scales,
                                 int64_t rows, int64_t cols, T* __restrict__ out, int64_t ldo) {
  const int64_t c = (int64_t)blockIdx.y * blockDim.x + threadIdx.x;
  const int64_t g = blockIdx.x;
  if (c >= cols) return;
  const int64_t at = g * cols + c;
  const uint16_t s = scales[at];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int64_t r = g * kRows + i;
    if (r < rows) out[r * ldo + c] = (T)q8_value(codes[at * kRows + i], s);
  }
}

// ---------------------------------------------------------------- activations
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == kActSilu) return z / (1.f + expf(-z));
  if (act == kActGelu) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
  if (act == kActGeluTanh) {
    // 0.5 (1 + tanh u) = 1 / (1 + e^(-2u))
    const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
    return z / (1.f + expf(-2.f * u));
  }
  return z;
}

__device__ __forceinline__ float act_slope(float z, int act) {
  // far out the slope is 0 or 1; a NaN stays one
  z = z > 1e4f ? 1e4f : z;
  z = z < -1e4f ? -1e4f : z;
  if (act == kActSilu) {
    const float p = 1.f / (1.f + expf(-z));
    return p * (1.f + z * (1.f - p));
  }
  if (act == kActGelu)
    return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
  if (act == kActGeluTanh) {
    const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
    const float s = 1.f / (1.f + expf(-2.f * u));
    return s + 2.f * z * s * (1.f - s) * 0.79788456080286536f * (1.f + 0.134145f * z * z);
  }
  return 1.f;
}

// ---------------------------------------------------------------- product
// C[i, j] = sum_k A[i, k] B[j, k] for operands held as
//   row    element (r, k) at p[r * ld + k]
//   col    element (r, k) at p[k * ld + r]
//   codes  8-bit groups along k: [k / 32][R][32] with a scale per group
enum : int { kRow = 0, kCol = 1, kCodes = 2 };

struct GemmArgs {
  const void* a;
  const void* b;
  int64_t lda, ldb;
  const uint16_t* bscales;   // codes only
  int64_t I, J, K;
  // epilogue: z = C + bias, y = act(z) + residual, z's checkpoint
  const void* bias;
  const void* residual;
  int64_t ldr;
  void* y;
  int64_t ldy;
  int8_t* zcodes;
  uint16_t* zscales;
  int act;
};

template <class T>
__device__ __forceinline__ void mma(const typename Vec<T>::type& a, const typename Vec<T>::type& b, f32x16& c);
template <>
__device__ __forceinline__ void mma<bf16>(const Vec<bf16>::type& a, const Vec<bf16>::type& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
template <>
__device__ __forceinline__ void mma<f16>(const Vec<f16>::type& a, const Vec<f16>::type& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// the contraction's order is free: the four k of a lane's 16 bytes go to four
// instructions, paired with those of lane + 32
template <>
__device__ __forceinline__ void mma<float>(const Vec<float>::type& a, const Vec<float>::type& b, f32x16& c) {
#pragma unroll
  for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[s], b[s], c, 0, 0, 0);
}

// 16 bytes of the operand: k .. k + E - 1 of row r, zero outside
template <class T, int MODE>
__device__ __forceinline__ typename Vec<T>::type chunk_at(const void* p, int64_t ld, const uint16_t* scales,
                                                          int64_t R, int64_t K, int64_t r, int64_t k) {
  constexpr int E = kPer16<T>;
  typename Vec<T>::type v;
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = (T)0.f;
  if (r >= R) return v;
  if (MODE == kCodes) {
    const int64_t at = (k / kRows) * R + r;
    if (k < K) {
      const int8_t* q = static_cast<const int8_t*>(p) + at * kRows + (k % kRows);
      const uint16_t s = scales[at];
      // a group with a non-finite value counts as NaN whole: its column of
      // the gradient is not finite in either case
      const float f = (s & 0x8000u) ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)s << 16);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = (T)((float)q[e] * f);
    }
    return v;
  }
  const T* t = static_cast<const T*>(p);
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (k + e < K) v[e] = MODE == kRow ? t[r * ld + k + e] : t[(k + e) * ld + r];
  return v;
}

// 128 x 128 of C per workgroup of four waves (64 x 64 each, 2 x 2 matrix
// instructions of 32 x 32), 128 bytes of k per step.  LDS rows are 128 bytes;
// 16-byte chunk c of row r lies at place c ^ (r & 7), so that the lanes of a
// read (consecutive rows, one chunk) meet all banks.
constexpr int kTile = 128;

template <class T, int AM, int BM>
__global__ __launch_bounds__(256) void gemm_kernel(GemmArgs g) {
  constexpr int E = kPer16<T>;
  using V = typename Vec<T>::type;
  __shared__ V sa[kTile * 8], sb[kTile * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t i0 = (int64_t)blockIdx.x * kTile, j0 = (int64_t)blockIdx.y * kTile;
  const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
  f32x16 acc[2][2];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;
  for (int64_t k0 = 0; k0 < g.K; k0 += 8 * E) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = tid + 256 * i;
      const int ra = AM == kCol ? c & 127 : c >> 3, ca = AM == kCol ? c >> 7 : c & 7;
      const int rb = BM == kCol ? c & 127 : c >> 3, cb = BM == kCol ? c >> 7 : c & 7;
      sa[ra * 8 + (ca ^ (ra & 7))] = chunk_at<T, AM>(g.a, g.lda, nullptr, g.I, g.K, i0 + ra, k0 + ca * E);
      sb[rb * 8 + (cb ^ (rb & 7))] = chunk_at<T, BM>(g.b, g.ldb, g.bscales, g.J, g.K, j0 + rb, k0 + cb * E);
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      V fa[2], fb[2];
      const int c = 2 * kk + (lane >> 5);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int ra = wi + 32 * x + (lane & 31), rb = wj + 32 * x + (lane & 31);
        fa[x] = sa[ra * 8 + (c ^ (ra & 7))];
        fb[x] = sb[rb * 8 + (c ^ (rb & 7))];
      }
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) mma<T>(fa[x], fb[y], acc[x][y]);
    }
    __syncthreads();
  }
  // lane: column j = lane & 31 of its 32 x 32 tile, rows 8 (r / 4) + 4 (lane /
  // 32) + r % 4 for r = 0..15; the other 16 rows of a group of 32 are with
  // lane ^ 32
  const T* bias = static_cast<const T*>(g.bias);
  const T* res = static_cast<const T*>(g.residual);
  T* out = static_cast<T*>(g.y);
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int64_t ib = i0 + wi + 32 * x, j = j0 + wj + 32 * y + (lane & 31);
      const bool jin = j < g.J;
      const float b = bias && jin ? (float)bias[j] : 0.f;
      f32x16 z = acc[x][y];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int64_t i = ib + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
        z[r] = i < g.I ? z[r] + b : 0.f;
        if (i < g.I && jin) {
          float v = act_value(z[r], g.act);
          if (res) v += (float)res[i * g.ldr + j];
          out[i * g.ldy + j] = (T)v;
        }
      }
      if (g.zcodes && ib < g.I) {
        float amax = 0.f;
        int bad = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if (finite_bits(z[r]))
            amax = fmaxf(amax, fabsf(z[r]));
          else
            bad = 1;
        }
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        bad |= __shfl_xor(bad, 32);
        if (jin) {
          const Q8 q = q8_of(amax, kEmin<float>, kEmax<float>);
          const int64_t at = (ib / kRows) * g.J + j;
#pragma unroll
          for (int b4 = 0; b4 < 4; ++b4) {
            uint32_t w = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) w |= (uint32_t)(q8_code(z[4 * b4 + r], q) & 255) << (8 * r);
            *reinterpret_cast<uint32_t*>(g.zcodes + at * kRows + 8 * b4 + 4 * (lane >> 5)) = w;
          }
          if (lane < 32) g.zscales[at] = q8_scale_bits(q, bad != 0);
        }
      }
    }
}

// ---------------------------------------------------------------- backward
// dz = dy * act'(z8), rounded to T for the matrix instructions (half a step of
// the type each, as dy itself), and the sum of the unrounded dz over each
// group's rows.  One thread per group.
template <class T>
__global__ void dz_kernel(const T* __restrict__ dy, int64_t ldd, const int8_t* __restrict__ zcodes,
                          const uint16_t* __restrict__ zscales, int act, int64_t rows, int64_t cols,
                          T* __restrict__ dz, float* __restrict__ part) {
  const int64_t c = (int64_t)blockIdx.y * blockDim.x + threadIdx.x;
  const int64_t g = blockIdx.x;
  if (c >= cols) return;
  const int64_t at = g * cols + c;
  const uint16_t s = act != kActNone ? zscales[at] : (uint16_t)0;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int64_t r = g * kRows + i;
    if (r >= rows) break;
    float v = (float)dy[r * ldd + c];
    if (act != kActNone) {
      v *= act_slope(q8_value(zcodes[at * kRows + i], s), act);
      dz[r * cols + c] = (T)v;
    }
    sum += v;
  }
  if (part) part[at] = sum;
}

template <class T>
__global__ void dbias_kernel(const float* __restrict__ part, int64_t groups, int64_t cols, T* __restrict__ out) {
  const int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= cols) return;
  double s = 0.;
  for (int64_t g = 0; g < groups; ++g) s += (double)part[g * cols + c];
  out[c] = (T)(float)s;
}

// ---------------------------------------------------------------- trellis codes
// A path s_0 .. s_{steps-1} as a bit string, most significant bit first in
// 32-bit words: the n bits of s_0, then k bits a step.  The state after step t
// is the n-bit window at bit t k.
__device__ __forceinline__ uint32_t window(uint32_t hi, uint32_t lo, int off, int n) {
  const uint64_t w = ((uint64_t)hi << 32) | lo;
  return (uint32_t)(w >> (64 - off - n)) & ((1u << n) - 1u);
}

// One thread per word of the string.
__global__ void pack_kernel(const int32_t* __restrict__ states, int64_t B, int64_t steps, int n, int k,
                            int64_t words, uint32_t* __restrict__ packed) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= B * words) return;
  const int64_t b = i / words, w = i - b * words;
  const int32_t* s = states + b * steps;
  const int64_t bits = n + (steps - 1) * k;
  uint32_t v = 0;
  for (int j = 0; j < 32; ++j) {
    const int64_t p = w * 32 + j;   // bit p of the string
    uint32_t bit = 0;
    if (p < n) {
      bit = ((uint32_t)s[0] >> (n - 1 - p)) & 1u;
    } else if (p < bits) {
      const int64_t t = (p - n) / k + 1;
      bit = ((uint32_t)s[t] >> (k - 1 - (int)((p - n) % k))) & 1u;
    }
    v = (v << 1) | bit;
  }
  packed[i] = v;
}

// Counts the states that are out of range or do not follow their predecessor
// (whole numbers: the order of the additions is of no account).
__global__ void pack_check_kernel(const int32_t* __restrict__ states, int64_t B, int64_t steps, int n, int k,
                                  int32_t* __restrict__ illegal) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= B * steps) return;
  const uint32_t mask = (1u << n) - 1u, s = (uint32_t)states[i];
  bool bad = s > mask;
  if (i % steps) bad |= ((((uint32_t)states[i - 1] << k) ^ s) & mask) >> k;
  if (bad) atomicAdd(illegal, 1);
}

__global__ void zero_kernel(int32_t* p) { *p = 0; }

__global__ void unpack_kernel(const uint32_t* __restrict__ packed, int64_t B, int64_t steps, int n, int k,
                              int64_t words, int32_t* __restrict__ states) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= B * steps) return;
  const int64_t b = i / steps, at = (i - b * steps) * k;
  const int64_t j = at >> 5;
  const uint32_t* p = packed + b * words;
  states[i] = (int32_t)window(p[j], j + 1 < words ? p[j + 1] : 0u, (int)(at & 31), n);
}

// scale * codeword in fp32: kept from being fused with a conversion to fp16,
// so that every type rounds the same product
__device__ __forceinline__ float scaled(float scale, float c) {
  float p = scale * c;
  asm("" : "+v"(p));
  return p;
}

// W = scale * codebook[state] in fp32, rounded to T.  One thread per step.
template <class T>
__global__ void dense_kernel(const uint32_t* __restrict__ packed, const float* __restrict__ codebook,
                             const float* __restrict__ scales, int64_t B, int64_t steps, int n, int k, int V,
                             int64_t words, T* __restrict__ W) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= B * steps) return;
  const int64_t b = i / steps, at = (i - b * steps) * k;
  const int64_t j = at >> 5;
  const uint32_t* p = packed + b * words;
  const uint32_t s = window(p[j], j + 1 < words ? p[j + 1] : 0u, (int)(at & 31), n);
  const float f = scales ? scales[b] : 1.f;
  for (int v = 0; v < V; ++v) W[i * V + v] = (T)scaled(f, codebook[(int64_t)s * V + v]);
}

}  // namespace qlin
}  // namespace bcjr
