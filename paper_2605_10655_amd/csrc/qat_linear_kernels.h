// qat_linear_kernels.h -- kernels around the product of the quantised linear
// layer: the 8-bit checkpoints of activations, the gradient of its
// pre-activation, and trellis-coded weights.
#pragma once
#include "qat_common.h"

namespace bcjr {
namespace qlin {

// ---------------------------------------------------------------- 8-bit checkpoints
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
