// qat_few_kernels.h -- a few tokens through a dense weight matrix: the weights
// are read once, straight into operands of the matrix instructions.
#pragma once
#include "qat_common.h"

namespace bcjr {
namespace qlin {

template <class T>
struct Frag;   // eight weights or activations of a lane
template <>
struct Frag<bf16> {
  typedef bf16 type __attribute__((ext_vector_type(8)));
};
template <>
struct Frag<f16> {
  typedef f16 type __attribute__((ext_vector_type(8)));
};
template <>
struct Frag<float> {
  typedef float type __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ void mma16(const Frag<bf16>::type& a, const Frag<bf16>::type& b, f32x4& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma16(const Frag<f16>::type& a, const Frag<f16>::type& b, f32x4& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma16(const Frag<float>::type& a, const Frag<float>::type& b, f32x4& c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
}

constexpr int kFewWaves = 16;     // of a workgroup at most

// What both kernels of few tokens share: the layer's operands but the weights,
// and how a workgroup's waves are laid over it.
struct FewArgs {
  const void* x;
  int64_t ldx;
  const void* bias;
  const void* residual;
  int64_t ldr;
  void* y;
  int64_t ldy;
  int act;
  int M, N, K;
  int tiles;                 // tiles of 16 / Q rows
  int parts, at_once;        // waves along K and along tiles
};

// Lays the waves out: as many along K as there are units of it, then as many
// tiles as leave a workgroup for each CU.  Returns the number of workgroups.
inline int lay_out(FewArgs& a, int q, int units) {
  const int rows = 16 / q;
  a.tiles = (a.N + rows - 1) / rows;
  a.parts = 1;
  while (a.parts < kFewWaves && a.parts < units) a.parts *= 2;
  a.at_once = kFewWaves / a.parts;
  while (a.at_once > 1 && (a.tiles + a.at_once - 1) / a.at_once < 256) a.at_once /= 2;
  return (a.tiles + a.at_once - 1) / a.at_once;
}

// The waves' sums of 16 x 16 products (rows 4 g + i and column lane % 16 of a
// lane, g = lane / 16) through LDS, added in the order of K, and the epilogue,
// for tokens 16 m .. 16 m + 15 of the tiles from t0 on.
template <class T, int Q>
__device__ __forceinline__ void finish_few(const FewArgs& a, float* sums, const f32x4& acc, int t0, int m, int tid,
                                           int threads) {
  constexpr int kRowsOf = 16 / Q;
  const int lane = tid & 63, wave = tid >> 6;
  const T* bias = static_cast<const T*>(a.bias);
  const T* res = static_cast<const T*>(a.residual);
  T* y = static_cast<T*>(a.y);
  __syncthreads();
  *reinterpret_cast<f32x4*>(sums + wave * 256 + (lane & 15) * 16 + 4 * (lane >> 4)) = acc;
  __syncthreads();
  const int tokens = a.M - 16 * m < 16 ? a.M - 16 * m : 16;
  // neighbouring threads take neighbouring rows: a token's outputs are
  // contiguous, and so are its sums in LDS
  for (int o = tid; o < a.at_once * kRowsOf * 16; o += threads) {
    const int row = o % (a.at_once * kRowsOf), tok = o / (a.at_once * kRowsOf);
    const int q = row / kRowsOf, rr = row % kRowsOf, r = t0 * kRowsOf + row;
    if (tok >= tokens || t0 + q >= a.tiles || r >= a.N) continue;
    float z = 0.f;
    for (int p = 0; p < a.parts; ++p) {
      const float* s = sums + (q * a.parts + p) * 256;
      z += s[tok * 16 + rr];
      if (Q == 2) z += s[(tok + 8) * 16 + rr + 8];
    }
    if (bias) z += (float)bias[r];
    z = act_value(z, a.act);
    const int64_t m0 = 16 * m + tok;
    if (res) z += (float)res[m0 * a.ldr + r];
    y[m0 * a.ldy + r] = (T)z;
  }
}

// eight values at p of which n exist, zeros for the others
template <class T>
__device__ __forceinline__ typename Frag<T>::type eight(const T* p, int n) {
  typename Frag<T>::type v;
  if (n >= 8) {
    __builtin_memcpy(&v, p, sizeof(v));   // which need not be aligned
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) v[e] = p[e];
  }
  return v;
}

// y = act(x W^T + bias) + residual for up to 16 tokens: bound by reading W.
//
// A wave takes 16 / Q rows and 256 Q weights of each, all loads of which are
// under way at once (8 KB of 16-bit weights).  Lane l of a matrix instruction
// holds row l % 16 and eight k, which k is free: with Q = 1 lane group l / 16
// takes the next 16 bytes of 64 of a row, with Q = 2 (at most 8 tokens) rows
// 8..15 are the same rows 64 bytes on, so that a load takes whole 128-byte
// lines; tokens 8..15 are then the same tokens there, the products of unlike
// halves are not used, and half the rows a tile fill twice the CUs.  bf16, one
// token, 2048 x 8192: 8.2 us, 4.1 TB/s of weights.
template <class T, int Q>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(FewArgs a, const T* W, int64_t ldw) {
  using F = typename Frag<T>::type;
  constexpr int kRowsOf = 16 / Q, kUnit = 256 * Q;
  __shared__ __align__(16) float sums[kFewWaves * 256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int part = wave % a.parts, of = wave / a.parts;
  const int row = lane & 15, g = lane >> 4;
  const int t0 = blockIdx.x * a.at_once, tile = t0 + of;
  const T* x = static_cast<const T*>(a.x);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (tile < a.tiles) {
    int r = tile * kRowsOf + row % kRowsOf;
    r = r < a.N ? r : a.N - 1;
    // of this lane's row, and of its token
    const int k0 = (row / kRowsOf) * 32 + 8 * g, kx = (Q == 2 ? row >> 3 : 0) * 32 + 8 * g;
    const T* wr = W + r * ldw;
    int tok = Q == 2 ? lane & 7 : row;
    tok = tok < a.M ? tok : a.M - 1;
    const T* xr = x + tok * a.ldx;
    for (int u = part * kUnit; u < a.K; u += a.parts * kUnit) {
      F w[8];
      if (u + kUnit <= a.K) {
#pragma unroll
        for (int f = 0; f < 8; ++f) __builtin_memcpy(&w[f], wr + u + 32 * Q * f + k0, sizeof(F));
#pragma unroll
        for (int f = 0; f < 8; ++f) {
          F v;
          __builtin_memcpy(&v, xr + u + 32 * Q * f + kx, sizeof(F));
          mma16(w[f], v, acc);
        }
      } else {
#pragma unroll 1
        for (int f = 0; f < 8; ++f) {
          const int k = u + 32 * Q * f;
          mma16(eight<T>(wr + k + k0, a.K - k - k0), eight<T>(xr + k + kx, a.K - k - kx), acc);
        }
      }
    }
  }
  finish_few<T, Q>(a, sums, acc, t0, 0, tid, blockDim.x);
}

}  // namespace qlin
}  // namespace bcjr
