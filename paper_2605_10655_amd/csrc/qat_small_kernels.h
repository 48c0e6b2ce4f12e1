// qat_small_kernels.h -- small layers, where launches are what counts: one
// launch each, in fp32 throughout.
#pragma once
#include "qat_few_kernels.h"

namespace bcjr {
namespace qlin {

// ---------------------------------------------------------------- backward
// v *= act'(z)
__device__ __forceinline__ void slopes(Frag<float>::type& v, const Frag<float>::type& z, int act) {
  if (act == kActSilu) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = scaled(act_slope(z[e], kActSilu), v[e]);
  } else if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = scaled(act_slope(z[e], kActGelu), v[e]);
  } else if (act == kActGeluTanh) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = scaled(act_slope(z[e], kActGeluTanh), v[e]);
  }
}

struct SmallVjp {
  const void* dy;
  int64_t ldd;
  const int8_t* xq;
  const uint16_t* xs;
  const void* W;
  int64_t ldw;
  const int8_t* zq;
  const uint16_t* zs;
  int act;
  int M, N, K;
  void *dx, *dW, *dbias;     // null where not wanted
  int xparts, wparts;        // waves along the sums of dx and of dW
  int xblocks;               // workgroups of dx; dW's and dbias's follow
};

// dx = dz W, dW = dz^T x and dbias = the columns' sums of dz = dy * act'(z), in
// one launch.  A wave takes 16 x 16 outputs and each workgroup's waves split
// the sum as well; dz is worked out anew for every tile, 32 of its values a
// row at a time, and goes into fp32 matrix instructions unrounded (lane l: row
// l % 16, the eight of the 32 from 8 (l / 16) on).  What bounds it is the
// latency of a launch and of two dependent loads, and the CU's address unit,
// which takes a value a lane and load.  us, against dz, dbias and the two
// products in a launch each: 64 x 64 x 64 5.5 and 18.7, 64 x 256 x 256 6.2 and
// 19.4, 16 x 512 x 512 9.1 and 16.9, 1 x 1024 x 1024 13.0 and 15.5; with sums
// of 4096 terms both take 25, and past 2^22 products dz's repetition counts.
template <class T>
__global__ __launch_bounds__(64 * kFewWaves) void vjp_small_kernel(SmallVjp a) {
  using F = Frag<float>::type;
  __shared__ __align__(16) float sums[kFewWaves * 256];
  __shared__ double columns[kFewWaves * 16];
  const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 63, wave = tid >> 6;
  const int row = lane & 15, g = lane >> 4;
  const bool is_x = (int)blockIdx.x < a.xblocks;
  const int parts = is_x ? a.xparts : a.wparts, at_once = (threads >> 6) / parts;
  const int R = is_x ? a.M : a.N, C = is_x ? a.N : a.M;   // rows of the output, terms of a sum
  const int ktiles = is_x || a.dW ? (a.K + 15) / 16 : 1, tiles = (R + 15) / 16 * ktiles;
  const int t0 = ((int)blockIdx.x - (is_x ? 0 : a.xblocks)) * at_once;
  const int tile = t0 + wave / parts < tiles ? t0 + wave / parts : tiles - 1;
  const int r0 = tile / ktiles * 16, k0 = tile % ktiles * 16;
  const int r = r0 + row < R ? r0 + row : R - 1, k = k0 + row < a.K ? k0 + row : a.K - 1;
  const T* dy = static_cast<const T*>(a.dy);
  const T* W = static_cast<const T*>(a.W);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  double column = 0.;
  for (int c0 = 32 * (wave % parts); c0 < C; c0 += 32 * parts) {
    const int c = c0 + 8 * g;
    // all loads before the first use of one
    F v, w, z;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = w[e] = 0.f;
    if (is_x) {
      // row r of dz, columns c .. c + 7
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int n = c + e < C ? c + e : C - 1;
        v[e] = (float)dy[r * a.ldd + n];
        w[e] = (float)W[n * a.ldw + k];
      }
      if (a.act != kActNone) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int n = c + e < C ? c + e : C - 1, o = (r / kRows) * a.N + n;
          z[e] = q8_value(a.zq[o * kRows + r % kRows], a.zs[o]);
        }
      }
    } else {
      // column r of dz, rows c .. c + 7 (all of one group of 32)
      const int first = c < C ? c : 0, o = (first / kRows) * a.N + r, p = (first / kRows) * a.K + k;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float)dy[(c + e < C ? c + e : C - 1) * a.ldd + r];
      if (a.dW) {
        int8_t q[8];
        __builtin_memcpy(q, __builtin_assume_aligned(a.xq + p * kRows + first % kRows, 8), 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = q8_value(q[e], a.xs[p]);
      }
      if (a.act != kActNone) {
        int8_t q[8];
        __builtin_memcpy(q, __builtin_assume_aligned(a.zq + o * kRows + first % kRows, 8), 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = q8_value(q[e], a.zs[o]);
      }
    }
    slopes(v, z, a.act);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e >= C) v[e] = w[e] = 0.f;
    mma16(v, w, acc);
    if (!is_x && k0 == 0) {
      // the sum of a group's 32 rows, by eights
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[e];
      s += __shfl_xor(s, 16);
      s += __shfl_xor(s, 32);
      column += (double)s;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sums[wave * 256 + (4 * g + i) * 16 + row] = acc[i];
  if (g == 0) columns[wave * 16 + row] = column;
  __syncthreads();
  T* out = static_cast<T*>(is_x ? a.dx : a.dW);
  for (int o = tid; o < at_once * 256; o += threads) {
    const int q = o >> 8, t = t0 + q;
    const int rr = t / ktiles * 16 + (o >> 4 & 15), kk = t % ktiles * 16 + (o & 15);
    if (t >= tiles || rr >= R) continue;
    if (out && kk < a.K) {
      float z = 0.f;
      for (int p = 0; p < parts; ++p) z += sums[(q * parts + p) * 256 + (o & 255)];
      out[(int64_t)rr * a.K + kk] = (T)z;
    }
    if (!is_x && a.dbias && kk == 0) {
      double s = 0.;
      for (int p = 0; p < parts; ++p) s += columns[(q * parts + p) * 16 + (o >> 4 & 15)];
      static_cast<T*>(a.dbias)[rr] = (T)(float)s;
    }
  }
}

// ---------------------------------------------------------------- codes
struct SmallCodes : FewArgs {
  const uint32_t* packed;
  const float* codebook;
  const float* scales;       // [N, K / block] or null
  int n, k, V, block, words;
};

// y = act(x W^T + bias) + residual for up to MT tokens and any trellis.
//
// A wave takes 512 weights of one row, eight a lane: scale * codebook[state] in
// fp32 with codewords from L2, multiplied with each token's in fp32.  The
// random reads of codewords bound it (1.1 cycles a weight and CU); with a row a
// wave and not 16, they spread over all CUs.  The lanes' sums are halved by
// exchange, so that 16 tokens take 17 exchanges and not 96.
//
// us (bf16, 16 state bits, 2 bits a step) for 1 and 16 tokens: 256 x 256 4.1
// and 7.3, 1024 x 1024 7.3 and 11.6.  Decoding into a dense matrix first takes
// 6.1 and 6.1, 19.8 and 19.8; a table in LDS 33.8 and 34.0, 18.2 and 11.4.
// With 12 state bits the table takes 4.7 for either at 1024 x 1024, this 5.1 and
// 9.7.  (fp32, more than 4 tokens: 54 of the 16 tokens' registers lie in scratch;
// 1024 x 1024 takes 20.2.)
constexpr int kSmallUnit = 512;

template <class T, int MT>
__global__ __launch_bounds__(64 * kFewWaves) void codes_small_kernel(SmallCodes a) {
  using F = Frag<float>::type;
  __shared__ float sums[kFewWaves * MT];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, part = wave % a.parts;
  const int r = blockIdx.x * a.at_once + wave / a.parts;
  const T* x = static_cast<const T*>(a.x);
  const int paths = a.K / a.block, last = (r + 1) * paths - 1;
  const float* scales = a.scales ? a.scales : a.codebook;   // read in any case, for a load without a branch
  const int any = a.scales ? -1 : 0;
  float acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = 0.f;
  if (r < a.N)
    for (int c = part * kSmallUnit + 8 * lane; c < a.K; c += a.parts * kSmallUnit) {
      // path, step and place in the step of weight c, then the windows of all
      // eight, then their codewords
      int path = r * paths + c / a.block, at = c % a.block;
      int step = at / a.V, v = at % a.V;
      uint32_t hi[8], lo[8];
      int off[8], place[8];
      F f, w;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int bit = step * a.k, j = bit >> 5;
        const int64_t p = (int64_t)path * a.words;
        hi[e] = a.packed[p + j];
        lo[e] = a.packed[p + (j + 1 < a.words ? j + 1 : j)];
        f[e] = scales[path & any];
        off[e] = bit & 31;
        place[e] = v;
        const bool next = ++v == a.V, end = ++at == a.block;
        v = next ? 0 : v;
        step = end ? 0 : next ? step + 1 : step;
        at = end ? 0 : at;
        path = end && path < last ? path + 1 : path;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t s = (uint32_t)((((uint64_t)hi[e] << 32 | lo[e]) << off[e]) >> (64 - a.n));
        w[e] = a.codebook[s * a.V + place[e]];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = c + e < a.K ? scaled(a.scales ? f[e] : 1.f, w[e]) : 0.f;
      constexpr int kMost = sizeof(T) == 4 ? 4 : 8, kAtOnce = MT < kMost ? MT : kMost;   // tokens loaded together
#pragma unroll
      for (int m0 = 0; m0 < MT; m0 += kAtOnce) {
        typename Frag<T>::type t[kAtOnce];
        if (c + 8 <= a.K) {
#pragma unroll
          for (int m = 0; m < kAtOnce; ++m)
            __builtin_memcpy(&t[m], x + (m0 + m < a.M ? m0 + m : a.M - 1) * a.ldx + c, sizeof(t[m]));
        } else {
#pragma unroll
          for (int m = 0; m < kAtOnce; ++m) t[m] = eight<T>(x + (m0 + m < a.M ? m0 + m : a.M - 1) * a.ldx + c, a.K - c);
        }
#pragma unroll
        for (int m = 0; m < kAtOnce; ++m)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[m0 + m] = __builtin_fmaf(w[e], (float)t[m][e], acc[m0 + m]);
      }
    }
  // lanes l and l ^ w keep half of the tokens each and add the other's share
  int token = 0, width = 32;
#pragma unroll
  for (int n = MT / 2; n >= 1; n /= 2, width /= 2) {
    const bool up = lane & width;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float give = up ? acc[i] : acc[i + n];
      acc[i] = (up ? acc[i + n] : acc[i]) + __shfl_xor(give, width);
    }
    token += up ? n : 0;
  }
  for (; width >= 1; width /= 2) acc[0] += __shfl_xor(acc[0], width);
  if (lane % (64 / MT) == 0) sums[wave * MT + token] = acc[0];
  __syncthreads();
  for (int o = tid; o < a.at_once * MT; o += blockDim.x) {
    const int q = o % a.at_once, m = o / a.at_once, n = blockIdx.x * a.at_once + q;
    if (m >= a.M || n >= a.N) continue;
    float z = 0.f;
    for (int p = 0; p < a.parts; ++p) z += sums[(q * a.parts + p) * MT + m];
    if (a.bias) z += (float)static_cast<const T*>(a.bias)[n];
    z = act_value(z, a.act);
    if (a.residual) z += (float)static_cast<const T*>(a.residual)[m * a.ldr + n];
    static_cast<T*>(a.y)[m * a.ldy + n] = (T)z;
  }
}

}  // namespace qlin
}  // namespace bcjr
