// qat_linear_kernels.h -- kernels around the product of the quantised linear
// layer: the 8-bit checkpoints of activations, the gradient of its
// pre-activation, and trellis-coded weights.
#pragma once
#include "qat_common.h"

namespace bcjr {
namespace qlin {

// ---------------------------------------------------------------- 8-bit checkpoints
// Rows of two neighbouring 16-bit columns (one of 32 bits) per thread: a wave
// then moves 256 contiguous bytes of each row, and both columns' codes are 64
// contiguous bytes.  Workgroups of one band of 32 rows are neighbours, so that
// whole rows of memory are open at a time.  Bound by the bytes: 8192 x 8192 in
// bf16 is stored in 48.5 us (4.2 TB/s; a large copy moves 5.1) and loaded in
// 34.4 (6.0, its codes partly from the last-level cache).
template <class T>
constexpr int kCols = 4 / (int)sizeof(T);
constexpr int kGroupThreads = 64;

struct Band {
  int64_t g, c;
  int n;            // columns of this thread: none past the edge
};

template <int C>
__device__ __forceinline__ Band band_of(int64_t cols, uint32_t id = blockIdx.x) {
  const uint32_t per = (uint32_t)((cols + kGroupThreads * C - 1) / (kGroupThreads * C));
  Band b;
  b.g = id / per;
  b.c = ((int64_t)(id % per) * kGroupThreads + threadIdx.x) * C;
  b.n = b.c >= cols ? 0 : (cols - b.c < C ? (int)(cols - b.c) : C);
  return b;
}

// n <= C values at p, which need not be aligned
template <class T, int C>
__device__ __forceinline__ void get(const T* p, int n, float* v) {
  T t[C] = {};
  if (n == C)
    __builtin_memcpy(t, p, sizeof(t));
  else
    t[0] = p[0];
#pragma unroll
  for (int c = 0; c < C; ++c) v[c] = (float)t[c];
}

template <class T, int C>
__device__ __forceinline__ void set(T* p, int n, const float* v) {
  T t[C];
#pragma unroll
  for (int c = 0; c < C; ++c) t[c] = (T)v[c];
  if (n == C)
    __builtin_memcpy(p, t, sizeof(t));
  else
    p[0] = t[0];
}

// N rows of a band, zeros past the last: all loads under way at once
template <class T, int C, int N>
__device__ __forceinline__ void get_rows(const T* p, int64_t ld, int left, int n, float (*v)[C]) {
  if (left >= N && n == C) {
    T t[N][C];
#pragma unroll
    for (int i = 0; i < N; ++i) __builtin_memcpy(t[i], p + i * ld, sizeof(t[i]));
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int c = 0; c < C; ++c) v[i][c] = (float)t[i][c];
  } else {
    // rows past the last read the last one (left - 1 from p, below 0 for the
    // second half of a band that ends in the first)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = i < left ? i : left - 1;
      float t[C];
      get<T, C>(p + (int64_t)r * ld, n, t);
#pragma unroll
      for (int c = 0; c < C; ++c) v[i][c] = i < left ? t[c] : 0.f;
    }
  }
}

__device__ __forceinline__ int code_at(const u32x4* w, int i) {
  return (int)(w[i >> 4][(i >> 2) & 3] << (24 - 8 * (i & 3))) >> 24;
}

template <class T>
__global__ __launch_bounds__(kGroupThreads) void act8_store_kernel(const T* __restrict__ x, int64_t rows,
                                                                   int64_t cols, int64_t ldx,
                                                                   int8_t* __restrict__ codes,
                                                                   uint16_t* __restrict__ scales) {
  constexpr int C = kCols<T>;
  const Band b = band_of<C>(cols);
  if (b.n == 0) return;
  float v[kRows][C];
  const T* src = x + b.g * kRows * ldx + b.c;
  const int left = rows - b.g * kRows < kRows ? (int)(rows - b.g * kRows) : kRows;
  get_rows<T, C, kRows>(src, ldx, left, b.n, v);
  const int64_t at = b.g * cols + b.c;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (c < b.n) {
      u32x4* o = reinterpret_cast<u32x4*>(codes + (at + c) * kRows);
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const uint32_t m = __float_as_uint(v[i][c]) & 0x7fffffffu;
        top = m > top ? m : top;
      }
      uint32_t w[8];
      if (q8_plain(top, kEmax<T>)) {
        const Q8 q = q8_of(__uint_as_float(top), kEmin<T>, kEmax<T>);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          w[i] = q8_codes4(v[4 * i][c], v[4 * i + 1][c], v[4 * i + 2][c], v[4 * i + 3][c], q.inv);
        scales[at + c] = q8_scale_bits(q, false);
      } else {
        // rare: the values are read again, so that this costs no registers
        float amax = 0.f;
        bool bad = false;
#pragma unroll 1
        for (int i = 0; i < left; ++i) {
          const float f = (float)src[i * ldx + c];
          if (finite_bits(f))
            amax = fmaxf(amax, fabsf(f));
          else
            bad = true;
        }
        const Q8 q = q8_of(amax, kEmin<T>, kEmax<T>);
#pragma unroll 1
        for (int i = 0; i < kRows; ++i)
          codes[(at + c) * kRows + i] = (int8_t)(i < left ? q8_code((float)src[i * ldx + c], q) : 0);
        scales[at + c] = q8_scale_bits(q, bad);
        continue;
      }
      o[0] = u32x4{w[0], w[1], w[2], w[3]};
      o[1] = u32x4{w[4], w[5], w[6], w[7]};
    }
  }
}

template <class T>
__global__ __launch_bounds__(kGroupThreads) void act8_load_kernel(const int8_t* __restrict__ codes,
                                                                  const uint16_t* __restrict__ scales, int64_t rows,
                                                                  int64_t cols, T* __restrict__ out, int64_t ldo) {
  constexpr int C = kCols<T>;
  const Band b = band_of<C>(cols);
  if (b.n == 0) return;
  const int64_t at = b.g * cols + b.c;
  u32x4 w[C][2];
  uint16_t s[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int64_t o = at + (c < b.n ? c : 0);
    s[c] = scales[o];
#pragma unroll
    for (int h = 0; h < 2; ++h) w[c][h] = reinterpret_cast<const u32x4*>(codes + o * kRows)[h];
  }
  T* dst = out + b.g * kRows * ldo + b.c;
  const int left = rows - b.g * kRows < kRows ? (int)(rows - b.g * kRows) : kRows;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (i < left) {
      float v[C];
#pragma unroll
      for (int c = 0; c < C; ++c) v[c] = q8_value(code_at(w[c], i), s[c]);
      set<T, C>(dst + i * ldo, b.n, v);
    }
  }
}

// ---------------------------------------------------------------- backward
// dz = dy * act'(z8), rounded to T for the matrix instructions (half a step of
// the type each, as dy itself; unrounded it would take two products in place of
// each.  bf16, 4096 tokens, 8192 -> 2048, SiLU: dx and dW are 2.33e-3 of their
// norm off, as torch's backward pass in bf16 is; rounded once they would be
// 1.66e-3), and the sums of the unrounded dz over 16 rows,
// half a group each.  A workgroup takes the half: with whole groups 4096 x 2048
// had eight waves a CU (bf16 17.5 us against 16.6; the derivative's 40
// instructions a value take 9, the bytes 8.5).  Small layers have dz and these
// sums by themselves, by the same operations in the same order: dbias does not
// depend on what else is wanted.
template <class T, int ACT>
__global__ __launch_bounds__(kGroupThreads) void dz_kernel(const T* __restrict__ dy, int64_t ldd,
                                                           const int8_t* __restrict__ zcodes,
                                                           const uint16_t* __restrict__ zscales, int64_t rows,
                                                           int64_t cols, T* __restrict__ dz, int64_t ldz,
                                                           float* __restrict__ part) {
  constexpr int C = kCols<T>, kHalf = kRows / 2;
  const int h = blockIdx.x & 1;
  const Band b = band_of<C>(cols, blockIdx.x >> 1);
  const int64_t at = b.g * cols + b.c, r0 = b.g * kRows + kHalf * h;
  const int left = (int)(rows - r0 < kHalf ? rows - r0 : kHalf);   // 0 or less: none
  if (b.n == 0) {
    // zeros to the end of dz's rows (ldz is a multiple of C)
    const float zeros[C] = {};
    if (ACT != kActNone && b.c < ldz)
      for (int i = 0; i < left; ++i) set<T, C>(dz + (r0 + i) * ldz + b.c, C, zeros);
    return;
  }
  float eights[2][C] = {};   // sums of eight rows
  if (left > 0) {
    u32x4 w[C];
    uint16_t s[C];
    if (ACT != kActNone)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int64_t o = at + (c < b.n ? c : 0);
        s[c] = zscales[o];
        w[c] = reinterpret_cast<const u32x4*>(zcodes + o * kRows)[h];
      }
    float v[kHalf][C];
    get_rows<T, C, kHalf>(dy + r0 * ldd + b.c, ldd, left, b.n, v);
    T* dst = dz + r0 * ldz + b.c;
#pragma unroll
    for (int i = 0; i < kHalf; ++i) {
      if (ACT != kActNone) {
#pragma unroll
        for (int c = 0; c < C; ++c) v[i][c] = scaled(act_slope(q8_value(code_at(&w[c], i), s[c]), ACT), v[i][c]);
      }
      if (i < left) {
        if (ACT != kActNone) {
#pragma unroll
          for (int c = 0; c < C; ++c) v[i][c] = c < b.n ? v[i][c] : 0.f;
          set<T, C>(dst + i * ldz, C, v[i]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) eights[i / 8][c] += v[i][c];
      }
    }
  }
  if (part)
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (c < b.n) part[(2 * b.g + h) * cols + b.c + c] = eights[0][c] + eights[1][c];
}

// Up to two matrices into rows of whole 16 bytes, zeros behind their columns: a
// thread per 16 bytes written.  Bound by its bytes; the rule for it stands with
// its call.
struct Pad {
  const void* src;
  int64_t ld;
  void* dst;
  int64_t rows, cols, chunks;   // chunks: of a row written
};

template <class T>
__global__ __launch_bounds__(256) void pad_kernel(Pad a, Pad b, unsigned first) {
  using V = typename Vec<T>::type;
  constexpr int E = kPer16<T>;
  const Pad p = blockIdx.x < first ? a : b;
  const int64_t id = (int64_t)(blockIdx.x - (blockIdx.x < first ? 0 : first)) * 256 + threadIdx.x;
  if (id >= p.rows * p.chunks) return;
  const int64_t row = id / p.chunks, c = (id - row * p.chunks) * E, n = p.cols - c;
  const T* src = static_cast<const T*>(p.src) + row * p.ld + c;
  V v;
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = (T)0.f;
  if (n >= E) {
    __builtin_memcpy(&v, src, 16);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < n) v[e] = src[e];
  }
  static_cast<V*>(p.dst)[id] = v;
}

// The groups' sums of a column, in 64 bits and a fixed order: 16 threads take
// every 16th group each, one adds them (4096 x 2048: 5.3 us, mostly latency).
template <class T>
__global__ __launch_bounds__(1024) void dbias_kernel(const float* __restrict__ part, int64_t groups, int64_t cols,
                                                     T* __restrict__ out) {
  __shared__ double sums[16][64];
  const int lane = threadIdx.x & 63, row = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  double s = 0.;
  if (c < cols)
    for (int64_t g = row; g < groups; g += 16)
      s += (double)(part[2 * g * cols + c] + part[(2 * g + 1) * cols + c]);
  sums[row][lane] = s;
  __syncthreads();
  if (row == 0 && c < cols) {
    for (int r = 1; r < 16; ++r) s += sums[r][lane];
    out[c] = (T)(float)s;
  }
}

// ---------------------------------------------------------------- trellis codes
// A path s_0 .. s_{steps-1} as a bit string, most significant bit first in
// 32-bit words: the n bits of s_0, then k bits a step.  The state after step t
// is the n-bit window at bit t k.  Packing and unpacking are done once a matrix
// and are bound by the states' four bytes each.
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

// W = scale * codebook[state] in fp32, rounded to T.  One thread per step, for
// the trellises and sizes that dense_large_kernel does not take.
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
