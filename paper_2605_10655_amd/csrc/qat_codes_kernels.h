// qat_codes_kernels.h -- a few tokens through trellis-coded weights: the bit
// strings are turned into operands of the matrix instructions as they are read.
#pragma once
#include "qat_few_kernels.h"

namespace bcjr {
namespace qlin {

struct CodesArgs : FewArgs {
  const uint32_t* packed;
  const float* codebook;
  const float* scales;       // [N, K / block] or null
  int n, block, words;
};

// y = act(x W^T + bias) + residual for up to 16 MT tokens.
//
// The codebook lies in LDS as T, V values a state, so that a step costs a
// funnel shift, a shift, an address and one LDS read.  Those reads meet random
// banks (64 lanes take 8.4 cycles) and are what bounds the kernel, not memory
// (2 bits a weight) nor the matrix instructions; a lane's weights are therefore
// decoded once and multiplied with all tokens.  A codebook of more than 128 KB
// (V = 2 or fp32 at 16 state bits) is taken in parts of that size: in each, the
// states of the others read a zero, all the same one, which costs no bank.
//
// A wave takes 16 / Q rows and 256 Q weights of each.  Lane l of a matrix
// instruction holds row l % 16 and eight k; which k is free, so lane group l /
// 16 takes 64 weights in a row, whose windows start at a word of the string.
// With Q = 2 (at most 8 tokens) rows 8..15 are the same rows at the next 256
// weights, tokens 8..15 the same tokens there: the products of unlike halves
// are not used, and half the rows a tile fill twice the CUs.
//
// Waves of a workgroup split K; their sums meet in LDS in a fixed order.
//
// bf16, 16 state bits: one token, 2048 -> 8192, 2 bits a weight 11.5 us (table
// reads 3.6, filling the tables and the launch most of the rest); 16 tokens,
// 2048 x 2048, two weights a step 14.5.
constexpr int kChunk = 256;       // weights of a row that a wave takes at once


// State bits of a part of the codebook: 128 KB
template <class T, int V>
constexpr int kTableBits = sizeof(T) * V == 2 ? 16 : sizeof(T) * V == 4 ? 15 : 14;

// LDS bytes: the codebook's part and a zero entry (16 bytes), then 16 x 16 sums
// a wave
template <class T, int V>
constexpr size_t codes_table(int n) {
  return (((size_t)sizeof(T) * V) << (n < kTableBits<T, V> ? n : kTableBits<T, V>)) / 16 * 16 + 32;
}

// Part h of the codebook as T, four values at a time.  The weights are the
// matrix instructions' operands, so they are rounded to T here, half a step
// each (their scale is applied to the fp32 sums): unrounded ones would take twice
// the table and so twice the passes over the bit strings.  An output's error
// against 64 bits is that of torch's product with weights in T, or less: bf16,
// one token 2048 -> 8192, 2.4e-3 of the outputs' norm (torch 3.2e-3; of an output
// rounded once 1.7e-3), 16 tokens 2048 -> 2048 2.4e-3 (2.4e-3).
template <class T, int V>
__device__ __forceinline__ void fill_table(T* table, const float* codebook, int n, int h, int tid, int threads) {
  const int count = V << (n < kTableBits<T, V> ? n : kTableBits<T, V>);
  codebook += (int64_t)h * count;
  if (tid < V) table[count + tid] = (T)0.f;   // what states of other parts read
  if (count < 4) {
    if (tid < count) table[tid] = (T)codebook[tid];
    return;
  }
  typedef T T4 __attribute__((ext_vector_type(4)));
  const f32x4* src = reinterpret_cast<const f32x4*>(codebook);
  T4* dst = reinterpret_cast<T4*>(table);
#pragma unroll 8
  for (int s = tid; s < count / 4; s += threads) {
    const f32x4 c = src[s];
    T4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (T)c[i];
    dst[s] = v;
  }
}

// (One workgroup fills a CU's LDS: four waves a SIMD and their 128 registers,
// which the compiler would otherwise not all use to keep loads under way: 16.2
// us against 14.5 for the second of the two above.  For 17 to 64 tokens that is
// too few: of the forms with 1 to 4 bits a step the fp32 ones keep up to 21
// registers in scratch, the 16-bit ones 2 and 16 at 3 and 4.)
template <class T, int KB, int V, int MT, int Q>
__global__ __launch_bounds__(64 * kFewWaves) __attribute__((amdgpu_waves_per_eu(4, 4))) void codes_kernel(
    CodesArgs a) {
  using F = typename Frag<T>::type;
  struct Entry {
    T v[V];
  };
  constexpr int kRowsOf = 16 / Q;
  constexpr int kSteps = 64 / V;                              // steps of a lane's 64 weights
  constexpr int kWords = ((kSteps - 1) * KB + 16 + 31) / 32;  // words that they span (16 state bits)
  extern __shared__ __align__(16) char lds[];
  Entry* table = reinterpret_cast<Entry*>(lds);
  float* sums = reinterpret_cast<float*>(lds + codes_table<T, V>(a.n));
  const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 63, wave = tid >> 6;
  const int part = wave % a.parts, of = wave / a.parts;
  const int row = lane & 15, g = lane >> 4;
  const int units = (a.K / kChunk + Q - 1) / Q;               // along K
  const int pieces = a.n > kTableBits<T, V> ? 1 << (a.n - kTableBits<T, V>) : 1;
  const int right = 32 - a.n;
  const T* x = static_cast<const T*>(a.x);

  // the words of this lane's 64 weights of its row in unit u
  auto words = [&](int tile, int u, uint32_t* w) __attribute__((always_inline)) {
    int r = tile * kRowsOf + row % kRowsOf;
    r = r < a.N ? r : a.N - 1;
    int at = (u * Q + row / kRowsOf) * kChunk;                // first weight of the chunk
    at = at < a.K ? at : 0;
    const int64_t path = (int64_t)r * (a.K / a.block) + at / a.block;
    const int word = (at % a.block + 64 * g) / V * KB / 32;
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = a.packed[path * a.words + (word + i < a.words ? word + i : a.words - 1)];
  };

  // a token's activations at eight of this lane's weights in unit u
  auto tokens = [&](int u, int m, int f) __attribute__((always_inline)) {
    int tok = Q == 2 ? lane & 7 : 16 * m + row;
    tok = tok < a.M ? tok : a.M - 1;
    const int from = (u * Q + (Q == 2 ? row >> 3 : 0)) * kChunk;   // of the token's half
    F xf;
#pragma unroll
    for (int e = 0; e < 8; ++e) xf[e] = (T)0.f;                    // none past the end of K
    if (Q == 1 || from < a.K) __builtin_memcpy(&xf, x + tok * a.ldx + from + 64 * g + 8 * f, sizeof(xf));
    return xf;
  };
  // the scales of the sums' rows 4 g + i (and of the half that those belong to)
  auto scales = [&](int tile, int u) __attribute__((always_inline)) {
    f32x4 sc = {1.f, 1.f, 1.f, 1.f};
    if (a.scales) {
      int ch = u * Q + 4 * g / kRowsOf;
      ch = ch * kChunk < a.K ? ch : 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int r = tile * kRowsOf + (4 * g + i) % kRowsOf;
        r = r < a.N ? r : a.N - 1;
        sc[i] = a.scales[(int64_t)r * (a.K / a.block) + ch * kChunk / a.block];
      }
    }
    return sc;
  };

  bool filled = false;
  for (int t0 = blockIdx.x * a.at_once; t0 < a.tiles; t0 += gridDim.x * a.at_once) {
    const int tile = t0 + of;
    const bool live = of < a.at_once && tile < a.tiles;
    f32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int h = 0; h < pieces; ++h) {
      // the first unit's words travel while the table is filled (its scales and
      // tokens too would leave the wave too few registers: 13.9 against 11.5 us)
      uint32_t w[kWords];
      if (live && part < units) words(tile, part, w);
      if (!filled || pieces > 1) {   // (a single piece stays)
        __syncthreads();
        fill_table<T, V>(reinterpret_cast<T*>(table), a.codebook, a.n, h, tid, threads);
        __syncthreads();
        filled = true;
      }
      const uint32_t before = (uint32_t)h << kTableBits<T, V>, none = 1u << kTableBits<T, V>;
      if (live)
#pragma unroll 1
        for (int u = part; u < units; u += a.parts) {
          const f32x4 sc = scales(tile, u);
          f32x4 now[MT];
#pragma unroll
          for (int m = 0; m < MT; ++m) now[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int f = 0; f < 8; ++f) {
            F wf;
#pragma unroll
            for (int e = 0; e < 8 / V; ++e) {
              // the n bits at bit KB * step of the string
              const int off = KB * (8 / V * f + e), j = off >> 5, o = off & 31;
              const uint32_t top = o == 0 ? w[j] : __builtin_amdgcn_alignbit(w[j], w[j + 1 < kWords ? j + 1 : j], 32 - o);
              uint32_t s = top >> right;
              if (kTableBits<T, V> < 16) {
                s -= before;
                s = s < none ? s : none;
              }
              const Entry c = table[s];
#pragma unroll
              for (int v = 0; v < V; ++v) wf[V * e + v] = c.v[v];
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) mma16(wf, tokens(u, m, f), now[m]);
          }
          if (u + a.parts < units) words(tile, u + a.parts, w);
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][i] = __builtin_fmaf(sc[i], now[m][i], acc[m][i]);
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) finish_few<T, Q>(a, sums, acc[m], t0, m, tid, threads);
  }
}

// W = scale * codebook[state] of many weights, the product in fp32, rounded to
// T once, as the next product's operand (the error of the whole is 2.1e-3 of the
// outputs' norm in bf16, 2048 tokens 8192 -> 2048; torch's product of weights
// in bf16 2.6e-3, of an output rounded once 1.7e-3).  A thread takes eight weights (16 bytes of a 16-bit type) in each of eight
// rows of 8192, kept in registers while the fp32 codebook passes through LDS in
// pieces of 128 KB; of each, states of the others read a zero.  (Read from L2
// a weight costs 1.1 cycles a CU and requests 64 bytes for 4: 16.8 million
// weights took 74 us; this takes 21, 7 of them reads of the tables.)
constexpr int kDenseThreads = 1024, kDenseGroups = 8;

template <class T, int KB, int V>
__global__ __launch_bounds__(kDenseThreads) void dense_large_kernel(const uint32_t* __restrict__ packed,
                                                                    const float* __restrict__ codebook,
                                                                    const float* __restrict__ scales, int64_t groups,
                                                                    int n, int per, int words, T* __restrict__ W) {
  struct Entry {
    float v[V];
  };
  typedef T T8 __attribute__((ext_vector_type(8)));
  extern __shared__ __align__(16) char lds[];
  const Entry* table = reinterpret_cast<const Entry*>(lds);
  const int tid = threadIdx.x;
  const int pieces = n > kTableBits<float, V> ? 1 << (n - kTableBits<float, V>) : 1;
  const int right = 32 - n;
  const uint32_t none = 1u << kTableBits<float, V>;
  constexpr int kSteps = 8 / V;
  bool filled = false;
  for (int64_t g0 = (int64_t)blockIdx.x * kDenseThreads * kDenseGroups; g0 < groups;
       g0 += (int64_t)gridDim.x * kDenseThreads * kDenseGroups) {
    // a group's window begins at a multiple of 8 bits and spans at most 44
    uint32_t hi[kDenseGroups], lo[kDenseGroups];
    float v[kDenseGroups][8];
#pragma unroll
    for (int i = 0; i < kDenseGroups; ++i) {
      int64_t g = g0 + i * kDenseThreads + tid;
      g = g < groups ? g : groups - 1;
      const uint32_t path = (uint32_t)g / (uint32_t)per;
      const int at = (int)((uint32_t)g - path * per) * kSteps * KB, j = at >> 5, o = at & 31;
      const uint32_t* p = packed + (int64_t)path * words;
      const uint64_t w = (((uint64_t)p[j] << 32) | p[j + 1 < words ? j + 1 : j]) << o;
      hi[i] = (uint32_t)(w >> 32);
      lo[i] = (uint32_t)w;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    }
#pragma unroll 1
    for (int h = 0; h < pieces; ++h) {
      if (!filled || pieces > 1) {
        __syncthreads();
        fill_table<float, V>(reinterpret_cast<float*>(lds), codebook, n, h, tid, kDenseThreads);
        __syncthreads();
        filled = true;
      }
      const uint32_t before = (uint32_t)h << kTableBits<float, V>;
#pragma unroll
      for (int i = 0; i < kDenseGroups; ++i) {
        // the states are worked out anew for each piece, not kept for all
        asm volatile("" : "+v"(hi[i]), "+v"(lo[i]));
#pragma unroll
        for (int e = 0; e < kSteps; ++e) {
          const uint32_t top = e == 0 ? hi[i] : __builtin_amdgcn_alignbit(hi[i], lo[i], 32 - KB * e);
          uint32_t s = (top >> right) - before;
          s = s < none ? s : none;
          const Entry c = table[s];
          // one piece adds the codeword, the others 0
#pragma unroll
          for (int u = 0; u < V; ++u) v[i][V * e + u] += c.v[u];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kDenseGroups; ++i) {
      const int64_t g = g0 + i * kDenseThreads + tid;
      if (g >= groups) continue;
      const float f = scales ? scales[(uint32_t)g / (uint32_t)per] : 1.f;
      T8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = (T)scaled(f, v[i][e]);
      __builtin_memcpy(W + g * 8, &o, sizeof(o));
    }
  }
}

}  // namespace qlin
}  // namespace bcjr
