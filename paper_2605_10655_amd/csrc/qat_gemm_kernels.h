// qat_gemm_kernels.h -- the matrix product of the quantised linear layer and
// its backward pass: C[i, j] = sum_k A[i, k] B[j, k] on the matrix
// instructions, with the epilogue bias, activation, residual and 8-bit
// checkpoint.
#pragma once
#include "qat_common.h"

namespace bcjr {
namespace qlin {

// How an operand is held in memory
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
  // k split over `splits` workgroups per tile: each writes its sums to
  // part [splits][I][J], and the epilogue is join_kernel's
  int splits;
  float* part;
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

// 16 bytes of zeros that loads past the end of k are pointed at
static __device__ __align__(64) const uint32_t kZeros[16] = {};

__device__ __forceinline__ void to_lds16(const void* g, void* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// ---------------------------------------------------------------- one operand's tile
// R rows x 128 bytes of k (kStep values), in units of 16 bytes ("chunks").
//   row, codes: place(r, c) = 8 r + (c ^ (r & 7)): a read takes one chunk of
//     each of 32 consecutive rows, and the exclusive or spreads those over
//     all banks.
//   col, 16 bits: [k][R], chunk c of k's row at c ^ swizzle(k): the transposed
//     read takes 64 bytes of each of 8 k, which then lie in different banks.
//   col, 32 bits: [k][R] as it is: a read takes 32 consecutive rows of one k.
template <class T, int MODE, int R, int THREADS>
struct Tile {
  static constexpr int E = kPer16<T>;
  static constexpr int kStep = 8 * E;                   // k of a tile
  static constexpr int kChunks = R * 8;                 // 16-byte chunks
  static constexpr int kPer = kChunks / THREADS;        // of them per thread
  static constexpr int kLine = MODE == kCol ? R / E : 8;  // chunks of an LDS line
  static constexpr int kCodeRuns = R * kStep / 16;      // 16-byte runs of codes
  static constexpr int kLoads = (kCodeRuns + THREADS - 1) / THREADS;
  using V = typename Vec<T>::type;

  static __device__ __forceinline__ int swizzle(int line) {
    if (MODE != kCol) return line & 7;
    if (sizeof(T) == 4) return 0;
    return R >= 128 ? (line & 3) << 2 : ((line >> 1) & 1) << 2;
  }
  static __device__ __forceinline__ int place(int line, int c) { return line * kLine + (c ^ swizzle(line)); }

  // Asynchronous copy of k0 .. k0 + kStep - 1 into LDS, straight from memory:
  // needs p and ld aligned to 16 bytes, K (row) or R (col) a whole number of
  // chunks, and a tile's span below 2 GiB.  A wave's 64 chunks go to 64
  // consecutive places, so each lane fetches the chunk that belongs at its
  // place: byte offsets from the tile's start, the same in every step.  Rows
  // past the end read the last one's (their sums are not stored), k past the
  // end zeros.
  struct Copy {
    uint32_t off[kPer];
    const char* base;
    int64_t step;
  };

  static __device__ __forceinline__ void start(Copy& s, const void* p, int64_t ld, int64_t rows, int64_t r0,
                                               int64_t k0, int tid) {
    const uint32_t ldb = (uint32_t)(ld * (int64_t)sizeof(T));
    const int last = (int)(rows - r0 < R ? rows - r0 : R);   // rows of this tile
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = i * THREADS + tid;
      const int line = at / kLine, c = (at % kLine) ^ swizzle(line);
      if (MODE == kRow)
        s.off[i] = (uint32_t)(line < last ? line : last - 1) * ldb + c * 16;
      else
        s.off[i] = (uint32_t)line * ldb + (c * E < last ? c * 16 : (last - E) * (int)sizeof(T));
    }
    const int64_t first = MODE == kRow ? r0 * ld + k0 : k0 * ld + r0;
    s.base = static_cast<const char*>(p) + first * (int64_t)sizeof(T);
    s.step = (MODE == kRow ? kStep : kStep * ld) * (int64_t)sizeof(T);
  }

  static __device__ __forceinline__ void copy(Copy& s, int64_t k_left, V* lds, int tid) {
    const int wave = tid >> 6;
    if (k_left >= kStep) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) to_lds16(s.base + s.off[i], lds + i * THREADS + wave * 64);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int at = i * THREADS + tid, line = at / kLine;
        const int k = MODE == kRow ? ((at % kLine) ^ swizzle(line)) * E : line;
        const char* src = s.base + s.off[i];
        if (k >= k_left) src = reinterpret_cast<const char*>(kZeros);
        to_lds16(src, lds + i * THREADS + wave * 64);
      }
    }
    s.base += s.step;
  }

  // The same through registers, for any alignment: whole chunks by one load
  // (which need not be aligned), those that cross an edge by value.
  struct Regs {
    V v[kPer];
    uint16_t s[kPer];
  };

  static __device__ __forceinline__ void fetch(const void* p, int64_t ld, const uint16_t* scales, int64_t rows,
                                               int64_t K, int64_t r0, int64_t k0, Regs& g, int tid) {
    if (MODE == kCodes) {
      // 16 codes a load; consecutive threads along a group's 32, then rows
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = i * THREADS + tid;
        if (kCodeRuns % THREADS && at >= kCodeRuns) break;
        const int64_t grp = k0 / kRows + at / (2 * R);
        int64_t r = r0 + (at >> 1) % R;
        r = r < rows ? r : rows - 1;
        const bool in = grp * kRows < K;
        const int64_t o = in ? grp * rows + r : 0;
        u32x4 q = *reinterpret_cast<const u32x4*>(static_cast<const int8_t*>(p) + o * kRows + (at & 1) * 16);
        if (!in) q = u32x4{0, 0, 0, 0};
        __builtin_memcpy(&g.v[i], &q, 16);
        g.s[i] = in ? scales[o] : (uint16_t)0;
      }
      return;
    }
    const T* t = static_cast<const T*>(p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = i * THREADS + tid;
      const int line = at / kLine, c = at % kLine;
      V v;
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = (T)0.f;
      const int64_t r = r0 + (MODE == kRow ? line : c * E), k = k0 + (MODE == kRow ? c * E : line);
      const T* src = t + (MODE == kRow ? r * ld + k : k * ld + r);
      // values of the chunk that exist
      const int64_t n = MODE == kRow ? (r < rows ? K - k : 0) : (k < K ? rows - r : 0);
      if (n >= E) {
        __builtin_memcpy(&v, src, 16);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e < n) v[e] = src[e];
      }
      g.v[i] = v;
    }
  }

  static __device__ __forceinline__ void put(const Regs& g, V* lds, int tid) {
    if (MODE == kCodes) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = i * THREADS + tid;
        if (kCodeRuns % THREADS && at >= kCodeRuns) break;
        const int r = (at >> 1) % R, c0 = (at / (2 * R)) * (kRows / E) + (at & 1) * (16 / E);
        // a group with a non-finite value counts as NaN whole: its column of
        // the gradient is not finite in either case
        const uint16_t s = g.s[i];
        const float f = (s & 0x8000u) ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)s << 16);
        uint32_t q[4];
        __builtin_memcpy(q, &g.v[i], 16);
#pragma unroll
        for (int u = 0; u < 16 / E; ++u) {
          V v;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int j = u * E + e;
            v[e] = (T)((float)((int)(q[j >> 2] << (24 - 8 * (j & 3))) >> 24) * f);
          }
          lds[place(r, c0 + u)] = v;
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = i * THREADS + tid;
      lds[place(at / kLine, at % kLine)] = g.v[i];
    }
  }

  // the operand of one matrix instruction: rows r0 .. r0 + 31, k of step kk
  static __device__ __forceinline__ V operand(const V* lds, int r0, int kk, int lane) {
    if (MODE != kCol) return lds[place(r0 + (lane & 31), 2 * kk + (lane >> 5))];
    V v;
    if constexpr (sizeof(T) == 4) {
      const float* f = reinterpret_cast<const float*>(lds);
#pragma unroll
      for (int s = 0; s < 4; ++s) v[s] = f[(8 * kk + 4 * (lane >> 5) + s) * R + r0 + (lane & 31)];
    } else {
      // 16 lanes read 4 k x 16 rows, a lane 8 bytes of one k, and receive
      // their row's four k
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      const int r = r0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      s16x4 h[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int k = 16 * kk + 8 * (lane >> 5) + 4 * t + ((lane & 15) >> 2);
        const char* at = reinterpret_cast<const char*>(lds) + place(k, r >> 3) * 16 + (r & 7) * 2;
        h[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(const_cast<char*>(at)));
      }
      __builtin_memcpy(&v, h, 16);
    }
    return v;
  }
};

// ---------------------------------------------------------------- epilogue
// LDS written by some lanes of a wave is read by others
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The 8-bit groups of 32 rows x WJ columns of C + bias in LDS: a lane (two,
// where WJ is 32) takes a column, so that no value crosses lanes and 32
// contiguous bytes are stored for each.
template <class T, int WJ>
__device__ __forceinline__ void checkpoint_strip(int8_t* codes, uint16_t* scales, const T* bias, const float* strip,
                                                 int lane, int64_t i0, int64_t j0, int64_t I, int64_t J) {
  constexpr int kN = kRows * WJ / 64;      // rows of a lane
  const int col = lane % WJ, r0 = lane / WJ * kN;
  const int64_t j = j0 + col;
  const int rows = I - i0 < kRows ? (int)(I - i0) : kRows;
  const float b = bias && j < J ? (float)bias[j] : 0.f;
  float z[kN], amax = 0.f;
  int bad = 0;
#pragma unroll
  for (int r = 0; r < kN; ++r) {
    z[r] = r0 + r < rows ? strip[(r0 + r) * (WJ + 4) + col] + b : 0.f;
    const bool fin = finite_bits(z[r]);
    amax = fmaxf(amax, fin ? fabsf(z[r]) : 0.f);
    bad |= !fin;
  }
  if (WJ == 32) {
    amax = fmaxf(amax, __shfl_xor(amax, 32));
    bad |= __shfl_xor(bad, 32);
  }
  if (j >= J) return;
  const Q8 q = q8_of(amax, kEmin<float>, kEmax<float>);
  const int64_t at = (i0 / kRows) * J + j;
#pragma unroll
  for (int o = 0; o < kN / 16; ++o) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < 16; ++r) w[r >> 2] |= (uint32_t)(q8_code(z[16 * o + r], q) & 255) << (8 * (r & 3));
    *reinterpret_cast<u32x4*>(codes + at * kRows + r0 + 16 * o) = u32x4{w[0], w[1], w[2], w[3]};
  }
  if (lane < WJ) scales[at] = q8_scale_bits(q, bad != 0);
}

// 32 rows x WJ columns of C from LDS: bias, activation, residual, out in runs
// of 16 bytes of a row (by one access each, which need not be aligned)
template <class T, int WJ>
__device__ __forceinline__ void put_strip(T* y, int64_t ldy, const T* bias, const T* res, int64_t ldr, int act,
                                          const float* strip, int lane, int64_t i0, int64_t j0, int64_t I, int64_t J) {
  constexpr int E = kPer16<T>, kRun = WJ / E;
  using V = typename Vec<T>::type;
#pragma unroll 2
  for (int u = lane; u < 32 * kRun; u += 64) {
    const int row = u / kRun, col = (u % kRun) * E;
    const int64_t i = i0 + row, j = j0 + col, n = J - j;
    if (i >= I || n <= 0) continue;
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = strip[row * (WJ + 4) + col + e];
    if (bias)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += e < n ? (float)bias[j + e] : 0.f;
    if (act != kActNone)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = act_value(v[e], act);
    T* out = y + i * ldy + j;
    const T* r = res ? res + i * ldr + j : nullptr;
    V o;
    if (n >= E) {
      if (r) {
        V rv;
        __builtin_memcpy(&rv, r, 16);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] += (float)rv[e];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = (T)v[e];
      __builtin_memcpy(out, &o, 16);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < n) out[e] = (T)(r ? v[e] + (float)r[e] : v[e]);
    }
  }
}

// ---------------------------------------------------------------- product
// BI x BJ of C per workgroup, WI x WJ of them per wave in 32 x 32 matrix
// instructions, 128 bytes of k a step, two LDS buffers: the next step's tiles
// travel while this one's are multiplied.  COPY: both operands straight into
// LDS (codes always through registers, where they become T).
template <class T, int AM, int BM, int BI, int BJ, int WI, int WJ, bool COPY>
__global__ __launch_bounds__((BI / WI) * (BJ / WJ) * 64) void gemm_kernel(GemmArgs g, int ti, int tj) {
  constexpr int kThreads = (BI / WI) * (BJ / WJ) * 64;
  constexpr int NI = WI / 32, NJ = WJ / 32;
  using TA = Tile<T, AM, BI, kThreads>;
  using TB = Tile<T, BM, BJ, kThreads>;
  using V = typename Vec<T>::type;
  constexpr bool kCopyA = COPY && AM != kCodes, kCopyB = COPY && BM != kCodes;
  // Two buffers of their own names: the compiler then knows that a copy into
  // one does not touch what is read from the other, and waits for neither.
  // The epilogue's strip of a wave is 32 rows x WJ sums in the first, rows
  // padded by 16 bytes.
  constexpr int kLine = WJ + 4, kStrip = 32 * kLine, kStrips = kThreads / 64 * kStrip / 4;
  constexpr int kBuf = TA::kChunks + TB::kChunks;
  __shared__ __align__(16) V lds0[kBuf > kStrips ? kBuf : kStrips];
  __shared__ __align__(16) V lds1[kBuf];

  // Consecutive workgroups go to the 8 dies in turn: give each die a
  // contiguous run of tiles, in bands of 8 tile rows, so that its L2 holds the
  // rows of A and B that its workgroups share.
  const int n = ti * tj * g.splits;
  int id = blockIdx.x;
  {
    const int per = n / 8, rest = n % 8, die = id % 8, in = id / 8;
    id = die * per + (die < rest ? die : rest) + in;
  }
  const int part = id / (ti * tj);
  id -= part * ti * tj;
  const int band = id / (8 * tj), rows_of = ti - band * 8 < 8 ? ti - band * 8 : 8, in = id - band * 8 * tj;
  const int64_t i0 = (int64_t)(band * 8 + in % rows_of) * BI, j0 = (int64_t)(in / rows_of) * BJ;

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wi = (wave / (BJ / WJ)) * WI, wj = (wave % (BJ / WJ)) * WJ;
  f32x16 acc[NI][NJ];
#pragma unroll
  for (int x = 0; x < NI; ++x)
#pragma unroll
    for (int y = 0; y < NJ; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;

  const int64_t steps = (g.K + TA::kStep - 1) / TA::kStep;
  const int64_t s0 = steps * part / g.splits, s1 = steps * (part + 1) / g.splits;
  typename TA::Regs ra;
  typename TB::Regs rb;
  typename TA::Copy ca;
  typename TB::Copy cb;
  if constexpr (kCopyA) TA::start(ca, g.a, g.lda, g.I, i0, s0 * TA::kStep, tid);
  if constexpr (kCopyB) TB::start(cb, g.b, g.ldb, g.J, j0, s0 * TA::kStep, tid);
  auto begin = [&](int64_t s, V* lds) __attribute__((always_inline)) {
    const int64_t k0 = s * TA::kStep;
    if constexpr (kCopyA)
      TA::copy(ca, g.K - k0, lds, tid);
    else
      TA::fetch(g.a, g.lda, nullptr, g.I, g.K, i0, k0, ra, tid);
    if constexpr (kCopyB)
      TB::copy(cb, g.K - k0, lds + TA::kChunks, tid);
    else
      TB::fetch(g.b, g.ldb, g.bscales, g.J, g.K, j0, k0, rb, tid);
  };
  auto end = [&](V* lds) __attribute__((always_inline)) {
    if constexpr (!kCopyA) TA::put(ra, lds, tid);
    if constexpr (!kCopyB) TB::put(rb, lds + TA::kChunks, tid);
  };
  auto step = [&](int64_t s, const V* now, V* next) __attribute__((always_inline)) {
    // this step's tiles have landed (every wave waits for its own part), and
    // no wave still reads the other buffer
    __syncthreads();
    if (s + 1 < s1) begin(s + 1, next);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      V fa[NI], fb[NJ];
#pragma unroll
      for (int x = 0; x < NI; ++x) fa[x] = TA::operand(now, wi + 32 * x, kk, lane);
#pragma unroll
      for (int y = 0; y < NJ; ++y) fb[y] = TB::operand(now + TA::kChunks, wj + 32 * y, kk, lane);
#pragma unroll
      for (int x = 0; x < NI; ++x)
#pragma unroll
        for (int y = 0; y < NJ; ++y) mma<T>(fa[x], fb[y], acc[x][y]);
    }
    if (s + 1 < s1) end(next);
  };

  if (s0 < s1) {
    begin(s0, lds0);
    end(lds0);
  }
  for (int64_t s = s0; s < s1; s += 2) {
    step(s, lds0, lds1);
    if (s + 1 < s1) step(s + 1, lds1, lds0);
  }

  // lane: column lane & 31 of a 32 x 32 tile, rows 8 (r / 4) + 4 (lane / 32) +
  // r % 4 for r = 0..15.  The sums go through the wave's own strip of LDS, so
  // that a lane stores 16 bytes of one row.
  __syncthreads();
  float* strip = reinterpret_cast<float*>(lds0) + wave * kStrip;
  const T* bias = static_cast<const T*>(g.bias);
#pragma unroll
  for (int x = 0; x < NI; ++x) {
    const int64_t ib = i0 + wi + 32 * x;
#pragma unroll
    for (int y = 0; y < NJ; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        strip[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * kLine + 32 * y + (lane & 31)] = acc[x][y][r];
    wave_sync();
    if (g.splits > 1) {
      put_strip<float, WJ>(g.part + (int64_t)part * g.I * g.J, g.J, nullptr, nullptr, 0, kActNone, strip, lane, ib,
                           j0 + wj, g.I, g.J);
    } else {
      if (g.zcodes && ib < g.I)
        checkpoint_strip<T, WJ>(g.zcodes, g.zscales, bias, strip, lane, ib, j0 + wj, g.I, g.J);
      put_strip<T, WJ>(static_cast<T*>(g.y), g.ldy, bias, static_cast<const T*>(g.residual), g.ldr, g.act, strip, lane,
                       ib, j0 + wj, g.I, g.J);
    }
    wave_sync();
  }
}

// The epilogue of a product whose k was split: the parts' sum (always in the
// same order), bias, activation, residual.  A thread per value, or with a
// checkpoint per group of 32 rows of one column.
template <class T, bool CODES>
__global__ void join_kernel(GemmArgs g) {
  const T* bias = static_cast<const T*>(g.bias);
  const T* res = static_cast<const T*>(g.residual);
  const int64_t j = (int64_t)blockIdx.y * blockDim.x + threadIdx.x, size = g.I * g.J;
  if (j >= g.J) return;
  const float b = bias ? (float)bias[j] : 0.f;
  constexpr int kN = CODES ? kRows : 1;
  const int64_t i0 = (int64_t)blockIdx.x * kN;
  float z[kN];
#pragma unroll
  for (int r = 0; r < kN; ++r) {
    z[r] = 0.f;
    if (i0 + r < g.I) {
      const float* p = g.part + (i0 + r) * g.J + j;
      float s = 0.f;
      for (int q = 0; q < g.splits; ++q) s += p[q * size];
      z[r] = s + b;
    }
  }
  if (CODES) {
    float amax = 0.f;
    bool bad = false;
#pragma unroll
    for (int r = 0; r < kN; ++r) {
      if (finite_bits(z[r]))
        amax = fmaxf(amax, fabsf(z[r]));
      else
        bad = true;
    }
    const Q8 q = q8_of(amax, kEmin<float>, kEmax<float>);
    const int64_t at = blockIdx.x * g.J + j;
#pragma unroll
    for (int r = 0; r < kN; r += 4) {
      uint32_t w = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) w |= (uint32_t)(q8_code(z[(r + u) % kN], q) & 255) << (8 * u);
      *reinterpret_cast<uint32_t*>(g.zcodes + at * kRows + r) = w;
    }
    g.zscales[at] = q8_scale_bits(q, bad);
  }
#pragma unroll
  for (int r = 0; r < kN; ++r) {
    const int64_t i = i0 + r;
    if (i >= g.I) break;
    float v = act_value(z[r], g.act);
    if (res) v += (float)res[i * g.ldr + j];
    static_cast<T*>(g.y)[i * g.ldy + j] = (T)v;
  }
}

}  // namespace qlin
}  // namespace bcjr
