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
// R rows x 128 bytes of k (kStep values; whole cache lines: with 64 bytes the
// copies alone took 1.4 times as long), in units of 16 bytes ("chunks").
//   row, codes: place(r, c) = 8 r + (c ^ (r / 2 & 7)): a read takes one chunk
//     of each of 32 consecutive rows; with the exclusive or any 16 of them that
//     are served together lie in the 256 bytes of all banks (with r & 7 in its
//     place they met in half of them: 0.46 of the LDS cycles were conflicts).
//   col, 16 bits: [k][R], chunk c of k's row at c ^ swizzle(k): the transposed
//     read takes 64 bytes of each of 8 k, which then lie in different banks.
//   col, 32 bits: [k][R] as it is: a read takes 32 consecutive rows of one k.
//
// The tile's row l is the operand's row r0 + (l / RUN) * STRIDE + l % RUN.
template <class T, int MODE, int R, int THREADS, int RUN = R, int STRIDE = R>
struct Tile {
  static constexpr int E = kPer16<T>;
  static constexpr int kRowChunks = 8;
  static constexpr int kStep = kRowChunks * E;          // k of a tile
  static constexpr int kChunks = R * kRowChunks;        // 16-byte chunks
  static constexpr int kPer = kChunks / THREADS;        // of them per thread
  static constexpr int kLine = MODE == kCol ? R / E : kRowChunks;  // chunks of an LDS line
  static constexpr int kRuns = kStep / 16;              // 16-byte runs of codes in a row
  static constexpr int kLoads = (R * kRuns + THREADS - 1) / THREADS;
  using V = typename Vec<T>::type;

  static __device__ __forceinline__ int swizzle(int line) {
    if (MODE != kCol) return (line >> 1) & 7;
    if (sizeof(T) == 4) return 0;
    return R >= 128 ? (line & 3) << 2 : ((line >> 1) & 1) << 2;
  }
  static __device__ __forceinline__ int row_of(int l) { return l / RUN * STRIDE + l % RUN; }
  static __device__ __forceinline__ int place(int line, int c) { return line * kLine + (c ^ swizzle(line)); }

  // Asynchronous copy of k0 .. k0 + kStep - 1 into LDS, straight from memory:
  // needs p and ld aligned to 16 bytes, K (row) or R (col) a whole number of
  // chunks (or rows that go on to one, by rows with zeros), and a tile's span
  // below 2 GiB.  A wave's 64 chunks go to 64
  // consecutive places, so each lane fetches the chunk that belongs at its
  // place: byte offsets from the tile's start, the same in every step.  Rows
  // past the end read the last one's (their sums are not stored), k past the
  // end zeros.
  struct Copy {
    uint32_t off[kPer];
    const char* base;
    int64_t step;
  };

  template <bool TO_LDS = true>
  static __device__ __forceinline__ void start(Copy& s, const void* p, int64_t ld, int64_t rows, int64_t r0,
                                               int64_t k0, int tid) {
    const uint32_t ldb = (uint32_t)(ld * (int64_t)sizeof(T));
    const int span = R / RUN * STRIDE;
    const int last = (int)(rows - r0 < span ? rows - r0 : span);   // rows from r0 on
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = i * THREADS + tid;
      // (through registers the places are swizzled on the way to LDS)
      const int line = at / kLine, c = TO_LDS ? (at % kLine) ^ swizzle(line) : at % kLine;
      if (MODE == kRow) {
        const int r = row_of(line);
        s.off[i] = (uint32_t)(r < last ? r : last - 1) * ldb + c * 16;
      } else {
        const int r = row_of(c * E);
        s.off[i] = (uint32_t)line * ldb + (r < last ? r : (TO_LDS ? (last - 1) / E * E : 0)) * (int)sizeof(T);
      }
    }
    const int64_t first = MODE == kRow ? r0 * ld + k0 : k0 * ld + r0;
    s.base = static_cast<const char*>(p) + first * (int64_t)sizeof(T);
    s.step = (MODE == kRow ? kStep : kStep * ld) * (int64_t)sizeof(T);
  }

  // A whole step.  The tile's start (a buffer resource) and the LDS places are
  // uniform: a load costs no vector instruction.  The caller moves base on.
  static __device__ __forceinline__ void copy(const Copy& s, V* lds, int tid) {
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(s.base), 0, 0x7fffffff, 0x00020000);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          r, (__attribute__((address_space(3))) void*)(lds + i * THREADS + wave * 64), 16, (int)s.off[i], 0, 0, 0);
  }

  // The ragged end of k from k0 on.
  static __device__ __forceinline__ void copy_rest(const void* p, int64_t ld, int64_t rows, int64_t K, int64_t r0,
                                                   int64_t k0, V* lds, int tid) {
    Copy s;
    start(s, p, ld, rows, r0, k0, tid);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = i * THREADS + tid, line = at / kLine;
      const int k = MODE == kRow ? ((at % kLine) ^ swizzle(line)) * E : line;
      const char* src = k0 + k < K ? s.base + s.off[i] : reinterpret_cast<const char*>(kZeros);
      to_lds16(src, lds + i * THREADS + wave * 64);
    }
  }

  // The same through registers, for any alignment: whole chunks by one load
  // (which need not be aligned), those that cross an edge by value.
  struct Regs {
    V v[MODE == kCodes ? kLoads : kPer];
    uint16_t s[MODE == kCodes ? kLoads : 1];
  };

  static __device__ __forceinline__ void fetch(const void* p, int64_t ld, const uint16_t* scales, int64_t rows,
                                               int64_t K, int64_t r0, int64_t k0, Regs& g, int tid) {
    if (MODE == kCodes) {
      // 16 codes a load, a row's runs by neighbouring threads.  Every thread
      // loads, those past the tile its first run again: the number of loads
      // under way is then the same in every wave.  A run past the end of k is
      // zero with a scale of zero: that of another group could be negative, and
      // put() would turn the run into NaN.
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = (i * THREADS + tid) % (R * kRuns);
        const int64_t k = k0 + at % kRuns * 16, grp = k / kRows;
        int64_t r = r0 + at / kRuns;
        r = r < rows ? r : rows - 1;
        const bool in = k < K;
        const int64_t o = in ? grp * rows + r : 0;
        u32x4 q = *reinterpret_cast<const u32x4*>(static_cast<const int8_t*>(p) + o * kRows + (in ? k % kRows : 0));
        if (!in) q = u32x4{0, 0, 0, 0};
        __builtin_memcpy(&g.v[i], &q, 16);
        const uint16_t sb = scales[o];
        g.s[i] = in ? sb : (uint16_t)0;
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

  // Codes of whole steps, one after another: offsets from the step's first
  // group that stay the same (below 2^28 bytes), so that a load costs no
  // vector instruction.  The caller moves the bases on.
  struct Codes {
    uint32_t off[kLoads], soff[kLoads];
    const char *base, *sbase;
    int64_t step;     // groups' rows of a step
  };

  static __device__ __forceinline__ void start_codes(Codes& c, const void* p, const uint16_t* scales, int64_t rows,
                                                     int64_t r0, int64_t k0, int tid) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = (i * THREADS + tid) % (R * kRuns);
      const int k = at % kRuns * 16;
      int64_t r = r0 + at / kRuns;
      r = r < rows ? r : rows - 1;
      const uint32_t o = (uint32_t)(k / kRows * rows + r);
      c.off[i] = o * kRows + k % kRows;
      c.soff[i] = o * 2;
    }
    c.base = static_cast<const char*>(p) + k0 * rows;
    c.sbase = reinterpret_cast<const char*>(scales + k0 / kRows * rows);
    c.step = kStep / kRows * rows;
  }

  static __device__ __forceinline__ void fetch_all(const Codes& c, Regs& g) {
    const __amdgpu_buffer_rsrc_t q =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(c.base), 0, 0x7fffffff, 0x00020000);
    const __amdgpu_buffer_rsrc_t s =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(c.sbase), 0, 0x7fffffff, 0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(q, (int)c.off[i], 0, 0);
      __builtin_memcpy(&g.v[i], &v, 16);
      g.s[i] = __builtin_amdgcn_raw_buffer_load_b16(s, (int)c.soff[i], 0, 0);
    }
  }

  // The same of whole steps: every chunk by one load.  (A column chunk that runs
  // past the last row reads on into what follows it in memory, which the k
  // after the last whole step leave room for: slack(); those sums are not
  // stored.)
  static __device__ __forceinline__ int64_t slack(int64_t ld) { return MODE == kCol ? (E + ld - 1) / ld : 0; }

  static __device__ __forceinline__ void fetch_whole(const Copy& s, Regs& g) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) __builtin_memcpy(&g.v[i], s.base + s.off[i], 16);
  }

  static __device__ __forceinline__ void put(const Regs& g, V* lds, int tid) {
    if (MODE == kCodes) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = i * THREADS + tid;
        if (R * kRuns % THREADS && at >= R * kRuns) break;
        const int r = at / kRuns, c0 = at % kRuns * (16 / E);
        // a group with a non-finite value counts as NaN whole: its column of
        // the gradient is not finite in either case
        const uint16_t s = g.s[i];
        const float f = (s & 0x8000u) ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)s << 16);
        uint32_t q[4];
        __builtin_memcpy(q, &g.v[i], 16);
        // codes + 128 are bytes, which convert in one instruction; the
        // products and their difference are exact
        const float shift = -128.f * f;
#pragma unroll
        for (int w = 0; w < 4; ++w) q[w] ^= 0x80808080u;
#pragma unroll
        for (int u = 0; u < 16 / E; ++u) {
          V v;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int j = u * E + e;
            v[e] = (T)__builtin_fmaf((float)((q[j >> 2] >> (8 * (j & 3))) & 255u), f, shift);
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
// Waits until at most N of this wave's loads are under way.
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N < 64, "six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
  asm volatile("" ::: "memory");
}

// A workgroup barrier that leaves loads under way: this wave's LDS reads and
// writes are done, and none moves across it.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);   // LDS
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

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
  float z[kN];
  uint32_t top = 0;     // the largest magnitude's bits
#pragma unroll
  for (int r = 0; r < kN; ++r) {
    z[r] = r0 + r < rows ? strip[(r0 + r) * (WJ + 4) + col] + b : 0.f;
    const uint32_t m = __float_as_uint(z[r]) & 0x7fffffffu;
    top = m > top ? m : top;
  }
  if (WJ == 32) {
    const uint32_t m = __shfl_xor(top, 32);
    top = m > top ? m : top;
  }
  const int64_t at = (i0 / kRows) * J + j;
  uint16_t s;
  uint32_t w[kN / 4];
  const bool plain = q8_plain(top, kEmax<float>);
  if (plain) {
    const Q8 q = q8_of(__uint_as_float(top), kEmin<float>, kEmax<float>);
#pragma unroll
    for (int r = 0; r < kN; r += 4) w[r >> 2] = q8_codes4(z[r], z[r + 1], z[r + 2], z[r + 3], q.inv);
    s = q8_scale_bits(q, false);
  }
  // (both lanes of a column agree which)
  if (!plain) {
    float amax = 0.f;
    int bad = 0;
#pragma unroll 1
    for (int r = 0; r < kRows; ++r) {
      const float v = r < rows ? strip[r * (WJ + 4) + col] + b : 0.f;
      if (finite_bits(v))
        amax = fmaxf(amax, fabsf(v));
      else
        bad = 1;
    }
    const Q8 q = q8_of(amax, kEmin<float>, kEmax<float>);
    s = q8_scale_bits(q, bad != 0);
    if (j < J) {
#pragma unroll 1
      for (int r = r0; r < r0 + kN; ++r)
        codes[at * kRows + r] = (int8_t)q8_code(r < rows ? strip[r * (WJ + 4) + col] + b : 0.f, q);
      if (lane < WJ) scales[at] = s;
    }
    return;
  }
  if (j >= J) return;
#pragma unroll
  for (int o = 0; o < kN / 16; ++o)
    *reinterpret_cast<u32x4*>(codes + at * kRows + r0 + 16 * o) =
        u32x4{w[4 * o], w[4 * o + 1], w[4 * o + 2], w[4 * o + 3]};
  if (lane < WJ) scales[at] = s;
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
    T* out = y + i * ldy + j;
    const T* r = res ? res + i * ldr + j : nullptr;
    V bv, rv, o;
#pragma unroll
    for (int e = 0; e < E; ++e) bv[e] = rv[e] = (T)0.f;
    if (n >= E) {
      if (bias) __builtin_memcpy(&bv, bias + j, 16);
      if (r) __builtin_memcpy(&rv, r, 16);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (bias && e < n) bv[e] = bias[j + e];
        if (r && e < n) rv[e] = r[e];
      }
    }
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = strip[row * (WJ + 4) + col + e];
    if (bias)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += (float)bv[e];
    if (act != kActNone)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = act_value(v[e], act);
    if (r)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += (float)rv[e];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = (T)v[e];
    if (n >= E) {
      __builtin_memcpy(out, &o, 16);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < n) out[e] = o[e];
    }
  }
}

// ---------------------------------------------------------------- product
template <int N>
struct Half {
  static constexpr int value = N;
};

// Consecutive workgroups go to the 8 dies in turn: each die is given a
// contiguous run of tiles, in bands of 8 tile rows, so that its L2 holds the
// rows of A and B that its workgroups share.
struct Place {
  int part, i, j;
};

__device__ __forceinline__ Place place_of(int ti, int tj, int splits) {
  const int n = ti * tj * splits, per = n / 8, rest = n % 8, die = blockIdx.x % 8;
  int id = die * per + (die < rest ? die : rest) + blockIdx.x / 8;
  Place p;
  p.part = id / (ti * tj);
  id -= p.part * ti * tj;
  const int band = id / (8 * tj), high = ti - band * 8 < 8 ? ti - band * 8 : 8, in = id - band * 8 * tj;
  p.i = band * 8 + in % high;
  p.j = in / high;
  return p;
}

// The sums of a wave (columns lane & 31 of its 32 x 32 tiles, rows 8 (r / 4) +
// 4 (lane / 32) + r % 4 for r = 0..15) through its strip of LDS, so that a lane
// stores 16 bytes of one row.
template <class T, int NI, int NJ>
__device__ __forceinline__ void finish(const GemmArgs& g, int part, f32x16 (&acc)[NI][NJ], float* strip, int lane,
                                       int64_t i0, int64_t j0) {
  constexpr int WJ = 32 * NJ;
  const T* bias = static_cast<const T*>(g.bias);
#pragma unroll
  for (int x = 0; x < NI; ++x) {
    const int64_t ib = i0 + 32 * x;
#pragma unroll
    for (int y = 0; y < NJ; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        strip[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * (WJ + 4) + 32 * y + (lane & 31)] = acc[x][y][r];
    wave_sync();
    if (g.splits > 1) {
      put_strip<float, WJ>(g.part + (int64_t)part * g.I * g.J, g.J, nullptr, nullptr, 0, kActNone, strip, lane, ib,
                           j0, g.I, g.J);
    } else {
      if (g.zcodes && ib < g.I) checkpoint_strip<T, WJ>(g.zcodes, g.zscales, bias, strip, lane, ib, j0, g.I, g.J);
      put_strip<T, WJ>(static_cast<T*>(g.y), g.ldy, bias, static_cast<const T*>(g.residual), g.ldr, g.act, strip, lane,
                       ib, j0, g.I, g.J);
    }
    wave_sync();
  }
}

// The smallest products, and those whose operands cannot be copied: BT x BT of
// C per workgroup of four waves, a quarter each in 32 x 32 matrix instructions,
// 128 bytes of k a step through four LDS buffers.  COPY: both operands straight
// into LDS, three steps under way; otherwise through registers, four steps
// under way (codes always so, becoming T on the way).  No step has a branch:
// what is left of k beyond whole steps goes first, and steps past the last
// fetch that one again, into buffers that nothing reads any more.  Tiles of 64
// leave the matrix instructions idle 0.4 of the time in fp32, while a SIMD's
// one wave reads its operands (500 tokens, 1024 -> 2048: 22 us; eight waves in
// turns, as below, take as long), and are bound by a step's latency in 16 bits
// (fp16 through registers, 333 tokens, 777 -> 1000: 11 us).
template <class T, int AM, int BM, int BT, bool COPY>
__global__ __launch_bounds__(256) void gemm_kernel(GemmArgs g, int ti, int tj) {
  constexpr int kThreads = 256, W = BT / 2, NT = W / 32;
  using TA = Tile<T, AM, BT, kThreads>;
  using TB = Tile<T, BM, BT, kThreads>;
  using V = typename Vec<T>::type;
  constexpr bool kCopyA = COPY && AM != kCodes, kCopyB = COPY && BM != kCodes;
  // Buffers of their own names: the compiler then knows that a copy into one
  // does not touch what is read from another, and waits for neither.  The
  // epilogue's strips (32 rows x W sums a wave, rows padded by 16 bytes) lie in
  // them, a wave's in each.
  constexpr int kBuf = TA::kChunks + TB::kChunks, kStrip = 32 * (W + 4);
  static_assert(kStrip * 4 <= kBuf * 16, "a strip fits a buffer");
  __shared__ __align__(16) V lds0[kBuf];
  __shared__ __align__(16) V lds1[kBuf];
  __shared__ __align__(16) V lds2[kBuf];
  __shared__ __align__(16) V lds3[kBuf];

  const Place p = place_of(ti, tj, g.splits);
  const int64_t i0 = (int64_t)p.i * BT, j0 = (int64_t)p.j * BT;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wi = (wave >> 1) * W, wj = (wave & 1) * W;
  f32x16 acc[NT][NT];
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int y = 0; y < NT; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;

  // Whole steps; through registers a few k stay after them.
  const int64_t sa = COPY ? 0 : TA::slack(g.lda), sb = COPY ? 0 : TB::slack(g.ldb), after = sa > sb ? sa : sb;
  const int64_t all = g.K > after ? (g.K - after) / TA::kStep : 0;
  const int64_t first = all * p.part / g.splits;
  const int steps = (int)(all * (p.part + 1) / g.splits - first);
  auto products = [&](const V* now) __attribute__((always_inline)) {
    V fa[4][NT], fb[4][NT];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        fa[kk][x] = TA::operand(now, wi + 32 * x, kk, lane);
        fb[kk][x] = TB::operand(now + TA::kChunks, wj + 32 * x, kk, lane);
      }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y) mma<T>(fa[kk][x], fb[kk][y], acc[x][y]);
  };
  // (one step's worth, or through registers up to two)
  if (p.part == g.splits - 1)
#pragma unroll 1
    for (int64_t k0 = all * TA::kStep; k0 < g.K; k0 += TA::kStep) {
      typename TA::Regs ra;
      typename TB::Regs rb;
      if constexpr (kCopyA) {
        TA::copy_rest(g.a, g.lda, g.I, g.K, i0, k0, lds0, tid);
      } else {
        TA::fetch(g.a, g.lda, nullptr, g.I, g.K, i0, k0, ra, tid);
        TA::put(ra, lds0, tid);
      }
      if constexpr (kCopyB) {
        TB::copy_rest(g.b, g.ldb, g.J, g.K, j0, k0, lds0 + TA::kChunks, tid);
      } else {
        TB::fetch(g.b, g.ldb, g.bscales, g.J, g.K, j0, k0, rb, tid);
        TB::put(rb, lds0 + TA::kChunks, tid);
      }
      wait_copies<0>();
      lds_barrier();
      products(lds0);
      lds_barrier();
    }
  if (steps > 0) {
    typename TA::Copy ca;
    typename TB::Copy cb;
    typename TB::Codes codes;
    // slots of registers for the operands that take them
    typename TA::Regs ra[4];
    typename TB::Regs rb[4];
    TA::template start<kCopyA>(ca, g.a, g.lda, g.I, i0, first * TA::kStep, tid);
    if constexpr (BM == kCodes)
      TB::start_codes(codes, g.b, g.bscales, g.J, j0, first * TA::kStep, tid);
    else
      TB::template start<kCopyB>(cb, g.b, g.ldb, g.J, j0, first * TA::kStep, tid);
    auto copy = [&](int s, V* lds) __attribute__((always_inline)) {
      if constexpr (kCopyA) {
        TA::copy(ca, lds, tid);
        ca.base += s + 1 < steps ? ca.step : 0;
      }
      if constexpr (kCopyB) {
        TB::copy(cb, lds + TA::kChunks, tid);
        cb.base += s + 1 < steps ? cb.step : 0;
      }
    };
    auto fetch = [&](int s, int slot) __attribute__((always_inline)) {
      asm volatile("" ::: "memory");
      if constexpr (!kCopyA) {
        TA::fetch_whole(ca, ra[slot]);
        ca.base += s + 1 < steps ? ca.step : 0;
      }
      if constexpr (BM == kCodes) {
        TB::fetch_all(codes, rb[slot]);
        codes.base += s + 1 < steps ? codes.step * kRows : 0;
        codes.sbase += s + 1 < steps ? codes.step * 2 : 0;
      } else if constexpr (!kCopyB) {
        TB::fetch_whole(cb, rb[slot]);
        cb.base += s + 1 < steps ? cb.step : 0;
      }
      asm volatile("" ::: "memory");
    };
    auto put = [&](int slot, V* lds) __attribute__((always_inline)) {
      if constexpr (!kCopyA) TA::put(ra[slot], lds, tid);
      if constexpr (!kCopyB) TB::put(rb[slot], lds + TA::kChunks, tid);
    };
    // Two steps' copies, and the codes loaded after them, may be under way when
    // a step's copies have landed.  (A run of codes is two loads, its codes and
    // its scale, and counts as one here: with codes the wait is for more than the
    // step needs, never for less.)
    constexpr int kD = (kCopyA ? TA::kPer : 0) + (kCopyB ? TB::kPer : 0);
    constexpr int kF = kCopyA && !kCopyB ? TB::kLoads : 0;
    // Step s from `now`; `last` (read by every wave in step s - 1) receives step
    // s + 3's copies, `then` (in step s - 2) step s + 2's registers.
    auto step = [&](int s, int slot, V* now, V* then, V* last) __attribute__((always_inline)) {
      if (kD > 0) wait_copies<2 * kD + 2 * kF>();
      lds_barrier();
      copy(s + 3, last);
      put(slot, then);
      fetch(s + 6, slot);
      products(now);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) fetch(i, i);
    put(0, lds0);
    put(1, lds1);
    copy(0, lds0);
    copy(1, lds1);
    copy(2, lds2);
#pragma unroll
    for (int i = 2; i < 6; ++i) fetch(i, i & 3);
#pragma unroll 1
    for (int s = 0; s < steps; s += 4) {
      step(s, 2, lds0, lds2, lds3);
      if (s + 1 == steps) break;
      step(s + 1, 3, lds1, lds3, lds0);
      if (s + 2 == steps) break;
      step(s + 2, 0, lds2, lds0, lds1);
      if (s + 3 == steps) break;
      step(s + 3, 1, lds3, lds1, lds2);
    }
    wait_copies<0>();
  }
  __syncthreads();
  V* const in = wave == 0 ? lds0 : wave == 1 ? lds1 : wave == 2 ? lds2 : lds3;
  finish<T, NT, NT>(g, p.part, acc, reinterpret_cast<float*>(in), lane, i0 + wi, j0 + wj);
}

// The same for large products: 256 x 256 of C per workgroup of eight waves, 128
// x 64 of them per wave, both operands always copied.
//
// A step's 128 bytes of k are multiplied in two halves: first the upper 64 rows
// of each wave's part, then the lower 64 with the operands of B kept in
// registers.  B's tile and A's upper half tile are then free half a step before
// A's lower one, and each is refilled at once for the step after next: every
// copy has a step and a half to travel, at any time there are copies under way,
// and two buffers suffice.  (With all copies started at the beginning of a step
// and waited for at its end the copies alone took 3460 cycles a step, the
// matrix instructions 2048.)
//
// A half has a reading and a multiplying turn, and the second four waves run
// one turn behind the first: while one wave of a SIMD multiplies, the other
// reads its operands from LDS and starts copies.  The turn before the first
// waves read a tile is a reading one of the second four's: by its end every
// wave has seen its copies of that tile land.
//
// 8192 cubed on one card: bf16 769 us (1.43 PFLOP/s; the library's product 698,
// on others 781 and 784, 791 and 870), dx 781, dW 775; fp32 7.55 ms (146
// TFLOP/s, the library 7.20), dx 7.66, dW 8.30.  Bound by the matrix
// instructions at the clock that they leave.  4096 tokens, 2048 -> 8192 with
// SiLU and a checkpoint take 139 us, without the checkpoint 125, the bare
// product 114: in the epilogues all workgroups write at once (100 MB) and none
// multiplies.
template <class T, int AM, int BM>
__global__ __launch_bounds__(512) void gemm_large_kernel(GemmArgs g, int ti, int tj) {
  constexpr int kThreads = 512, BT = 256, NJ = 2;
  using TA = Tile<T, AM, 128, kThreads, 64, 128>;   // half h: rows 64 h of every 128
  using TB = Tile<T, BM, 256, kThreads>;
  using V = typename Vec<T>::type;
  // tiles of their own names (see gemm_kernel)
  __shared__ __align__(16) V up0[TA::kChunks];
  __shared__ __align__(16) V up1[TA::kChunks];
  __shared__ __align__(16) V low0[TA::kChunks];
  __shared__ __align__(16) V low1[TA::kChunks];
  __shared__ __align__(16) V b0[TB::kChunks];
  __shared__ __align__(16) V b1[TB::kChunks];
  constexpr int kStrip = 32 * (64 + 4);   // 8.5 KB
  static_assert(3 * kStrip * 4 <= TB::kChunks * 16 && kStrip * 4 <= TA::kChunks * 16, "strips fit the tiles");

  const Place p = place_of(ti, tj, g.splits);
  const int64_t i0 = (int64_t)p.i * BT, j0 = (int64_t)p.j * BT;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wi = (wave >> 2) * 128, wj = (wave & 3) * 64;
  const bool behind = wave >= 4;
  f32x16 acc[4][NJ];
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < NJ; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;

  // Whole steps; what is left of k goes first, on its own.
  const int64_t all = g.K / TA::kStep;
  const int64_t first = all * p.part / g.splits;
  const int steps = (int)(all * (p.part + 1) / g.splits - first);
  V fa[4][2], fb[4][NJ];
  int at = lane;
  auto read_a = [&](const V* a) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x) fa[kk][x] = TA::operand(a, wi / 2 + 32 * x, kk, at);
  };
  auto read_b = [&](const V* b) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int y = 0; y < NJ; ++y) fb[kk][y] = TB::operand(b, wj + 32 * y, kk, at);
  };
  auto multiply = [&](auto half) __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < NJ; ++y) mma<T>(fa[kk][x], fb[kk][y], acc[2 * decltype(half)::value + x][y]);
    __builtin_amdgcn_s_setprio(0);
  };
  // (a lower half past the last row reads from the first)
  const int64_t il = i0 + 64 < g.I ? i0 + 64 : i0;
  if (g.K % TA::kStep && p.part == g.splits - 1) {
    const int64_t k0 = all * TA::kStep;
    TA::copy_rest(g.a, g.lda, g.I, g.K, i0, k0, up0, tid);
    TA::copy_rest(g.a, g.lda, g.I, g.K, il, k0, low0, tid);
    TB::copy_rest(g.b, g.ldb, g.J, g.K, j0, k0, b0, tid);
    wait_copies<0>();
    lds_barrier();
    read_b(b0);
    read_a(up0);
    multiply(Half<0>());
    read_a(low0);
    multiply(Half<1>());
    lds_barrier();
  }
  if (steps > 0) {
    typename TA::Copy cu, cl;
    typename TB::Copy cb;
    TA::start(cu, g.a, g.lda, g.I, i0, first * TA::kStep, tid);
    TA::start(cl, g.a, g.lda, g.I, il, first * TA::kStep, tid);
    TB::start(cb, g.b, g.ldb, g.J, j0, first * TA::kStep, tid);
    // Copies of step s; past the last they fetch that one again, into tiles
    // that nothing reads any more, so that no turn has a branch (with branches
    // for the end in it a step took 3200 cycles, without them 2360).
    auto copy_upper = [&](int s, V* up, V* b) __attribute__((always_inline)) {
      TB::copy(cb, b, tid);
      cb.base += s + 1 < steps ? cb.step : 0;
      TA::copy(cu, up, tid);
      cu.base += s + 1 < steps ? cu.step : 0;
    };
    auto copy_lower = [&](int s, V* lo) __attribute__((always_inline)) {
      TA::copy(cl, lo, tid);
      cl.base += s + 1 < steps ? cl.step : 0;
    };
    // What may be under way when the next turn's tiles have landed: all of one
    // step's copies.
    constexpr int kNew = 2 * TA::kPer + TB::kPer;
    // Step s in the tiles up, lo, b; the other parity's lower one is lo2.
    auto step = [&](int s, V* up, V* lo, V* b, V* lo2) __attribute__((always_inline)) {
      // (fp32 columns: the addresses, worked out before the loop, would not leave
      // the values registers enough; spilled, 8192 cubed took 14.5 ms, not 8.3)
      if (AM == kCol && sizeof(T) == 4) asm volatile("" : "+v"(at));
      read_b(b);
      read_a(up);
      // step s - 1's lower half has been read by every wave
      copy_lower(s + 1, lo2);
      wait_copies<kNew>();
      lds_barrier();
      multiply(Half<0>());
      lds_barrier();
      // this step's B and upper half have
      copy_upper(s + 2, up, b);
      read_a(lo);
      wait_copies<kNew>();
      lds_barrier();
      multiply(Half<1>());
      lds_barrier();
    };
    copy_upper(0, up0, b0);
    copy_lower(0, low0);
    copy_upper(1, up1, b1);
    wait_copies<kNew>();
    lds_barrier();
    if (behind) lds_barrier();
#pragma unroll 1
    for (int s = 0; s < steps; s += 2) {
      step(s, up0, low0, b0, low1);
      if (s + 1 == steps) break;
      step(s + 1, up1, low1, b1, low0);
    }
    if (!behind) lds_barrier();
    wait_copies<0>();
  }
  __syncthreads();
  // strips: three in each tile of B, one in each of two of A's
  V* const in = wave < 3 ? b0 : wave < 6 ? b1 : wave == 6 ? up0 : up1;
  finish<T, 4, NJ>(g, p.part, acc, reinterpret_cast<float*>(in) + (wave < 6 ? wave % 3 : 0) * kStrip, lane, i0 + wi,
                   j0 + wj);
}

// For products of too few such tiles to fill the CUs: 128 x 128 of C per
// workgroup of eight waves, A always copied, three of four buffers' copies under
// way.  A wave takes 64 x 64 of C, four of them the even steps of k, four the
// odd: in each turn one four read the next step's operands from LDS while the
// others multiply the last one's, and the two sums meet in LDS at the end.
// (With 64 x 32 and every step for each wave the operands' reads took 768 cycles
// of LDS a step, the matrix instructions 512: 74 us; with half of each step's k
// 69.)  bf16, 2048 tokens, 8192 -> 2048: 69 us, 1.0 PFLOP/s, the matrix
// instructions busy 0.55 of the time; fp32 2048 cubed 129.
template <class T, int AM, int BM>
__global__ __launch_bounds__(512) void gemm_mid_kernel(GemmArgs g, int ti, int tj) {
  constexpr int kThreads = 512, BT = 128;
  using TA = Tile<T, AM, BT, kThreads>;
  using TB = Tile<T, BM, BT, kThreads>;
  using V = typename Vec<T>::type;
  constexpr bool kCopyB = BM != kCodes;
  constexpr int kBuf = TA::kChunks + TB::kChunks, kStrip = 32 * (64 + 4), kGiven = 2 * 16 * 64;
  static_assert(3 * kStrip * 4 <= kBuf * 16 && 4 * kGiven * 4 <= kBuf * 16, "strips and sums fit the buffers");
  __shared__ __align__(16) V lds0[kBuf];
  __shared__ __align__(16) V lds1[kBuf];
  __shared__ __align__(16) V lds2[kBuf];
  __shared__ __align__(16) V lds3[kBuf];

  const Place p = place_of(ti, tj, g.splits);
  const int64_t i0 = (int64_t)p.i * BT, j0 = (int64_t)p.j * BT;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wi = (wave >> 1 & 1) * 64, wj = (wave & 1) * 64;
  const bool odd = __builtin_amdgcn_readfirstlane(wave) >= 4;   // takes the odd steps
  f32x16 acc[2][2];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;

  // Whole steps; what is left of k goes first, on its own.
  const int64_t all = g.K / TA::kStep;
  const int64_t first = all * p.part / g.splits;
  const int steps = (int)(all * (p.part + 1) / g.splits - first);
  V fa[4][2], fb[4][2];
  auto read = [&](const V* lds) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        fa[kk][x] = TA::operand(lds, wi + 32 * x, kk, lane);
        fb[kk][x] = TB::operand(lds + TA::kChunks, wj + 32 * x, kk, lane);
      }
  };
  auto multiply = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) mma<T>(fa[kk][x], fb[kk][y], acc[x][y]);
    __builtin_amdgcn_s_setprio(0);
  };
  typename TB::Regs rb[2];
  if (g.K % TA::kStep && p.part == g.splits - 1) {
    const int64_t k0 = all * TA::kStep;
    TA::copy_rest(g.a, g.lda, g.I, g.K, i0, k0, lds0, tid);
    if constexpr (kCopyB) {
      TB::copy_rest(g.b, g.ldb, g.J, g.K, j0, k0, lds0 + TA::kChunks, tid);
    } else {
      TB::fetch(g.b, g.ldb, g.bscales, g.J, g.K, j0, k0, rb[0], tid);
      TB::put(rb[0], lds0 + TA::kChunks, tid);
    }
    wait_copies<0>();
    lds_barrier();
    if (!odd) {
      read(lds0);
      multiply();
    }
    lds_barrier();
  }
  if (steps > 0) {
    typename TA::Copy ca;
    typename TB::Copy cb;
    typename TB::Codes codes;
    TA::start(ca, g.a, g.lda, g.I, i0, first * TA::kStep, tid);
    if constexpr (kCopyB)
      TB::start(cb, g.b, g.ldb, g.J, j0, first * TA::kStep, tid);
    else
      TB::start_codes(codes, g.b, g.bscales, g.J, j0, first * TA::kStep, tid);
    // step s; past the last that one again (see gemm_large_kernel)
    auto copy = [&](int s, V* lds) __attribute__((always_inline)) {
      TA::copy(ca, lds, tid);
      ca.base += s + 1 < steps ? ca.step : 0;
      if constexpr (kCopyB) {
        TB::copy(cb, lds + TA::kChunks, tid);
        cb.base += s + 1 < steps ? cb.step : 0;
      }
    };
    // codes: two steps' under way
    auto fetch = [&](int s, int slot) __attribute__((always_inline)) {
      if constexpr (!kCopyB) {
        asm volatile("" ::: "memory");
        TB::fetch_all(codes, rb[slot]);
        asm volatile("" ::: "memory");
        codes.base += s + 1 < steps ? codes.step * kRows : 0;
        codes.sbase += s + 1 < steps ? codes.step * 2 : 0;
      }
    };
    auto put = [&](int slot, V* lds) __attribute__((always_inline)) {
      if constexpr (!kCopyB) TB::put(rb[slot], lds + TA::kChunks, tid);
    };
    constexpr int kD = TA::kPer + (kCopyB ? TB::kPer : 0), kF = kCopyB ? 0 : TB::kLoads;
    // What every wave does in turn t: step t + 3's copies go to the buffer read
    // in turn t - 1, step t + 2's codes to that of turn t - 2.  Two steps' copies
    // and codes may be under way when those of turn t + 1 have landed.  (A run
    // of codes is two loads and counts as one: the wait is then for some of turn
    // t + 2's copies too.)
    auto feed = [&](int t, int slot, V* then, V* last) __attribute__((always_inline)) {
      copy(t + 3, last);
      put(slot, then);
      fetch(t + 4, slot);
    };
    auto end = [&]() __attribute__((always_inline)) {
      wait_copies<2 * kD + 2 * kF>();
      lds_barrier();
    };
    auto read_turn = [&](int t, int slot, V* now, V* then, V* last) __attribute__((always_inline)) {
      feed(t, slot, then, last);
      read(now);
      end();
    };
    auto multiply_turn = [&](int t, int slot, V* then, V* last) __attribute__((always_inline)) {
      // (of 16 bits the instructions are soon done: with the copies started
      // before them 71 us, after them 69; in fp32 the reverse, 132 and 137)
      if (sizeof(T) == 4) feed(t, slot, then, last);
      multiply();
      if (sizeof(T) == 2) feed(t, slot, then, last);
      end();
    };
    fetch(0, 0);
    fetch(1, 1);
    put(0, lds0);
    put(1, lds1);
    copy(0, lds0);
    copy(1, lds1);
    copy(2, lds2);
    fetch(2, 0);
    fetch(3, 1);
    end();
    // turns 0 .. steps, one barrier each; what is read in turn `steps` is not used
    if (!odd) {
#pragma unroll 1
      for (int t = 0; t <= steps; t += 4) {
        read_turn(t, 0, lds0, lds2, lds3);
        if (t + 1 > steps) break;
        multiply_turn(t + 1, 1, lds3, lds0);
        if (t + 2 > steps) break;
        read_turn(t + 2, 0, lds2, lds0, lds1);
        if (t + 3 > steps) break;
        multiply_turn(t + 3, 1, lds1, lds2);
      }
    } else {
      feed(0, 0, lds2, lds3);
      end();
#pragma unroll 1
      for (int t = 1; t <= steps; t += 4) {
        read_turn(t, 1, lds1, lds3, lds0);
        if (t + 1 > steps) break;
        multiply_turn(t + 1, 0, lds0, lds1);
        if (t + 2 > steps) break;
        read_turn(t + 2, 1, lds3, lds1, lds2);
        if (t + 3 > steps) break;
        multiply_turn(t + 3, 0, lds2, lds3);
      }
    }
    wait_copies<0>();
  }
  __syncthreads();
  // Of its 64 rows a wave of the even steps keeps the upper 32, one of the odd
  // the lower; it adds what the other wave has of them.
  f32x16 sum[1][2];
  float* const given = reinterpret_cast<float*>(wave < 4 ? lds0 : lds1) + (wave & 3) * kGiven + lane;
  const float* const got = reinterpret_cast<float*>(wave < 4 ? lds1 : lds0) + (wave & 3) * kGiven + lane;
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      given[(16 * y + r) * 64] = odd ? acc[0][y][r] : acc[1][y][r];
      sum[0][y][r] = odd ? acc[1][y][r] : acc[0][y][r];
    }
  __syncthreads();
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[0][y][r] += got[(16 * y + r) * 64];
  __syncthreads();
  // strips: three in each of two buffers, two in another
  V* const in = wave < 3 ? lds0 : wave < 6 ? lds1 : lds2;
  finish<T, 1, 2>(g, p.part, sum, reinterpret_cast<float*>(in) + wave % 3 * kStrip, lane, i0 + wi + 32 * odd,
                  j0 + wj);
}

// The epilogue of a product whose k was split: the parts' sum (always in the
// same order), bias, activation, residual.  A thread per value, or with a
// checkpoint per four rows of a group of one column, eight of which agree on
// the group's scale through LDS.  Bound by reading the parts, and by its launch.
template <class T, bool CODES>
__global__ __launch_bounds__(256) void join_kernel(GemmArgs g) {
  constexpr int kShare = 8, kN = CODES ? kRows / kShare : 1, kWide = 256 / kShare;
  __shared__ uint32_t tops[kShare][kWide];
  __shared__ int bads[kShare][kWide];
  const int lane = threadIdx.x % kWide, share = CODES ? threadIdx.x / kWide : 0;
  const T* bias = static_cast<const T*>(g.bias);
  const T* res = static_cast<const T*>(g.residual);
  const int64_t j = CODES ? (int64_t)blockIdx.y * kWide + lane : (int64_t)blockIdx.y * 256 + threadIdx.x;
  const int64_t size = g.I * g.J, i0 = CODES ? (int64_t)blockIdx.x * kRows + share * kN : (int64_t)blockIdx.x;
  float z[kN];
#pragma unroll
  for (int r = 0; r < kN; ++r) z[r] = 0.f;
  if (j < g.J) {
    const float b = bias ? (float)bias[j] : 0.f;
    const float* p[kN];
#pragma unroll
    for (int r = 0; r < kN; ++r) p[r] = g.part + (i0 + r < g.I ? i0 + r : g.I - 1) * g.J + j;
#pragma unroll 8
    for (int q = 0; q < g.splits; ++q)
#pragma unroll
      for (int r = 0; r < kN; ++r) z[r] += p[r][q * size];
#pragma unroll
    for (int r = 0; r < kN; ++r) z[r] = i0 + r < g.I ? z[r] + b : 0.f;
  }
  if (CODES) {
    // the largest finite magnitude, and whether all are finite
    uint32_t top = 0;
    int bad = 0;
#pragma unroll
    for (int r = 0; r < kN; ++r) {
      const uint32_t m = __float_as_uint(z[r]) & 0x7fffffffu;
      if (m < 0x7f800000u)
        top = m > top ? m : top;
      else
        bad = 1;
    }
    tops[share][lane] = top;
    bads[share][lane] = bad;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kShare; ++q) {
      top = tops[q][lane] > top ? tops[q][lane] : top;
      bad |= bads[q][lane];
    }
    if (j < g.J) {
      const Q8 q = q8_of(__uint_as_float(top), kEmin<float>, kEmax<float>);
      const int64_t at = blockIdx.x * g.J + j;
#pragma unroll
      for (int r = 0; r < kN; r += 4) {
        uint32_t w = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) w |= (uint32_t)(q8_code(z[(r + u) % kN], q) & 255) << (8 * u);
        *reinterpret_cast<uint32_t*>(g.zcodes + at * kRows + share * kN + r) = w;
      }
      if (share == 0) g.zscales[at] = q8_scale_bits(q, bad != 0);
    }
  }
  if (j >= g.J) return;
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
