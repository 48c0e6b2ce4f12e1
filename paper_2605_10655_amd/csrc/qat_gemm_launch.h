// qat_gemm_launch.h -- choice of the product's tile and split, and its launch.
// Instantiated for one type in each of qat_gemm_{bf16,f16,f32}.hip.
#pragma once
#include <cstddef>
#include <cstdint>

#include "bcjr.h"
#include "qat_gemm_kernels.h"

namespace bcjr {
namespace qlin {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
// a launch has fewer than 2^32 threads along an axis
inline bool grid_fits(int64_t groups, int threads) { return groups < ((int64_t)1 << 32) / threads; }
inline int launched() { return hipGetLastError() == hipSuccess ? BCJR_OK : BCJR_ERR_HIP; }

inline dim3 group_grid(int64_t rows, int64_t cols, int threads) {
  return dim3((unsigned)ceil_div(rows, kRows), (unsigned)ceil_div(cols, threads));
}

// A product's tile and its split of k.
struct GemmPlan {
  int tile;        // 256, 128 or 64
  int ti, tj;      // tiles
  int splits;
  size_t part;     // bytes of the partial sums
};

// The tile and split that a model of the kernels' times finds shortest, in
// cycles (of about 1.5 GHz in 16 bits and 1.1 in fp32, as they run): a step of
// 128 bytes of k, what a workgroup takes before and after its steps, and the
// workgroups that run at once (each measured; fp32 tiles of 64 are bound by the
// matrix instructions, so that one a CU is quicker than two); the parts of a
// split are written, read and joined in a launch of their own.  A part has at
// least four steps.  us, fp32, split in two and whole: 1024 cubed 28.0 and
// 21.5; in four and whole: 512 cubed 10.6 and 12.1.
inline GemmPlan gemm_plan(int dtype, int64_t I, int64_t J, int64_t K) {
  struct Kind {
    int tile;
    double step, fixed;
    int at_once;
  };
  static constexpr Kind half[] = {{256, 2400, 9000, 256}, {128, 700, 4000, 256}, {64, 480, 3000, 512}};
  static constexpr Kind full[] = {{256, 8250, 12000, 256}, {128, 2150, 5000, 256}, {64, 1150, 3500, 512}, {64, 700, 3500, 256}};
  const int64_t steps = ceil_div(K, dtype == kF32 ? 32 : 64);
  GemmPlan best = {};
  double least = 0.;
  const Kind* const kinds = dtype == kF32 ? full : half;
  for (int n = 0; n < (dtype == kF32 ? 4 : 3); ++n) {
    const Kind& k = kinds[n];
    const int64_t ti = ceil_div(I, k.tile), tj = ceil_div(J, k.tile), tiles = ti * tj;
    for (int64_t s = 1; s == 1 || (s <= steps / 4 && s <= 64 && tiles * s <= 2 * k.at_once); ++s) {
      const double rounds = (double)ceil_div(tiles * s, k.at_once);
      double t = rounds * ((double)ceil_div(steps, s) * k.step + k.fixed);
      if (s > 1) t += dtype == kF32 ? 5500. + (double)(s * I * J) / 440. : 9000. + (double)(s * I * J) / 250.;
      if (best.tile == 0 || t < least) {
        least = t;
        best.tile = k.tile;
        best.ti = (int)ti;
        best.tj = (int)tj;
        best.splits = (int)s;
      }
    }
  }
  best.part = best.splits > 1 ? align_up((size_t)best.splits * I * J * sizeof(float)) : 0;
  return best;
}

template <class T, int AM, int BM, int BT, bool COPY>
void launch_gemm(const GemmArgs& g, const GemmPlan& p, hipStream_t stream) {
  hipLaunchKernelGGL((gemm_kernel<T, AM, BM, BT, COPY>), dim3((unsigned)(p.ti * p.tj * p.splits)), dim3(256),
                     0, stream, g, p.ti, p.tj);
}

// Whether tiles of an operand can be copied straight into LDS (Tile::copy).
// padded: rows go on to a whole number of 16 bytes, in an operand by rows with
// zeros (as its k is then multiplied).
inline bool copies(int mode, const void* p, int64_t ld, int64_t rows, int64_t K, int es, int tile, bool padded) {
  if (mode == kCodes) return true;
  const int e = 16 / es;
  return !misaligned(p, 16) && ld % e == 0 && (padded || (mode == kRow ? K : rows) % e == 0) &&
         (int64_t)(mode == kRow ? tile : 8 * e) * ld * es < ((int64_t)1 << 31);
}

// The epilogue of a split product.
template <class T>
int join(const GemmArgs& g, hipStream_t stream) {
  if (g.zcodes)
    hipLaunchKernelGGL((join_kernel<T, true>), group_grid(g.I, g.J, 32), dim3(256), 0, stream, g);
  else
    hipLaunchKernelGGL((join_kernel<T, false>), dim3((unsigned)g.I, (unsigned)ceil_div(g.J, 256)), dim3(256), 0,
                       stream, g);
  return launched();
}

// A product that gemm_plan gives tiles of 256, of operands that can be copied.
template <class T, int AM, int BM>
int gemm_large(GemmArgs g, const GemmPlan& p, void* ws, hipStream_t stream) {
  g.splits = p.splits;
  g.part = static_cast<float*>(ws);
  hipLaunchKernelGGL((gemm_large_kernel<T, AM, BM>), dim3((unsigned)(p.ti * p.tj * p.splits)), dim3(512), 0, stream, g,
                     p.ti, p.tj);
  if (launched() != BCJR_OK) return BCJR_ERR_HIP;
  return p.splits > 1 ? join<T>(g, stream) : BCJR_OK;
}

// The product and its epilogue (of zero sums where K == 0).  a_padded, b_padded:
// as padded of copies().
template <class T, int AM, int BM>
int gemm(GemmArgs g, void* ws, hipStream_t stream, bool a_padded = false, bool b_padded = false) {
  if (g.I == 0 || g.J == 0) return BCJR_OK;
  constexpr int es = (int)sizeof(T), dtype = es == 4 ? kF32 : kBF16;
  GemmPlan p = gemm_plan(dtype, g.I, g.J, g.K);
  // (a tile of 256 may become four workgroups of 512 threads)
  if (!grid_fits((int64_t)p.ti * p.tj * p.splits, p.tile == 256 ? 2048 : p.tile == 128 ? 512 : 256))
    return BCJR_ERR_UNSUPPORTED;
  const bool copied = copies(AM, g.a, g.lda, g.I, g.K, es, p.tile, a_padded) &&
                      copies(BM, g.b, g.ldb, g.J, g.K, es, p.tile, b_padded);
  if constexpr (BM != kCodes)
    if (copied && p.tile == 256) return gemm_large<T, AM, BM>(g, p, ws, stream);
  if (p.tile == 256) {
    p.ti = (int)ceil_div(g.I, 128);
    p.tj = (int)ceil_div(g.J, 128);
  }
  g.splits = p.splits;
  g.part = static_cast<float*>(ws);
  if (copied && p.tile >= 128)
    hipLaunchKernelGGL((gemm_mid_kernel<T, AM, BM>), dim3((unsigned)(p.ti * p.tj * p.splits)), dim3(512), 0, stream, g,
                       p.ti, p.tj);
  else if (copied)
    launch_gemm<T, AM, BM, 64, true>(g, p, stream);
  else if (p.tile >= 128)
    launch_gemm<T, AM, BM, 128, false>(g, p, stream);
  else
    launch_gemm<T, AM, BM, 64, false>(g, p, stream);
  if (launched() != BCJR_OK) return BCJR_ERR_HIP;
  return p.splits > 1 ? join<T>(g, stream) : BCJR_OK;
}

}  // namespace qlin
}  // namespace bcjr
