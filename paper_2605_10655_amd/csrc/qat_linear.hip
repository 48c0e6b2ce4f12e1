// qat_linear.hip -- C ABI of the quantised linear layer (declared in
// include/bcjr.h): argument checks, choice of kernels, workspace carving and
// launches.  Its own translation unit.
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "bcjr.h"
#include "qat_codes_kernels.h"
#include "qat_gemm_launch.h"
#include "qat_linear_kernels.h"
#include "qat_small_kernels.h"

namespace bcjr {
namespace qlin {

#define QAT_GEMM_EXTERN(T)                                                   \
  extern template int gemm<T, kRow, kRow>(GemmArgs, void*, hipStream_t, bool, bool);   \
  extern template int gemm<T, kRow, kCol>(GemmArgs, void*, hipStream_t, bool, bool);   \
  extern template int gemm<T, kCol, kCodes>(GemmArgs, void*, hipStream_t, bool, bool); \
  extern template int gemm_large<T, kCol, kCol>(GemmArgs, const GemmPlan&, void*, hipStream_t);
QAT_GEMM_EXTERN(bf16)
QAT_GEMM_EXTERN(f16)
QAT_GEMM_EXTERN(float)
#undef QAT_GEMM_EXTERN

// qat_codes.hip
bool codes_take(int k, int V, int64_t block, int64_t M, int64_t N, int64_t K);
int codes_linear(const CodesArgs& a, int dtype, int k, int V, hipStream_t stream);
bool dense_large_takes(int k, int V, int64_t block, int64_t B);
int dense_large(const uint32_t* packed, int64_t B, const float* codebook, int n, int k, int V, int64_t block,
                int64_t words, const float* scales, void* W, int dtype, hipStream_t stream);

namespace {

// Columns are below 2^22, so that a group's codes and a tile's offsets stay
// below 2^31.
constexpr int64_t kMaxRows = (int64_t)1 << 31, kMaxCols = (int64_t)1 << 22;

int elem_size(int dtype) { return dtype == kF32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == kF32 || dtype == kBF16 || dtype == kF16; }
bool act_ok(int act) { return act >= kActNone && act <= kActGeluTanh; }
bool dims_ok(int64_t M, int64_t N, int64_t K) { return M >= 0 && N >= 1 && K >= 1; }
// a tile's rows stay within 32-bit offsets
bool strides_fit(int64_t a, int64_t b, size_t es) { return a < (1 << 25) / (int64_t)es && b < (1 << 25) / (int64_t)es; }
bool dims_fit(int64_t M, int64_t N, int64_t K) { return M < kMaxRows && N < kMaxCols && K < kMaxCols; }
template <class F>
int by_type(int dtype, F f) {
  if (dtype == kBF16) return f(bf16());
  if (dtype == kF16) return f(f16());
  return f(float());
}

template <class T>
dim3 band_grid(int64_t rows, int64_t cols) {
  return dim3((unsigned)(ceil_div(rows, kRows) * ceil_div(cols, kGroupThreads * kCols<T>)));
}

bool bands_fit(int dtype, int64_t rows, int64_t cols) {
  const int64_t wide = kGroupThreads * (dtype == kF32 ? kCols<float> : kCols<bf16>);
  return grid_fits(ceil_div(rows, kRows) * ceil_div(cols, wide), kGroupThreads);
}

// n rounded up to whole 16 bytes
int64_t whole(int dtype, int64_t n) {
  const int e = 16 / elem_size(dtype);
  return ceil_div(n, e) * e;
}

// Whether operands of a product I x J whose rows of n values make no whole 16
// bytes (along k, or b's columns) are padded first: where tiles are large, each
// value padded is used often and a launch of 4 us is little (bf16, us, padded and through registers: 8191 x 6282, K = 1023 147 and
// 389, 4096 x 4097, K = 4099 227 and 322, 3666 x 224, K = 4685 43 and 42; fp32:
// 888 and 1024, 1186 and 1184, 108 and 95; bf16 1000 x 777, K = 999 14.0 and 13.1).
bool pads(const GemmPlan& p, int dtype, int64_t I, int64_t J, int64_t K, int64_t n) {
  return p.tile >= 128 && I >= 512 && J >= 512 && (double)I * J * K >= 2147483648. && whole(dtype, n) != n;
}

template <class T>
int pad(const void* a, int64_t lda, int64_t rows, int64_t cols, void* to, const void* b, int64_t ldb, int64_t brows,
        void* bto, hipStream_t stream) {
  const int64_t chunks = ceil_div(cols, kPer16<T>);
  const int64_t first = ceil_div(rows * chunks, 256), all = first + (b ? ceil_div(brows * chunks, 256) : 0);
  if (!grid_fits(all, 256)) return BCJR_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(pad_kernel<T>, dim3((unsigned)all), dim3(256), 0, stream, Pad{a, lda, to, rows, cols, chunks},
                     Pad{b, ldb, bto, brows, cols, chunks}, (unsigned)first);
  return launched();
}

struct LinearPlan {
  size_t part, x, W, total;
};

// the partial sums, then x and W padded
LinearPlan linear_plan(int dtype, int64_t M, int64_t N, int64_t K) {
  LinearPlan p = {};
  const GemmPlan g = gemm_plan(dtype, M, N, K);
  p.part = g.part;
  if (pads(g, dtype, M, N, K, K)) {
    p.x = align_up((size_t)(M * whole(dtype, K)) * elem_size(dtype));
    p.W = align_up((size_t)(N * whole(dtype, K)) * elem_size(dtype));
  }
  p.total = p.part + p.x + p.W;
  return p;
}

int run_linear(GemmArgs g, int dtype, char* ws, hipStream_t stream) {
  return by_type(dtype, [&](auto t) -> int {
    using T = decltype(t);
    const LinearPlan p = linear_plan(dtype, g.I, g.J, g.K);
    if (p.x) {
      char *x = ws + p.part, *W = x + p.x;
      const int st = pad<T>(g.a, g.lda, g.I, g.K, x, g.b, g.ldb, g.J, W, stream);
      if (st != BCJR_OK) return st;
      g.a = x;
      g.b = W;
      g.lda = g.ldb = whole(dtype, g.K);
    }
    return gemm<T, kRow, kRow>(g, ws, stream, p.x != 0, p.x != 0);
  });
}

FewArgs few_args(const void* x, int64_t ldx, const void* bias, const void* residual, int64_t ldr, void* y,
                 int64_t ldy, int act, int64_t M, int64_t N, int64_t K) {
  return {x, ldx, bias, residual, ldr, y, ldy, act, (int)M, (int)N, (int)K, 0, 0, 0};
}

template <class T, int Q>
int launch_few(FewArgs a, const void* W, int64_t ldw, hipStream_t stream) {
  const int groups = lay_out(a, Q, (a.K + 256 * Q - 1) / (256 * Q));
  hipLaunchKernelGGL((few_kernel<T, Q>), dim3((unsigned)groups), dim3((unsigned)(64 * a.parts * a.at_once)), 0,
                     stream, a, static_cast<const T*>(W), ldw);
  return launched();
}

// Up to 16 tokens without a checkpoint.  (More are quicker in the products'
// tiles: 32 tokens through 8192 x 8192 take 42 to 46 us there, 64 us here.)
int run_few(const FewArgs& a, const void* W, int64_t ldw, int dtype, hipStream_t stream) {
  return by_type(dtype, [&](auto t) -> int {
    using T = decltype(t);
    if (a.M <= 8) return launch_few<T, 2>(a, W, ldw, stream);
    return launch_few<T, 1>(a, W, ldw, stream);
  });
}

// A layer this small has its backward pass in one launch (figures of both sides
// beside the kernel).
bool small_vjp(int64_t M, int64_t N, int64_t K) {
  return M >= 1 && M <= 1024 && N <= 1024 && M * N * K <= ((int64_t)1 << 22);
}

int waves_along(int64_t terms) {
  int parts = 1;
  while (parts < kFewWaves && parts * 32 < terms) parts *= 2;
  return parts;
}

template <class T>
int run_small_vjp(SmallVjp a, hipStream_t stream) {
  a.xparts = waves_along(a.N);
  a.wparts = waves_along(a.M);
  int waves = a.xparts > a.wparts ? a.xparts : a.wparts;
  waves = waves < 4 ? 4 : waves;
  const int64_t k = ceil_div(a.K, 16);
  a.xblocks = a.dx ? (int)ceil_div(ceil_div(a.M, 16) * k, waves / a.xparts) : 0;
  const int64_t wtiles = a.dW ? ceil_div(a.N, 16) * k : a.dbias ? ceil_div(a.N, 16) : 0;
  hipLaunchKernelGGL(vjp_small_kernel<T>, dim3((unsigned)(a.xblocks + ceil_div(wtiles, waves / a.wparts))),
                     dim3((unsigned)(64 * waves)), 0, stream, a);
  return launched();
}

struct VjpPlan {
  size_t dz, part, x, W, sums, total;
  int64_t ldz, ldx;
  GemmPlan dW;
};

// dz (or dy padded), the groups' sums of dbias, x for a large dW, W padded for
// dx, then the partial sums of the products.  Workgroups that turn x's codes into T for themselves do it N / 256
// times over: from tiles of 256 on x is read back once instead (4096 tokens,
// 2048 x 8192, bf16: 174 us against 121 + 21; with tiles of 128 that costs as
// much as it gives, 44.7 and 44.3 us for 2048 cubed, with smaller ones 5 us
// more).  Rows of dz and x are padded to 16 bytes, for whole copies.
VjpPlan vjp_plan(int dtype, int64_t M, int64_t N, int64_t K, int act) {
  VjpPlan p = {};
  if (small_vjp(M, N, K)) return p;
  const int es = elem_size(dtype);
  const GemmPlan dx = M ? gemm_plan(dtype, M, K, N) : GemmPlan{};
  p.ldz = whole(dtype, N);
  p.ldx = whole(dtype, K);
  p.dz = act == kActNone && !pads(dx, dtype, M, K, N, N) ? 0 : align_up((size_t)(M * p.ldz) * es);
  p.W = pads(dx, dtype, M, K, N, K) ? align_up((size_t)(N * p.ldx) * es) : 0;
  p.part = align_up((size_t)(2 * ceil_div(M, kRows) * N) * sizeof(float));
  p.dW = gemm_plan(dtype, N, K, M);
  p.x = p.dW.tile == 256 ? align_up((size_t)(M * p.ldx) * es) : 0;
  p.sums = dx.part > p.dW.part ? dx.part : p.dW.part;
  p.total = p.dz + p.part + p.x + p.W + p.sums;
  return p;
}

struct Code {
  int n, k, V;
  int64_t block, steps, words;
};

// false where the arguments name no trellis
bool code_of(int state_bits, int k, int V, int64_t block, Code* c) {
  if (k < 1 || state_bits < k || state_bits > 16 || V < 1 || V > 8 || block < 1 || block % V || block > (1 << 24))
    return false;
  c->n = state_bits;
  c->k = k;
  c->V = V;
  c->block = block;
  c->steps = block / V;
  c->words = ceil_div(state_bits + (c->steps - 1) * k, 32);
  return true;
}

int run_dense(const uint32_t* packed, const float* codebook, const float* scales, const Code& c, int64_t B, void* W,
              int dtype, hipStream_t stream) {
  if (dense_large_takes(c.k, c.V, c.block, B))
    return dense_large(packed, B, codebook, c.n, c.k, c.V, c.block, c.words, scales, W, dtype, stream);
  return by_type(dtype, [&](auto t) -> int {
    using T = decltype(t);
    hipLaunchKernelGGL(dense_kernel<T>, dim3((unsigned)ceil_div(B * c.steps, 256)), dim3(256), 0, stream, packed,
                       codebook, scales, B, c.steps, c.n, c.k, c.V, c.words, static_cast<T*>(W));
    return launched();
  });
}

template <class T, int MT>
int launch_small(SmallCodes a, hipStream_t stream) {
  const int groups = lay_out(a, 16, (a.K + kSmallUnit - 1) / kSmallUnit);
  hipLaunchKernelGGL((codes_small_kernel<T, MT>), dim3((unsigned)groups), dim3((unsigned)(64 * a.parts * a.at_once)),
                     0, stream, a);
  return launched();
}

// Up to 16 tokens and so few weights that filling a table of the codebook for
// them, or a second launch, is what would count (of 16384 columns 16 tokens take
// 18.7 us in one launch, 11 in two; figures of others beside the kernel).
bool small_codes(const Code& c, int64_t M, int64_t N, int64_t K) {
  if (M > 16 || K > 8192 || N * K > ((int64_t)1 << 20)) return false;
  // a table of 2^n states against 16 and more weights a state; of a small one
  // the fp32 product costs up to 4 tokens nothing (512 x 1024, 8 state bits: 4.2
  // to 4.5 us against 4.0 to 4.1), 16 tokens 3 us
  const int64_t table = (int64_t)c.V << (c.n + 4), few = (int64_t)1 << (M <= 4 ? 18 : 16);
  return !codes_take(c.k, c.V, c.block, M, N, K) || N * K <= (table > few ? table : few);
}

bool threads_fit(int64_t n) { return grid_fits(ceil_div(n, 256), 256); }

}  // namespace
}  // namespace qlin
}  // namespace bcjr

using namespace bcjr::qlin;

extern "C" {

int qat_act8_store(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes,
                   uint16_t* scales, hipStream_t stream) {
  if (!dtype_ok(dtype) || rows < 0 || cols < 1 || ldx < cols) return BCJR_ERR_INVALID_ARG;
  if (rows >= kMaxRows || cols >= kMaxCols || !bands_fit(dtype, rows, cols)) return BCJR_ERR_UNSUPPORTED;
  if (rows == 0) return BCJR_OK;
  if (!x || !codes || !scales || misaligned(x, elem_size(dtype)) || misaligned(codes, 16) || misaligned(scales, 2))
    return BCJR_ERR_INVALID_ARG;
  return by_type(dtype, [&](auto t) -> int {
    using T = decltype(t);
    hipLaunchKernelGGL(act8_store_kernel<T>, band_grid<T>(rows, cols), dim3(kGroupThreads), 0, stream,
                       static_cast<const T*>(x), rows, cols, ldx, codes, scales);
    return launched();
  });
}

int qat_act8_load(const int8_t* codes, const uint16_t* scales, int64_t rows, int64_t cols, void* out, int dtype,
                  int64_t ldo, hipStream_t stream) {
  if (!dtype_ok(dtype) || rows < 0 || cols < 1 || ldo < cols) return BCJR_ERR_INVALID_ARG;
  if (rows >= kMaxRows || cols >= kMaxCols || !bands_fit(dtype, rows, cols)) return BCJR_ERR_UNSUPPORTED;
  if (rows == 0) return BCJR_OK;
  if (!out || !codes || !scales || misaligned(out, elem_size(dtype)) || misaligned(codes, 16) ||
      misaligned(scales, 2))
    return BCJR_ERR_INVALID_ARG;
  return by_type(dtype, [&](auto t) -> int {
    using T = decltype(t);
    hipLaunchKernelGGL(act8_load_kernel<T>, band_grid<T>(rows, cols), dim3(kGroupThreads), 0, stream, codes, scales, rows,
                       cols, static_cast<T*>(out), ldo);
    return launched();
  });
}

size_t qat_linear_act_workspace_bytes(int dtype, int64_t M, int64_t N, int64_t K) {
  if (!dtype_ok(dtype) || !dims_ok(M, N, K) || !dims_fit(M, N, K) || M == 0) return 0;
  return linear_plan(dtype, M, N, K).total;
}

int qat_linear_act(const void* x, int64_t ldx, const void* W, int64_t ldw, const void* bias, const void* residual,
                   int64_t ldr, int dtype, int activation, int64_t M, int64_t N, int64_t K, void* y, int64_t ldy,
                   int8_t* z_codes, uint16_t* z_scales, void* workspace, size_t ws_bytes, hipStream_t stream) {
  if (!dtype_ok(dtype) || !act_ok(activation) || !dims_ok(M, N, K) || ldx < K || ldw < K || ldy < N ||
      (residual && ldr < N) || (!z_codes != !z_scales))
    return BCJR_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype);
  if (!dims_fit(M, N, K) || !strides_fit(ldx, ldw, es)) return BCJR_ERR_UNSUPPORTED;
  if (M == 0) return BCJR_OK;
  if (!x || !W || !y || misaligned(x, es) || misaligned(W, es) || misaligned(y, es) || misaligned(bias, es) ||
      misaligned(residual, es) || misaligned(z_codes, 16) || misaligned(z_scales, 2))
    return BCJR_ERR_INVALID_ARG;
  if (M <= QAT_FEW_TOKENS && !z_codes)   // (before the plan of a product that is not launched)
    return run_few(few_args(x, ldx, bias, residual, ldr, y, ldy, activation, M, N, K), W, ldw, dtype, stream);
  const size_t need = qat_linear_act_workspace_bytes(dtype, M, N, K);
  if (need && (!workspace || misaligned(workspace, 16) || ws_bytes < need)) return BCJR_ERR_WORKSPACE;
  const GemmArgs g = {x, W, ldx, ldw, nullptr, M, N, K, bias, residual, ldr, y, ldy, z_codes, z_scales, activation};
  return run_linear(g, dtype, static_cast<char*>(workspace), stream);
}

size_t qat_linear_act_vjp_workspace_bytes(int dtype, int64_t M, int64_t N, int64_t K, int activation) {
  if (!dtype_ok(dtype) || !act_ok(activation) || !dims_ok(M, N, K) || !dims_fit(M, N, K)) return 0;
  return vjp_plan(dtype, M, N, K, activation).total;
}

int qat_linear_act_vjp(const void* dy, int64_t ldd, const int8_t* x_codes, const uint16_t* x_scales, const void* W,
                       int64_t ldw, const int8_t* z_codes, const uint16_t* z_scales, int dtype, int activation,
                       int64_t M, int64_t N, int64_t K, void* dx, void* dW, void* dbias, void* workspace,
                       size_t ws_bytes, hipStream_t stream) {
  if (!dtype_ok(dtype) || !act_ok(activation) || !dims_ok(M, N, K) || ldd < N || (dx && ldw < K))
    return BCJR_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype);
  if (!dims_fit(M, N, K) || !bands_fit(dtype, 2 * M, N) || !strides_fit(ldd, dx ? ldw : 1, es)) return BCJR_ERR_UNSUPPORTED;
  if (!dx && !dW && !dbias) return BCJR_OK;
  if (misaligned(dy, es) || misaligned(W, es) || misaligned(dx, es) || misaligned(dW, es) || misaligned(dbias, es) ||
      misaligned(x_codes, 16) || misaligned(z_codes, 16) || misaligned(x_scales, 2) || misaligned(z_scales, 2))
    return BCJR_ERR_INVALID_ARG;
  if (M > 0 && (!dy || (dx && !W) || (dW && (!x_codes || !x_scales)) ||
                (activation != kActNone && (!z_codes || !z_scales))))
    return BCJR_ERR_INVALID_ARG;
  if (small_vjp(M, N, K)) {
    const SmallVjp a = {dy, ldd, x_codes, x_scales, W, ldw, z_codes, z_scales, activation, (int)M, (int)N, (int)K,
                        dx, dW, dbias, 0, 0, 0};
    return by_type(dtype, [&](auto t) -> int { return run_small_vjp<decltype(t)>(a, stream); });
  }
  const VjpPlan p = vjp_plan(dtype, M, N, K, activation);
  if (p.total && (!workspace || misaligned(workspace, 16) || ws_bytes < p.total)) return BCJR_ERR_WORKSPACE;
  return by_type(dtype, [&](auto t) -> int {
    using T = decltype(t);
    char* ws = static_cast<char*>(workspace);
    void* sums = ws + p.dz + p.part + p.x + p.W;
    const T* dz = static_cast<const T*>(dy);
    int64_t ldz = ldd;
    float* part = reinterpret_cast<float*>(ws + p.dz);
    if (M > 0 && (activation != kActNone || dbias)) {
      const auto kernel = activation == kActNone   ? dz_kernel<T, kActNone>
                          : activation == kActSilu ? dz_kernel<T, kActSilu>
                          : activation == kActGelu ? dz_kernel<T, kActGelu>
                                                   : dz_kernel<T, kActGeluTanh>;
      const dim3 grid(2 * band_grid<T>(M, N).x);   // halves of groups
      hipLaunchKernelGGL(kernel, grid, dim3(kGroupThreads), 0, stream, static_cast<const T*>(dy), ldd,
                         z_codes, z_scales, M, N, reinterpret_cast<T*>(ws), p.ldz, dbias ? part : nullptr);
      if (launched() != BCJR_OK) return BCJR_ERR_HIP;
      if (activation != kActNone) {
        dz = reinterpret_cast<const T*>(ws);
        ldz = p.ldz;
      }
    }
    if (p.dz && activation == kActNone && M > 0 && (dx || dW)) {
      const int st = pad<T>(dy, ldd, M, N, ws, nullptr, 0, 0, nullptr, stream);
      if (st != BCJR_OK) return st;
      dz = reinterpret_cast<const T*>(ws);
      ldz = p.ldz;
    }
    if (dbias) {
      hipLaunchKernelGGL(dbias_kernel<T>, dim3((unsigned)ceil_div(N, 64)), dim3(1024), 0, stream, (const float*)part,
                         ceil_div(M, kRows), N, static_cast<T*>(dbias));
      if (launched() != BCJR_OK) return BCJR_ERR_HIP;
    }
    if (dx && M > 0) {
      GemmArgs g = {dz, W, ldz, ldw, nullptr, M, K, N, nullptr, nullptr, 0, dx, K, nullptr, nullptr, kActNone};
      if (p.W) {
        void* to = ws + p.dz + p.part + p.x;
        const int st = pad<T>(W, ldw, N, K, to, nullptr, 0, 0, nullptr, stream);
        if (st != BCJR_OK) return st;
        g.b = to;
        g.ldb = p.ldx;
      }
      const int st = gemm<T, kRow, kCol>(g, sums, stream, p.dz != 0, p.W != 0);
      if (st != BCJR_OK) return st;
    }
    if (dW) {
      GemmArgs g = {dz, x_codes, ldz, 0, x_scales, N, K, M, nullptr, nullptr, 0, dW, K, nullptr, nullptr, kActNone};
      const bool padded = p.dz != 0;
      if (!p.x || !bands_fit(dtype, M, K) || !copies(kCol, dz, ldz, N, M, (int)es, 256, padded))
        return gemm<T, kCol, kCodes>(g, sums, stream, padded);
      T* x = reinterpret_cast<T*>(ws + p.dz + p.part);
      hipLaunchKernelGGL(act8_load_kernel<T>, band_grid<T>(M, K), dim3(kGroupThreads), 0, stream, x_codes, x_scales, M,
                         K, x, p.ldx);
      if (launched() != BCJR_OK) return BCJR_ERR_HIP;
      g.b = x;
      g.ldb = p.ldx;
      return gemm_large<T, kCol, kCol>(g, p.dW, sums, stream);
    }
    return BCJR_OK;
  });
}

int64_t trellis_words(int state_bits, int k, int V, int64_t block) {
  Code c;
  return code_of(state_bits, k, V, block, &c) ? c.words : 0;
}

int trellis_pack(const int32_t* states, int64_t B, int64_t steps, int state_bits, int k, uint32_t* packed,
                 int32_t* illegal, hipStream_t stream) {
  Code c;
  if (B < 0 || !code_of(state_bits, k, 1, steps, &c)) return BCJR_ERR_INVALID_ARG;
  if (!threads_fit(B * c.words) || !threads_fit(B * steps)) return BCJR_ERR_UNSUPPORTED;
  if ((B && (!states || !packed)) || misaligned(states, 4) || misaligned(packed, 4) || misaligned(illegal, 4))
    return BCJR_ERR_INVALID_ARG;
  if (illegal) {
    hipLaunchKernelGGL(zero_kernel, dim3(1), dim3(1), 0, stream, illegal);
    if (launched() != BCJR_OK) return BCJR_ERR_HIP;
  }
  if (B == 0) return BCJR_OK;
  if (illegal) {
    hipLaunchKernelGGL(pack_check_kernel, dim3((unsigned)ceil_div(B * steps, 256)), dim3(256), 0, stream, states, B,
                       steps, c.n, c.k, illegal);
    if (launched() != BCJR_OK) return BCJR_ERR_HIP;
  }
  hipLaunchKernelGGL(pack_kernel, dim3((unsigned)ceil_div(B * c.words, 256)), dim3(256), 0, stream, states, B, steps,
                     c.n, c.k, c.words, packed);
  return launched();
}

int trellis_unpack(const uint32_t* packed, int64_t B, int64_t steps, int state_bits, int k, int32_t* states,
                   hipStream_t stream) {
  Code c;
  if (B < 0 || !code_of(state_bits, k, 1, steps, &c)) return BCJR_ERR_INVALID_ARG;
  if (!threads_fit(B * steps)) return BCJR_ERR_UNSUPPORTED;
  if ((B && (!states || !packed)) || misaligned(states, 4) || misaligned(packed, 4)) return BCJR_ERR_INVALID_ARG;
  if (B == 0) return BCJR_OK;
  hipLaunchKernelGGL(unpack_kernel, dim3((unsigned)ceil_div(B * steps, 256)), dim3(256), 0, stream, packed, B, steps,
                     c.n, c.k, c.words, states);
  return launched();
}

int trellis_dense(const uint32_t* packed, int64_t B, const float* codebook, int state_bits, int k, int V,
                  int64_t block, const float* scales, void* W, int dtype, hipStream_t stream) {
  Code c;
  if (!dtype_ok(dtype) || B < 0 || !code_of(state_bits, k, V, block, &c)) return BCJR_ERR_INVALID_ARG;
  if (!threads_fit(B * c.steps)) return BCJR_ERR_UNSUPPORTED;
  if (!codebook || (B && (!W || !packed)) || misaligned(packed, 4) || misaligned(codebook, 16) ||
      misaligned(scales, 4) || misaligned(W, elem_size(dtype)))
    return BCJR_ERR_INVALID_ARG;
  if (B == 0) return BCJR_OK;
  return run_dense(packed, codebook, scales, c, B, W, dtype, stream);
}

size_t trellis_linear_workspace_bytes(int dtype, int64_t M, int64_t N, int64_t K, int state_bits, int k, int V,
                                      int64_t block) {
  Code c;
  if (!dtype_ok(dtype) || !dims_ok(M, N, K) || !dims_fit(M, N, K) || !code_of(state_bits, k, V, block, &c) ||
      K % block)
    return 0;
  if (M == 0 || small_codes(c, M, N, K) || codes_take(c.k, c.V, c.block, M, N, K)) return 0;
  return align_up((size_t)(N * K) * elem_size(dtype)) + gemm_plan(dtype, M, N, K).part;
}

int trellis_linear(const void* x, int64_t ldx, const uint32_t* packed, const float* codebook, int state_bits, int k,
                   int V, int64_t block, const float* scales, const void* bias, const void* residual, int64_t ldr,
                   int dtype, int activation, int64_t M, int64_t N, int64_t K, void* y, int64_t ldy,
                   void* workspace, size_t ws_bytes, hipStream_t stream) {
  Code c;
  if (!dtype_ok(dtype) || !act_ok(activation) || !dims_ok(M, N, K) || !code_of(state_bits, k, V, block, &c) ||
      K % block || ldx < K || ldy < N || (residual && ldr < N))
    return BCJR_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype);
  if (!dims_fit(M, N, K) || !threads_fit(N * K) || !strides_fit(ldx, 1, es)) return BCJR_ERR_UNSUPPORTED;
  if (M == 0) return BCJR_OK;
  if (!x || !packed || !codebook || !y || misaligned(x, es) || misaligned(packed, 4) || misaligned(codebook, 16) ||
      misaligned(scales, 4) || misaligned(bias, es) || misaligned(residual, es) || misaligned(y, es))
    return BCJR_ERR_INVALID_ARG;
  const size_t need = trellis_linear_workspace_bytes(dtype, M, N, K, state_bits, k, V, block);
  if (need && (!workspace || misaligned(workspace, 16) || ws_bytes < need)) return BCJR_ERR_WORKSPACE;
  if (small_codes(c, M, N, K)) {
    SmallCodes a = {};
    static_cast<FewArgs&>(a) = few_args(x, ldx, bias, residual, ldr, y, ldy, activation, M, N, K);
    a.packed = packed;
    a.codebook = codebook;
    a.scales = scales;
    a.n = c.n;
    a.k = c.k;
    a.V = c.V;
    a.block = (int)c.block;
    a.words = (int)c.words;
    return by_type(dtype, [&](auto t) -> int {
      using T = decltype(t);
      return M == 1 ? launch_small<T, 1>(a, stream) : M <= 4 ? launch_small<T, 4>(a, stream) : launch_small<T, 16>(a, stream);
    });
  }
  if (codes_take(c.k, c.V, c.block, M, N, K)) {
    CodesArgs a = {};
    static_cast<FewArgs&>(a) = few_args(x, ldx, bias, residual, ldr, y, ldy, activation, M, N, K);
    a.packed = packed;
    a.codebook = codebook;
    a.scales = scales;
    a.n = c.n;
    a.block = (int)c.block;
    a.words = (int)c.words;
    return codes_linear(a, dtype, c.k, c.V, stream);
  }
  return by_type(dtype, [&](auto t) -> int {
    using T = decltype(t);
    T* W = static_cast<T*>(workspace);
    const int st = run_dense(packed, codebook, scales, c, N * (K / block), W, dtype, stream);
    if (st != BCJR_OK) return st;
    const GemmArgs g = {x, W, ldx, K, nullptr, M, N, K, bias, residual, ldr, y, ldy, nullptr, nullptr, activation};
    return gemm<T, kRow, kRow>(g, reinterpret_cast<char*>(W) + align_up((size_t)(N * K) * es), stream);
  });
}

}  // extern "C"
