// qat_codes.hip -- launches of qat_codes_kernels.h, in their own translation
// unit.
#include <hip/hip_runtime.h>

#include "bcjr.h"
#include "qat_codes_kernels.h"

namespace bcjr {
namespace qlin {
namespace {

template <class T, int KB, int V, int MT, int Q>
int launch(CodesArgs a, hipStream_t stream) {
  constexpr int kRowsOf = 16 / Q;
  const int units = (a.K / kChunk + Q - 1) / Q;
  a.tiles = (a.N + kRowsOf - 1) / kRowsOf;
  a.parts = 1;
  while (a.parts < kCodesWaves && a.parts < units) a.parts *= 2;
  // as many tiles at once as leave a workgroup for each CU
  a.rows_at_once = kCodesWaves / a.parts;
  while (a.rows_at_once > 1 && (a.tiles + a.rows_at_once - 1) / a.rows_at_once < 256) a.rows_at_once /= 2;
  const int groups = (a.tiles + a.rows_at_once - 1) / a.rows_at_once;
  const int waves = a.parts * a.rows_at_once;
  const size_t lds = codes_table<T, V>(a.n) + (size_t)waves * 256 * sizeof(float);
  const void* kernel = reinterpret_cast<const void*>(&codes_kernel<T, KB, V, MT, Q>);
  if (lds > 65536 &&
      hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
    return BCJR_ERR_HIP;
  void* args[] = {&a};
  if (hipLaunchKernel(kernel, dim3((unsigned)(groups < 256 ? groups : 256)), dim3((unsigned)(64 * waves)), args, lds,
                      stream) != hipSuccess)
    return BCJR_ERR_HIP;
  return hipGetLastError() == hipSuccess ? BCJR_OK : BCJR_ERR_HIP;
}

template <class T, int KB, int V>
int by_tokens(const CodesArgs& a, hipStream_t stream) {
  if (a.M <= 8) return launch<T, KB, V, 1, 2>(a, stream);
  if (a.M <= 16) return launch<T, KB, V, 1, 1>(a, stream);
  return launch<T, KB, V, 4, 1>(a, stream);
}

template <class T>
int by_code(const CodesArgs& a, int k, int V, hipStream_t stream) {
  if (V == 2) return by_tokens<T, 4, 2>(a, stream);
  if (k == 1) return by_tokens<T, 1, 1>(a, stream);
  if (k == 2) return by_tokens<T, 2, 1>(a, stream);
  if (k == 3) return by_tokens<T, 3, 1>(a, stream);
  return by_tokens<T, 4, 1>(a, stream);
}

}  // namespace

// Whether the kernels take a product: the trellises with 1 to 4 bits a step
// (two weights a step with 4) and blocks of whole 256 weights (below them
// scales would change inside a matrix instruction).  Past 64 tokens the weights
// are better decoded once.
bool codes_take(int k, int V, int64_t block, int64_t M, int64_t N, int64_t K) {
  return ((V == 1 && k <= 4) || (V == 2 && k == 4)) && block % kChunk == 0 && M <= 64 && N < ((int64_t)1 << 24) &&
         K < ((int64_t)1 << 24);
}

int codes_linear(const CodesArgs& a, int dtype, int k, int V, hipStream_t stream) {
  if (dtype == kBF16) return by_code<bf16>(a, k, V, stream);
  if (dtype == kF16) return by_code<f16>(a, k, V, stream);
  return by_code<float>(a, k, V, stream);
}

}  // namespace qlin
}  // namespace bcjr
