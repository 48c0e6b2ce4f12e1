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
  const int groups = lay_out(a, Q, (a.K / kChunk + Q - 1) / Q);
  // a large table is filled by 16 waves, of which those past parts * at_once do
  // nothing else (14 state bits, 4096 x 256 weights: 5.5 us, with 4 waves 7.4)
  const int waves = (V << a.n) > 64 * 32 * a.parts * a.at_once ? kFewWaves : a.parts * a.at_once;
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

template <class T, int KB, int V>
int launch_dense(const uint32_t* packed, int64_t B, const float* codebook, int n, int64_t block, int64_t words,
                 const float* scales, T* W, hipStream_t stream) {
  const int64_t groups = B * (block / 8), each = (int64_t)kDenseThreads * kDenseGroups;
  const int64_t grid = (groups + each - 1) / each;
  const void* kernel = reinterpret_cast<const void*>(&dense_large_kernel<T, KB, V>);
  const size_t lds = codes_table<float, V>(n);
  if (lds > 65536 &&
      hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
    return BCJR_ERR_HIP;
  hipLaunchKernelGGL((dense_large_kernel<T, KB, V>), dim3((unsigned)(grid < 256 ? grid : 256)), dim3(kDenseThreads), lds,
                     stream, packed, codebook, scales, groups, n, (int)(block / 8), (int)words, W);
  return hipGetLastError() == hipSuccess ? BCJR_OK : BCJR_ERR_HIP;
}

template <class T>
int dense_by_code(const uint32_t* packed, int64_t B, const float* codebook, int n, int k, int V, int64_t block,
                  int64_t words, const float* scales, T* W, hipStream_t stream) {
  if (V == 2) return launch_dense<T, 4, 2>(packed, B, codebook, n, block, words, scales, W, stream);
  if (k == 1) return launch_dense<T, 1, 1>(packed, B, codebook, n, block, words, scales, W, stream);
  if (k == 2) return launch_dense<T, 2, 1>(packed, B, codebook, n, block, words, scales, W, stream);
  if (k == 3) return launch_dense<T, 3, 1>(packed, B, codebook, n, block, words, scales, W, stream);
  return launch_dense<T, 4, 1>(packed, B, codebook, n, block, words, scales, W, stream);
}

}  // namespace

// Whether dense_large_kernel takes a decode: codes of whole groups of eight
// weights, and enough of them that filling the table pays.
bool dense_large_takes(int k, int V, int64_t block, int64_t B) {
  return ((V == 1 && k <= 4) || (V == 2 && k == 4)) && block % 8 == 0 && B * block >= ((int64_t)1 << 20) &&
         B * (block / 8) < ((int64_t)1 << 31);
}

int dense_large(const uint32_t* packed, int64_t B, const float* codebook, int n, int k, int V, int64_t block,
                int64_t words, const float* scales, void* W, int dtype, hipStream_t stream) {
  if (dtype == kBF16)
    return dense_by_code(packed, B, codebook, n, k, V, block, words, scales, static_cast<bf16*>(W), stream);
  if (dtype == kF16)
    return dense_by_code(packed, B, codebook, n, k, V, block, words, scales, static_cast<f16*>(W), stream);
  return dense_by_code(packed, B, codebook, n, k, V, block, words, scales, static_cast<float*>(W), stream);
}

// Whether the kernels take a product: the trellises with 1 to 4 bits a step
// (two weights a step with 4) and blocks of whole 256 weights (below them
// scales would change inside a matrix instruction).  Past 16 tokens a lane's
// products outlast its decoding, and weights decoded once into a dense matrix
// do better unless they are so few that a second launch is what counts
// (bf16, 16 state bits, 2 bits a step, us, this against decoding first:
// 2048 x 2048 with 32 tokens 16.9 and 24.9, 2048 x 8192 with 64 57.8 and 39.8).
bool codes_take(int k, int V, int64_t block, int64_t M, int64_t N, int64_t K) {
  return ((V == 1 && k <= 4) || (V == 2 && k == 4)) && block % kChunk == 0 &&
         (M <= 16 || (M <= 64 && N * K <= ((int64_t)1 << 22))) && N < ((int64_t)1 << 24) &&
         K < ((int64_t)1 << 24);
}

int codes_linear(const CodesArgs& a, int dtype, int k, int V, hipStream_t stream) {
  if (dtype == kBF16) return by_code<bf16>(a, k, V, stream);
  if (dtype == kF16) return by_code<f16>(a, k, V, stream);
  return by_code<float>(a, k, V, stream);
}

}  // namespace qlin
}  // namespace bcjr
