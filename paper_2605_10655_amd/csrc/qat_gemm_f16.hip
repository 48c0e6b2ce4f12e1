// qat_gemm_f16.hip -- the products of qat_gemm_launch.h in f16: forward (row,
// row), gradient of x (row, col), gradient of W (col, codes; large ones
// col, col).
#include <hip/hip_runtime.h>

#include "qat_gemm_launch.h"

namespace bcjr {
namespace qlin {

template int gemm<f16, kRow, kRow>(GemmArgs, void*, hipStream_t, bool, bool);
template int gemm<f16, kRow, kCol>(GemmArgs, void*, hipStream_t, bool, bool);
template int gemm<f16, kCol, kCodes>(GemmArgs, void*, hipStream_t, bool, bool);
template int gemm_large<f16, kCol, kCol>(GemmArgs, const GemmPlan&, void*, hipStream_t);

}  // namespace qlin
}  // namespace bcjr
