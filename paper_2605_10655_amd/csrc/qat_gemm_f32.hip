// qat_gemm_f32.hip -- the products of qat_gemm_launch.h in float: forward (row,
// row), gradient of x (row, col), gradient of W (col, codes; large ones
// col, col).
#include <hip/hip_runtime.h>

#include "qat_gemm_launch.h"

namespace bcjr {
namespace qlin {

template int gemm<float, kRow, kRow>(GemmArgs, void*, hipStream_t, bool, bool);
template int gemm<float, kRow, kCol>(GemmArgs, void*, hipStream_t, bool, bool);
template int gemm<float, kCol, kCodes>(GemmArgs, void*, hipStream_t, bool, bool);
template int gemm_large<float, kCol, kCol>(GemmArgs, const GemmPlan&, void*, hipStream_t);

}  // namespace qlin
}  // namespace bcjr
