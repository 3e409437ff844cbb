// 4-bit weights with few rows of bf16 x: the instantiations of q4_few.cuh.
#include "q4_few.cuh"

namespace sn {
namespace k {

cudaError_t q4_few_bf16(const Q4P &q, int rows, const __nv_bfloat16 *x, int64_t ldx, __nv_bfloat16 *y, int64_t ldy, cudaStream_t st) {
    return q4_few<__nv_bfloat16, __nv_bfloat16>(q, rows, x, ldx, y, ldy, st);
}

}  // namespace k
}  // namespace sn
