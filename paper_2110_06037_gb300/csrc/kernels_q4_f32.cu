// 4-bit weights with few rows of fp32 x: the instantiations of q4_few.cuh.
#include "q4_few.cuh"

namespace sn {
namespace k {

cudaError_t q4_few_f32(const Q4P &q, int rows, const float *x, int64_t ldx, float *y, int64_t ldy, cudaStream_t st) {
    return q4_few<__nv_bfloat16, float>(q, rows, x, ldx, y, ldy, st);
}

}  // namespace k
}  // namespace sn
