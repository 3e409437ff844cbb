// 4-bit weights with few rows of fp16 x: the instantiations of q4_few.cuh.
#include "q4_few.cuh"

namespace sn {
namespace k {

cudaError_t q4_few_f16(const Q4P &q, int rows, const __half *x, int64_t ldx, __half *y, int64_t ldy, cudaStream_t st) {
    return q4_few<__half, __half>(q, rows, x, ldx, y, ldy, st);
}

}  // namespace k
}  // namespace sn
