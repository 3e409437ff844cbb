// Few queries over a long cache: bf16.
#include "attn_few.cuh"

namespace sn {
namespace k {

few::Shape few_shape_bf16(int d, int64_t rows) { return few::shape_any<__nv_bfloat16, __nv_bfloat16>(d, rows); }
cudaError_t attend_few_bf16(const AttnP &p, int64_t grid, cudaStream_t st) { return few::launch_any<__nv_bfloat16, __nv_bfloat16>(p, grid, st); }

}  // namespace k
}  // namespace sn
