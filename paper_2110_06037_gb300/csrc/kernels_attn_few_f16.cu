// Few queries over a long cache: fp16.
#include "attn_few.cuh"

namespace sn {
namespace k {

few::Shape few_shape_f16(int d, int64_t rows) { return few::shape_any<__half, __half>(d, rows); }
cudaError_t attend_few_f16(const AttnP &p, int64_t grid, cudaStream_t st) { return few::launch_any<__half, __half>(p, grid, st); }

}  // namespace k
}  // namespace sn
