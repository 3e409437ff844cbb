// Few queries over a long cache, and queries in any number: fp32.
#include "attn_few.cuh"

namespace sn {
namespace k {

few::Shape few_shape_f32(int d, int64_t rows) { return few::shape_any<float, float>(d, rows); }
cudaError_t attend_few_f32(const AttnP &p, int64_t grid, cudaStream_t st) { return few::launch_any<float, float>(p, grid, st); }

}  // namespace k
}  // namespace sn
