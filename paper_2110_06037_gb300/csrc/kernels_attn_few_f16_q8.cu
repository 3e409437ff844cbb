// Few queries over a long cache: fp16 queries, codes.
#include "attn_few.cuh"

namespace sn {
namespace k {

few::Shape few_shape_f16_q8(int d, int64_t rows) { return few::shape_any<__half, int8_t>(d, rows); }
cudaError_t attend_few_f16_q8(const AttnP &p, int64_t grid, cudaStream_t st) { return few::launch_any<__half, int8_t>(p, grid, st); }

}  // namespace k
}  // namespace sn
