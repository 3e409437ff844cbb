// Many queries over a cache of fp16.
#include "attn_prompt.cuh"

namespace sn {
namespace k {

cudaError_t attend_prompt_f16(const AttnP &p, int64_t grid, cudaStream_t st) { return prompt::launch_any<__half>(p, SN_F16, grid, st); }

}  // namespace k
}  // namespace sn
