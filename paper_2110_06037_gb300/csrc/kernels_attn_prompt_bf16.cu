// Many queries over a cache of bf16.
#include "attn_prompt.cuh"

namespace sn {
namespace k {

cudaError_t attend_prompt_bf16(const AttnP &p, int64_t grid, cudaStream_t st) { return prompt::launch_any<__nv_bfloat16>(p, SN_BF16, grid, st); }

}  // namespace k
}  // namespace sn
