// When the softmax of prompt attention waits for products (attn_prompt.cuh).  Host code too: no CUDA here.
#pragma once

#ifdef __CUDACC__
#define SN_HOST_DEVICE __host__ __device__
#else
#define SN_HOST_DEVICE
#endif

namespace sn {
namespace k {

// A wait by parity tells a phase from its neighbours only: it holds where the phase before is known to be over and the one
// after cannot be.  The scores of tile j are asked for behind the product with values `ahead` tiles earlier.  With one in
// between, two products are open when a piece of n tiles ends, and a wait for the last alone might take the one before the
// other for it; so the last weights are handed over behind the product before theirs.  (Later it might be too late: with
// both over, a wait for the first lasts for ever.)
SN_HOST_DEVICE constexpr bool waits_before_weights(int j, int n, int ahead) { return ahead > 1 && j > 0 && j == n - 1; }

}  // namespace k
}  // namespace sn
