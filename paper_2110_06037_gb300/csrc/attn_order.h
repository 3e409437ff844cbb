// What the end of a piece of prompt attention waits for (attn_prompt.cuh).  Host code too: no CUDA here.
#pragma once

#ifdef __CUDACC__
#define SN_HOST_DEVICE __host__ __device__
#else
#define SN_HOST_DEVICE
#endif

namespace sn {
namespace k {

// A wait by parity tells a phase from the one before it only, so it holds when that one is known to be over.  The last
// scores of n tiles are asked for behind the product with values `ahead` tiles earlier: when they have come, products
// 0 to n - 1 - ahead are over, and the next ones may not be.  The end so waits for each product from this one on.
SN_HOST_DEVICE constexpr int first_open_product(int n, int ahead) { return n > ahead ? n - ahead : 0; }

}  // namespace k
}  // namespace sn
