// Multi-query attention over bf16 pools with many query rows a page.
#include "mq_attn.hpp"

namespace ga {

hipError_t launch_mq_attn(const AttnArgs& a, int head_dim, int grid, hipStream_t stream,
                          hipEvent_t t0, hipEvent_t t1) {
  if (head_dim == 64) return launch_mq<64, false>(a, grid, stream, t0, t1);
  if (head_dim == 128) return launch_mq<128, false>(a, grid, stream, t0, t1);
  return hipErrorInvalidValue;
}

}  // namespace ga
