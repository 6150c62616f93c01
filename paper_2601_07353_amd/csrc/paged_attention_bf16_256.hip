// The attention kernels over a paged cache in bf16 with heads of 256.
#include "paged_few.h"

namespace talon {

hipError_t launch_paged_attention_bf16_256(const PagedAttnArgs& a, int waves, hipStream_t s) {
  return waves == 0 ? launch_few<false, 256>(a, s) : launch_paged<false, 256>(a, waves, s);
}

}  // namespace talon
