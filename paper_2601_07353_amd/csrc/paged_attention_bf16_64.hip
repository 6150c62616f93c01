// The attention kernels over a paged cache in bf16 with heads of 64.
#include "paged_few.h"

namespace talon {

hipError_t launch_paged_attention_bf16_64(const PagedAttnArgs& a, int waves, hipStream_t s) {
  return waves == 0 ? launch_few<false, 64>(a, s) : launch_paged<false, 64>(a, waves, s);
}

}  // namespace talon
