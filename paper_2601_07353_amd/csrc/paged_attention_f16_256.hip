// The attention kernels over a paged cache in f16 with heads of 256.
#include "paged_few.h"

namespace talon {

hipError_t launch_paged_attention_f16_256(const PagedAttnArgs& a, int waves, hipStream_t s) {
  return waves == 0 ? launch_few<true, 256>(a, s) : launch_paged<true, 256>(a, waves, s);
}

}  // namespace talon
