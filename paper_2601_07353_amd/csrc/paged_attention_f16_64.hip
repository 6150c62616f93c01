// The attention kernels over a paged cache in f16 with heads of 64.
#include "paged_few.h"

namespace talon {

hipError_t launch_paged_attention_f16_64(const PagedAttnArgs& a, int waves, hipStream_t s) {
  return waves == 0 ? launch_few<true, 64>(a, s) : launch_paged<true, 64>(a, waves, s);
}

}  // namespace talon
