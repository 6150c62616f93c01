// The attention kernels over a paged cache in bf16 with heads of 128.
#include "paged_few.h"

namespace talon {

hipError_t launch_paged_attention_bf16_128(const PagedAttnArgs& a, int waves, hipStream_t s) {
  return waves == 0 ? launch_few<false, 128>(a, s) : launch_paged<false, 128>(a, waves, s);
}

}  // namespace talon
