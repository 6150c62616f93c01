// The kernels of paged_attention.h for a cache in bf16.
#include "paged_attention.h"

namespace talon {

hipError_t launch_paged_attention_bf16(const PagedAttnArgs& a, int Dh, int waves, hipStream_t s) {
  return launch_paged<false>(a, Dh, waves, s);
}

}  // namespace talon
