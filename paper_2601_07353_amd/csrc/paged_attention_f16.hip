// The kernels of paged_attention.h for a cache in f16.
#include "paged_attention.h"

namespace talon {

hipError_t launch_paged_attention_f16(const PagedAttnArgs& a, int Dh, int waves, hipStream_t s) {
  return launch_paged<true>(a, Dh, waves, s);
}

}  // namespace talon
