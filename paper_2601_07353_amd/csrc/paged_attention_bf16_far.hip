// Attention over a paged cache in bf16, caps above kNearCap.
#include "paged_few.h"

namespace talon {

namespace {

template <int DH>
hipError_t launch_far(const PagedAttnArgs& a, int waves, hipStream_t s) {
  return waves == 0 ? launch_few<false, DH, true>(a, s) : launch_paged<false, DH, true>(a, waves, s);
}

}  // namespace

hipError_t launch_paged_attention_bf16_far(const PagedAttnArgs& a, int Dh, int waves, hipStream_t s) {
  switch (Dh) {
    case 64: return launch_far<64>(a, waves, s);
    case 128: return launch_far<128>(a, waves, s);
    default: return launch_far<256>(a, waves, s);
  }
}

}  // namespace talon
