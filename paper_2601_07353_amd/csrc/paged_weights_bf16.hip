// The kernels of paged_weights.h for a cache in bf16.
#include "paged_weights.h"

namespace talon {

hipError_t launch_paged_weights_bf16(const PagedWeightArgs& wa, int Dh, bool few, hipStream_t s) { return launch_weights<false>(wa, Dh, few, s); }

}  // namespace talon
