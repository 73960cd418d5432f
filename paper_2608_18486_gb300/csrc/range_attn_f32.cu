// Instantiations of the range attention kernel for f32 caches.
#include "range_attn.cuh"

namespace wm {

cudaError_t launch_range_f32(const RangeParams& p, int d, int units, cudaStream_t s) {
  using namespace range_detail;
  if (d == 64) return launch_d<float, 64>(p, units, s);
  if (d == 96) return launch_d<float, 96>(p, units, s);
  if (d == 128) return launch_d<float, 128>(p, units, s);
  return cudaErrorInvalidValue;
}

}  // namespace wm
