// Instantiations of the range attention kernel for bf16 caches.
#include "range_attn.cuh"

namespace wm {

cudaError_t launch_range_bf16(const RangeParams& p, int d, int units, cudaStream_t s) {
  using namespace range_detail;
  if (d == 64) return launch_d<__nv_bfloat16, 64>(p, units, s);
  if (d == 96) return launch_d<__nv_bfloat16, 96>(p, units, s);
  if (d == 128) return launch_d<__nv_bfloat16, 128>(p, units, s);
  return cudaErrorInvalidValue;
}

}  // namespace wm
