// f32 instances of the 4-bit cache's attention (q4_attn.cuh).
#include "q4_attn.cuh"

namespace wm {

cudaError_t launch_q4_attn_f32(const Q4AttnParams& p, int d, cudaStream_t s) {
  if (d == 64) return q4_detail::launch_d<float, 64>(p, s);
  if (d == 96) return q4_detail::launch_d<float, 96>(p, s);
  return q4_detail::launch_d<float, 128>(p, s);
}

}  // namespace wm
