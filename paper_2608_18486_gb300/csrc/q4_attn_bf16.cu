// bf16 instances of the 4-bit cache's attention (q4_attn.cuh).
#include "q4_attn.cuh"

namespace wm {

cudaError_t launch_q4_attn_bf16(const Q4AttnParams& p, int d, cudaStream_t s) {
  if (d == 64) return q4_detail::launch_d<__nv_bfloat16, 64>(p, s);
  if (d == 96) return q4_detail::launch_d<__nv_bfloat16, 96>(p, s);
  return q4_detail::launch_d<__nv_bfloat16, 128>(p, s);
}

}  // namespace wm
