// The small kernels around many query rows over a 4-bit cache: what the tensor-core
// kernel (tile_attn.cu) needs to know of the rows that are read back for it, and the
// join of its partial records.
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "q4.h"
#include "range_attn.h"

namespace wm {
namespace {

// One CTA per sequence: the slots that its rows see, and where their pages will be.
__global__ void __launch_bounds__(256) q4_rows_prep_kernel(const Q4RowsPrep p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ int top_s[8];
  const int b = blockIdx.x, tid = threadIdx.x, slots = p.max_pages * p.P;
  int top = 0;
  for (int r = tid; r < p.Tq; r += 256) {
    const int x = __ldg(p.pos + (int64_t)b * p.Tq + r), n = x >= 0 && x < slots ? x + 1 : -1;
    p.lens[(int64_t)b * p.Tq + r] = n;
    top = max(top, n);
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if ((tid & 31) == 0) top_s[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, top_s[i]);
  if (tid == 0) p.last[b] = top;
  for (int y = tid; y < p.max_pages; y += 256) {
    const int64_t entry = (int64_t)b * p.max_pages + y;
    int page = -1;
    if ((int64_t)y * p.P < top) {
      const int pg = __ldg(p.q4_table + entry);
      if (pg >= 0 && pg < p.q4_pages) page = (int)entry;
    }
    p.table[entry] = page;
  }
}

// out = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i over a row's records; a warp per row.
// A record without a visible slot (m = -inf) holds no outputs; where all of a record's
// scores are NaN, its sum is.
template <int HD>
__global__ void __launch_bounds__(256) q4_rows_join_kernel(const Q4RowsJoin p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int REC = tile_rec(HD);
  const int rows = p.Tq * p.G, lane = threadIdx.x & 31;
  const int64_t y = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);  // (sequence, kv head, row)
  if (y >= (int64_t)p.B * p.Hkv * rows) return;
  const int x = (int)(y % rows), bh = (int)(y / rows), b = bh / p.Hkv, h = bh - b * p.Hkv;
  const float* part = p.part + y * p.records * REC;
  float M = -INFINITY;
  for (int i = 0; i < p.records; ++i) M = fmaxf(M, __ldcg(part + (int64_t)i * REC + HD));
  float L = 0.f;
  float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < p.records; ++i) {
    const float2 ml = __ldcg(reinterpret_cast<const float2*>(part + (int64_t)i * REC + HD));
    if (ml.x == -INFINITY) {
      if (ml.y != ml.y) L = ml.y;
      continue;
    }
    const float w = exp2f(ml.x - M);
    L = fmaf(w, ml.y, L);
    if (lane < HD / 4) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(part + (int64_t)i * REC) + lane);
      O.x = fmaf(w, v.x, O.x);
      O.y = fmaf(w, v.y, O.y);
      O.z = fmaf(w, v.z, O.z);
      O.w = fmaf(w, v.w, O.w);
    }
  }
  if (lane >= HD / 4) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const __nv_bfloat162 lo = __floats2bfloat162_rn(O.x * inv, O.y * inv), hi = __floats2bfloat162_rn(O.z * inv, O.w * inv);
  uint2 u;
  u.x = *reinterpret_cast<const uint32_t*>(&lo);
  u.y = *reinterpret_cast<const uint32_t*>(&hi);
  __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out) +
                       (((int64_t)b * p.Tq + x / p.G) * p.Hq + h * p.G + x % p.G) * HD;
  reinterpret_cast<uint2*>(out)[lane] = u;
}

template <typename Kern, typename P>
cudaError_t launch(Kern kern, const P& p, unsigned grid, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

}  // namespace

cudaError_t launch_q4_rows_prep(const Q4RowsPrep& p, int B, cudaStream_t s) {
  return launch(q4_rows_prep_kernel, p, (unsigned)B, s);
}

cudaError_t launch_q4_rows_join(const Q4RowsJoin& p, int d, cudaStream_t s) {
  const unsigned grid = (unsigned)(((int64_t)p.B * p.Hkv * p.Tq * p.G + 7) / 8);
  if (d == 64) return launch(q4_rows_join_kernel<64>, p, grid, s);
  if (d == 96) return launch(q4_rows_join_kernel<96>, p, grid, s);
  return launch(q4_rows_join_kernel<128>, p, grid, s);
}

}  // namespace wm
