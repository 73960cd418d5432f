// Host side of the range attention (kernel in range_attn.cuh), and the kernel
// that joins the partial records of a long decode attention and adds its
// weights to the slots' sums.
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "range_attn.h"

namespace wm {

cudaError_t launch_range_bf16(const RangeParams& p, int d, int units, cudaStream_t s);
cudaError_t launch_range_f32(const RangeParams& p, int d, int units, cudaStream_t s);

int range_stage_slots(int dtype, int d) {
  if (dtype == WM_DT_F32) return d == 64 ? 16 : 8;
  return d == 64 ? 32 : 16;
}

cudaError_t launch_range_attn(const RangeParams& p, int dtype, int d, int units, cudaStream_t s) {
  return dtype == WM_DT_F32 ? launch_range_f32(p, d, units, s) : launch_range_bf16(p, d, units, s);
}

namespace {

// mass[t] += sum_g 2^(s_g[t] - m_g) / l_g over the G query heads of a unit
// (sequence, kv head), after the unit's partial records are joined:
//   out_e = sum_i 2^(m_i - M) O_i,e / sum_i 2^(m_i - M) l_i.
// Every slot is added to by one thread, so the sums do not depend on the order
// of anything.  blockIdx.y 0 writes the output rows, the others add a part of
// the slots each: bound by HBM / L2 (G + 2 floats per slot), four slots per
// 16-byte access.
constexpr int kMassThreads = 256;
constexpr int kMassSlots = kMassThreads * 16;  // per CTA
template <typename T, int HD, int G>
__global__ void __launch_bounds__(kMassThreads, G <= 2 ? 8 : 4) mass_add_kernel(const MassParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ float m_s[kRangeRows], inv_s[kRangeRows], w_s[kRangeRows][kMassMaxPieces];
  const int unit = blockIdx.x, b = unit / p.Hkv, h = unit - b * p.Hkv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int recf = range_rec(G, HD);
  const float* part = p.part + (int64_t)unit * p.pieces * recf;
  const int S_in = __ldg(p.seq_lens + b);
  const int S = S_in >= 0 && S_in <= p.max_slots ? S_in : 0;
  const int t0 = ((int)blockIdx.y - 1) * kMassSlots;
  if (t0 >= S) return;
  if (warp < G) {  // 8 warps: one per query head
    const float* ml = part + G * HD + 2 * warp;
    float M = -INFINITY, L = 0.f;
    for (int i = lane; i < p.pieces; i += 32) M = fmaxf(M, __ldcg(ml + (int64_t)i * recf));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
    for (int i = lane; i < p.pieces; i += 32) {
      const float m = __ldcg(ml + (int64_t)i * recf);
      const float w = m == -INFINITY ? 0.f : exp2f(m - M);
      w_s[warp][i] = w;
      if (w != 0.f) L = fmaf(w, __ldcg(ml + (int64_t)i * recf + 1), L);
    }
    L = warp_sum(L);
    if (lane == 0) {
      m_s[warp] = M;
      inv_s[warp] = L > 0.f ? 1.f / L : 0.f;
    }
  }
  __syncthreads();
  if (blockIdx.y == 0) {
    T* out = reinterpret_cast<T*>(p.out) + ((int64_t)b * p.Hq + h * G) * HD;
    for (int q = tid; q < G * HD / 4; q += kMassThreads) {  // four outputs, NB records in flight
      const int r = q / (HD / 4);
      constexpr int NB = G <= 2 ? 4 : 10;
      float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i0 = 0; i0 < p.pieces; i0 += NB) {
        float4 v[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i)
          if (i0 + i < p.pieces) v[i] = __ldcg(reinterpret_cast<const float4*>(part + (int64_t)(i0 + i) * recf) + q);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          if (i0 + i >= p.pieces) continue;
          const float w = w_s[r][i0 + i];
          O.x = fmaf(w, v[i].x, O.x);
          O.y = fmaf(w, v[i].y, O.y);
          O.z = fmaf(w, v[i].z, O.z);
          O.w = fmaf(w, v[i].w, O.w);
        }
      }
      const float inv = inv_s[r];
      out[4 * q] = Elem<T>::from_f(O.x * inv);
      out[4 * q + 1] = Elem<T>::from_f(O.y * inv);
      out[4 * q + 2] = Elem<T>::from_f(O.z * inv);
      out[4 * q + 3] = Elem<T>::from_f(O.w * inv);
    }
    return;
  }
  const float* sc = p.scores + (int64_t)unit * G * p.score_stride;
  float* mass = p.mass + (int64_t)unit * p.max_slots;
  auto weight = [&](float s, int g, float w) { return s == -INFINITY ? w : fmaf(exp2f(s - m_s[g]), inv_s[g], w); };
  const int64_t step = (int64_t)(gridDim.y - 1) * kMassSlots;
  for (int64_t base = t0; base < S; base += step) {
    const int t1 = (int)min((int64_t)S, base + kMassSlots);
    if (p.vec4) {
      for (int t = (int)base + tid * 4; t < t1; t += kMassThreads * 4) {
        float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
        float4* at = reinterpret_cast<float4*>(mass + t);
        float4 a = *at, s[G];
#pragma unroll
        for (int g = 0; g < G; ++g)  // (scores past S are not weights: not added below)
          s[g] = __ldcg(reinterpret_cast<const float4*>(sc + (int64_t)g * p.score_stride + t));
#pragma unroll
        for (int g = 0; g < G; ++g) {
          w.x = weight(s[g].x, g, w.x);
          w.y = weight(s[g].y, g, w.y);
          w.z = weight(s[g].z, g, w.z);
          w.w = weight(s[g].w, g, w.w);
        }
        a.x += w.x;
        if (t + 1 < S) a.y += w.y;
        if (t + 2 < S) a.z += w.z;
        if (t + 3 < S) a.w += w.w;
        *at = a;
      }
    } else {
      for (int t = (int)base + tid; t < t1; t += kMassThreads) {
        float w = 0.f;
        for (int g = 0; g < G; ++g) w = weight(__ldcg(sc + (int64_t)g * p.score_stride + t), g, w);
        mass[t] += w;
      }
    }
  }
}

template <typename Kern, typename P>
cudaError_t launch_chained(Kern kern, const P& p, dim3 grid, int threads, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

template <typename T, int HD>
cudaError_t launch_mass_g(const MassParams& p, dim3 grid, cudaStream_t s) {
  switch (p.G) {
    case 1: return launch_chained(mass_add_kernel<T, HD, 1>, p, grid, kMassThreads, s);
    case 2: return launch_chained(mass_add_kernel<T, HD, 2>, p, grid, kMassThreads, s);
    case 4: return launch_chained(mass_add_kernel<T, HD, 4>, p, grid, kMassThreads, s);
    case 8: return launch_chained(mass_add_kernel<T, HD, 8>, p, grid, kMassThreads, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace

cudaError_t launch_mass_add(MassParams p, int dtype, int d, cudaStream_t s) {
  // rows of mass on 16-byte boundaries
  p.vec4 = p.max_slots % 4 == 0 && ((uintptr_t)p.mass & 15) == 0 ? 1 : 0;
  const int parts = (p.max_slots + kMassSlots - 1) / kMassSlots;
  const dim3 grid((unsigned)(p.B * p.Hkv), (unsigned)(1 + (parts < 65534 ? parts : 65534)));
  if (dtype == WM_DT_F32) {
    if (d == 64) return launch_mass_g<float, 64>(p, grid, s);
    if (d == 96) return launch_mass_g<float, 96>(p, grid, s);
    return launch_mass_g<float, 128>(p, grid, s);
  }
  if (d == 64) return launch_mass_g<__nv_bfloat16, 64>(p, grid, s);
  if (d == 96) return launch_mass_g<__nv_bfloat16, 96>(p, grid, s);
  return launch_mass_g<__nv_bfloat16, 128>(p, grid, s);
}

}  // namespace wm
