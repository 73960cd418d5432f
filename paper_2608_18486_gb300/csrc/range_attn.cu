// Host side of the range attention (kernel in range_attn.cuh) and the kernels
// that join its partial records: of a shared prefix with each sequence's
// suffix, and of decode attention with the weights added to the slots' sums.
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

// Joins n partial records of one row: out_e = sum_i 2^(m_i - M) O_i,e / sum_i 2^(m_i - M) l_i.
// rec(i): the i-th record's row of HD outputs; ml(i): its (max, sum).  One warp per row.
template <typename T, int HD, typename Rec, typename Ml>
__device__ __forceinline__ void join_row(T* out, int n, int lane, Rec rec, Ml ml) {
  float M = -INFINITY;
  for (int i = lane; i < n; i += 32) M = fmaxf(M, ml(i).x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
  float L = 0.f, O[HD / 32] = {};
  for (int i = 0; i < n; ++i) {
    const float2 x = ml(i);
    if (x.x == -INFINITY) continue;
    const float w = exp2f(x.x - M);
    L = fmaf(w, x.y, L);
    const float* r = rec(i);
#pragma unroll
    for (int e = 0; e < HD / 32; ++e) O[e] = fmaf(w, __ldcg(r + lane + 32 * e), O[e]);
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
#pragma unroll
  for (int e = 0; e < HD / 32; ++e) out[lane + 32 * e] = Elem<T>::from_f(O[e] * inv);
}

constexpr int kJoinWarps = 4;

// One warp per output row (sequence b, query head hq).
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinWarps * 32) prefix_join_kernel(const PrefixJoinParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int row = (int)blockIdx.x * kJoinWarps + (int)(threadIdx.x >> 5);
  if (row >= p.B * p.Hq) return;
  const int b = row / p.Hq, hq = row - b * p.Hq, h = hq / p.G, g = hq - h * p.G;
  // the row's records: of the prefix, then of its suffix
  const int np = p.prefix_pieces, srec = range_rec(p.G, HD);
  const int x = b * p.G + g, grp = x / kRangeRows, xr = x - grp * kRangeRows;
  const int prec = p.tiles ? tile_rec(HD) : range_rec(kRangeRows, HD);
  const float* pre = p.prefix + (p.tiles ? ((int64_t)h * p.B * p.G + x) * np * prec
                                         : ((int64_t)grp * p.Hkv + h) * np * prec + xr * HD);
  const int pml = p.tiles ? HD : kRangeRows * HD + 2 * xr - xr * HD;  // (max, sum) of a record, from its outputs
  const float* suf = p.suffix + ((int64_t)b * p.Hkv + h) * p.suffix_pieces * srec;
  auto rec = [&](int i) -> const float* {
    return i < np ? pre + (int64_t)i * prec : suf + (int64_t)(i - np) * srec + g * HD;
  };
  auto ml = [&](int i) -> float2 {
    const float* r = i < np ? pre + (int64_t)i * prec + pml : suf + (int64_t)(i - np) * srec + p.G * HD + 2 * g;
    return make_float2(__ldcg(r), __ldcg(r + 1));
  };
  join_row<T, HD>(reinterpret_cast<T*>(p.out) + (int64_t)row * HD, np + p.suffix_pieces, lane, rec, ml);
}

// mass[t] += sum_g 2^(s_g[t] - m_g) / l_g over the G query heads of a unit
// (sequence, kv head).  Every slot is added to by one thread, so the sums do
// not depend on the order of anything.  blockIdx.y: part of the slots; part 0
// also joins the output rows.
constexpr int kMassThreads = 256;
template <typename T, int HD>
__global__ void __launch_bounds__(kMassThreads) mass_add_kernel(const MassParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ float lse_s[kRangeRows], inv_s[kRangeRows];
  const int unit = blockIdx.x, b = unit / p.Hkv, h = unit - b * p.Hkv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int recf = range_rec(p.G, HD);
  const float* part = p.part + (int64_t)unit * p.pieces * recf;
  if (warp < p.G) {
    float M = -INFINITY, L = 0.f;
    for (int i = 0; i < p.pieces; ++i) M = fmaxf(M, __ldcg(part + (int64_t)i * recf + p.G * HD + 2 * warp));
    for (int i = 0; i < p.pieces; ++i) {
      const float* r = part + (int64_t)i * recf + p.G * HD + 2 * warp;
      const float m = __ldcg(r);
      if (m != -INFINITY) L = fmaf(exp2f(m - M), __ldcg(r + 1), L);
    }
    if (lane == 0) {
      lse_s[warp] = M;
      inv_s[warp] = L > 0.f ? 1.f / L : 0.f;
    }
    if (blockIdx.y == 0) {
      auto rec = [&](int i) -> const float* { return part + (int64_t)i * recf + warp * HD; };
      auto ml = [&](int i) -> float2 {
        const float* r = part + (int64_t)i * recf + p.G * HD + 2 * warp;
        return make_float2(__ldcg(r), __ldcg(r + 1));
      };
      join_row<T, HD>(reinterpret_cast<T*>(p.out) + ((int64_t)b * p.Hq + h * p.G + warp) * HD, p.pieces, lane, rec, ml);
    }
  }
  __syncthreads();
  const int S_in = __ldg(p.seq_lens + b);
  const int S = S_in >= 0 && S_in <= p.max_slots ? S_in : 0;
  const float* sc = p.scores + (int64_t)unit * p.G * p.score_stride;
  float* mass = p.mass + (int64_t)unit * p.max_slots;
  for (int t = (int)blockIdx.y * kMassThreads + tid; t < S; t += (int)gridDim.y * kMassThreads) {
    float w = 0.f;
    for (int g = 0; g < p.G; ++g) {
      const float s = __ldcg(sc + (int64_t)g * p.score_stride + t);
      if (s != -INFINITY) w = fmaf(exp2f(s - lse_s[g]), inv_s[g], w);
    }
    mass[t] += w;
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

}  // namespace

cudaError_t launch_prefix_join(const PrefixJoinParams& p, int dtype, int d, cudaStream_t s) {
  const dim3 grid((unsigned)(((int64_t)p.B * p.Hq + kJoinWarps - 1) / kJoinWarps));
  const int n = kJoinWarps * 32;
  if (dtype == WM_DT_F32) {
    if (d == 64) return launch_chained(prefix_join_kernel<float, 64>, p, grid, n, s);
    if (d == 96) return launch_chained(prefix_join_kernel<float, 96>, p, grid, n, s);
    return launch_chained(prefix_join_kernel<float, 128>, p, grid, n, s);
  }
  if (d == 64) return launch_chained(prefix_join_kernel<__nv_bfloat16, 64>, p, grid, n, s);
  if (d == 96) return launch_chained(prefix_join_kernel<__nv_bfloat16, 96>, p, grid, n, s);
  return launch_chained(prefix_join_kernel<__nv_bfloat16, 128>, p, grid, n, s);
}

cudaError_t launch_mass_add(const MassParams& p, int dtype, int d, cudaStream_t s) {
  // four slots per thread and pass at most
  int ny = (p.max_slots + 4 * kMassThreads - 1) / (4 * kMassThreads);
  if (ny > 65535) ny = 65535;
  const dim3 grid((unsigned)(p.B * p.Hkv), (unsigned)ny);
  const int n = kMassThreads;
  if (dtype == WM_DT_F32) {
    if (d == 64) return launch_chained(mass_add_kernel<float, 64>, p, grid, n, s);
    if (d == 96) return launch_chained(mass_add_kernel<float, 96>, p, grid, n, s);
    return launch_chained(mass_add_kernel<float, 128>, p, grid, n, s);
  }
  if (d == 64) return launch_chained(mass_add_kernel<__nv_bfloat16, 64>, p, grid, n, s);
  if (d == 96) return launch_chained(mass_add_kernel<__nv_bfloat16, 96>, p, grid, n, s);
  return launch_chained(mass_add_kernel<__nv_bfloat16, 128>, p, grid, n, s);
}

}  // namespace wm
