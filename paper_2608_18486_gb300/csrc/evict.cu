// Eviction: cuts every (channel, sequence, kv head) of the cache to `budget`
// slots.  The sinks (the first slots), the most recent slots and, of the rest,
// those with the largest sums of attention weight stay; rows keep their order.
//
//  select: one CTA per unit.  The sums of the middle slots, mapped to unsigned
//    keys of the same order, are cut by an 8-bit radix select (four histogram
//    passes) to the threshold key and the number of slots taken among its
//    equals (lowest slots first); one ordered pass then lists the kept slots
//    and compacts the sums.
//  move: one CTA per unit copies row kept[j] to slot j, in waves: every row of
//    a wave is read before any is written.  kept[j] >= j and rises with j, so
//    a wave's rows are written only over slots that no later wave reads.
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "range_attn.h"

namespace wm {
namespace {

constexpr int kSelThreads = 512;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kMoveThreads = 256;
constexpr int kMoveVecs = 4;  // 16-byte vectors of K (and of V) per thread and wave

// Unsigned key in the order of the sums: NaN below everything, -0 equal to +0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Slots a sequence has (0 and a report for a bad length).
__device__ __forceinline__ int checked_len(const EvictParams& p, int b, bool tell) {
  const int n = __ldg(p.seq_lens + b);
  if (n >= 0 && n <= p.max_pages * p.P) return n;
  if (tell) report(p.status, WM_ERR_BOUNDS);
  return 0;
}

__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const EvictParams p) {
  __shared__ int hist[256];
  __shared__ int wsum[2][kSelWarps];
  __shared__ uint32_t prefix_s;
  __shared__ int need_s;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int unit = blockIdx.x, b = (unit / p.Hkv) % p.B;  // (c B + b) Hkv + h
  const bool first = unit == b * p.Hkv;                   // channel 0, head 0
  const int64_t slots = (int64_t)p.max_pages * p.P;
  const float* mass = p.mass + unit * slots;
  float* mass_out = p.mass_out + unit * slots;
  int32_t* kept = p.kept + (int64_t)unit * p.budget;
  const int n = checked_len(p, b, first && tid == 0);
  const int out_n = min(n, p.budget);
  if (first && tid == 0) p.new_lens[b] = out_n;

  // the middle slots [lo, hi), of which `want` stay
  const bool cut = n > p.budget;
  const int lo = cut ? p.sinks : 0, hi = cut ? n - p.recent : 0;
  const int want = cut ? p.budget - p.sinks - p.recent : 0;
  uint32_t prefix = 0;
  int need = want;  // still to take among the keys that match the prefix
  if (cut && want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += kSelThreads) {
        const uint32_t k = order_key(mass[t]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (warp == 0) {
        // bins from the top: lane l sums bins 255 - 8 l .. 248 - 8 l
        int sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += hist[255 - 8 * lane - i];
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
          if (lane >= o) incl += v;
        }
        int above = incl - sum;
        if (above < need && need <= incl) {  // the threshold's bin is one of this lane's
          int bin = 255 - 8 * lane;
          while (above + hist[bin] < need) above += hist[bin--];
          prefix_s = prefix | ((uint32_t)bin << shift);
          need_s = need - above;
        }
      }
      __syncthreads();
      prefix = prefix_s;
      need = need_s;
    }
  }
  // ---- ordered list of the kept slots
  int taken = 0, eq_seen = 0;  // over the slots before this pass's
  for (int t0 = 0; t0 < n; t0 += kSelThreads) {
    const int t = t0 + tid;
    const float x = t < n ? mass[t] : 0.f;
    bool keep = t < n && (!cut || t < lo || t >= hi), eq = false;
    if (t < n && cut && t >= lo && t < hi && want > 0) {
      const uint32_t k = order_key(x);
      keep = k > prefix;
      eq = k == prefix;
    }
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t eqs = __ballot_sync(0xFFFFFFFFu, eq);
    if (lane == 0) wsum[0][warp] = __popc(eqs);
    __syncthreads();  // also: every sum of this pass is read before any is written
    int eq_before = eq_seen, eq_total = 0;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) {
      eq_before += w < warp ? wsum[0][w] : 0;
      eq_total += wsum[0][w];
    }
    if (eq) keep = eq_before + __popc(eqs & below) < need;
    const uint32_t keeps = __ballot_sync(0xFFFFFFFFu, keep);
    if (lane == 0) wsum[1][warp] = __popc(keeps);
    __syncthreads();
    int at = taken, total = 0;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) {
      at += w < warp ? wsum[1][w] : 0;
      total += wsum[1][w];
    }
    at += __popc(keeps & below);
    if (keep) {
      kept[at] = t;
      mass_out[at] = x;
    }
    taken += total;
    eq_seen += eq_total;
    __syncthreads();
  }
  for (int j = out_n + tid; j < p.budget; j += kSelThreads) kept[j] = -1;
  for (int64_t t = out_n + tid; t < slots; t += kSelThreads) mass_out[t] = 0.f;
}

template <int ROWV>  // 16-byte vectors per row
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int unit = blockIdx.x, cb = unit / p.Hkv, h = unit - cb * p.Hkv, c = cb / p.B, b = cb - c * p.B;
  const int n = checked_len(p, b, false);
  if (n <= p.budget) return;  // nothing moves
  const int32_t* ptab = p.page_table + (int64_t)b * p.max_pages;
  const int32_t* kept = p.kept + (int64_t)unit * p.budget;
  uint4* kb = reinterpret_cast<uint4*>(p.k_pool);
  uint4* vb = reinterpret_cast<uint4*>(p.v_pool);
  auto vec_of = [&](int t, int v) -> int64_t {  // -1: no such page
    const int pg = __ldg(ptab + (t >> p.log2P));
    if (pg < 0 || pg >= p.num_pages) return -1;
    return ((((int64_t)c * p.num_pages + pg) * p.Hkv + h) * p.P + (t & (p.P - 1))) * ROWV + v;
  };
  const int64_t total = (int64_t)p.budget * ROWV;
  for (int64_t x0 = 0; x0 < total; x0 += kMoveThreads * kMoveVecs) {
    uint4 kv[kMoveVecs], vv[kMoveVecs];
    int64_t dst[kMoveVecs];
#pragma unroll
    for (int i = 0; i < kMoveVecs; ++i) {
      const int64_t x = x0 + i * kMoveThreads + threadIdx.x;
      dst[i] = -1;
      if (x >= total) continue;
      const int j = (int)(x / ROWV), v = (int)(x - (int64_t)j * ROWV);
      const int t = __ldcg(kept + j);
      if (t == j) continue;
      const int64_t src = vec_of(t, v);
      dst[i] = vec_of(j, v);
      if (src < 0 || dst[i] < 0) {
        report(p.status, WM_ERR_BOUNDS);
        dst[i] = -1;
        continue;
      }
      kv[i] = __ldcg(kb + src);
      vv[i] = __ldcg(vb + src);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMoveVecs; ++i)
      if (dst[i] >= 0) {
        kb[dst[i]] = kv[i];
        vb[dst[i]] = vv[i];
      }
  }
}

template <typename Kern>
cudaError_t launch_units(Kern kern, const EvictParams& p, int threads, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.k * (unsigned)p.B * (unsigned)p.Hkv);
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

cudaError_t launch_cache_evict(const EvictParams& p, int dtype, int d, cudaStream_t s) {
  if (cudaError_t e = launch_units(evict_select_kernel, p, kSelThreads, s); e != cudaSuccess) return e;
  switch (d * (dtype == WM_DT_F32 ? 4 : 2) / 16) {
    case 8: return launch_units(evict_move_kernel<8>, p, kMoveThreads, s);
    case 12: return launch_units(evict_move_kernel<12>, p, kMoveThreads, s);
    case 16: return launch_units(evict_move_kernel<16>, p, kMoveThreads, s);
    case 24: return launch_units(evict_move_kernel<24>, p, kMoveThreads, s);
    case 32: return launch_units(evict_move_kernel<32>, p, kMoveThreads, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace wm
