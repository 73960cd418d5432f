// Eviction: cuts every (channel, sequence, kv head) unit of the cache to
// `budget` slots.  The sinks (the first slots), the most recent slots and, of
// the rest, those with the largest sums of attention weight stay; rows keep
// their order.
//
// One kernel, one cluster of C CTAs per unit (C = 1 where the units alone fill
// the SMs):
//  select (first CTA): the middle slots' sums, mapped to unsigned keys of the
//    same order, are cut by a radix select from the top (11, 11 and 10 bits,
//    ending as soon as the threshold's bin is taken whole) to the threshold
//    and the number of slots taken among its equals, lowest slots first.  An
//    ordered pass then lists the kept slots and compacts the sums.  A thread
//    holds 16 consecutive slots; up to 8192 slots the sums are read once.
//  move (all CTAs): row kept[j] goes to slot j, in waves: every row of a wave
//    is read before any is written.  kept[j] >= j and rises with j, so a wave
//    writes only over slots that no later wave reads.  While a wave's rows are
//    on their way the next wave's slots and pages are looked up.
// The move is bound by HBM (every kept row behind the first gap is read and
// written once), the select by its chain of block-wide steps; units in
// different phases share an SM, so that one covers the other.
#include <cooperative_groups.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "range_attn.h"

namespace wm {
namespace {

namespace cg = cooperative_groups;

constexpr int kEvThreads = 512;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvHold = 16;                         // sums per thread
constexpr int kEvTile = kEvThreads * kEvHold;       // sums per pass over the block
constexpr int kEvBins = 2048;
constexpr int kEvVecs = 4;                          // 16-byte vectors of K (and of V) per thread and wave
constexpr int kEvMaxCluster = 8;

// Unsigned key in the order of the sums: NaN below everything, -0 equal to +0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix sum over the block; total gets the sum.  red: [kEvWarps].
__device__ __forceinline__ int block_scan(int v, int* red, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += u;
  }
  __syncthreads();  // the last scan's sums have been read
  if (lane == 31) red[warp] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kEvWarps; ++w) {
    before += w < warp ? red[w] : 0;
    total += red[w];
  }
  return before + incl - v;
}

struct SelectShared {
  int hist[kEvBins];
  int red[kEvWarps];
  uint32_t prefix;
  int need, count;
};

// Lists the kept slots of a unit of n slots and compacts its sums.
__device__ void select_unit(const EvictParams& p, int n, const float* mass, float* mass_out, int32_t* kept,
                            SelectShared& sh) {
  const int tid = threadIdx.x;
  const int64_t slots = (int64_t)p.max_pages * p.P;
  const bool cut = n > p.budget;
  const int lo = cut ? p.sinks : 0, hi = cut ? n - p.recent : 0;  // the middle slots
  const int want = cut ? p.budget - p.sinks - p.recent : 0;       // of which this many stay
  const bool once = n <= kEvTile;
  float x[kEvHold];
  auto load = [&](int base) {
    const int t0 = base + tid * kEvHold;
#pragma unroll
    for (int i = 0; i < kEvHold; ++i) x[i] = t0 + i < n ? mass[t0 + i] : 0.f;
  };
  if (once) load(0);

  // ---- threshold: keys above it stay, and the first `need` of its equals, both
  // compared without their low `shift` bits
  uint32_t prefix = 0;
  int need = want, shift = 32;
  if (want > 0) {
    while (shift > 0) {
      const int bits = shift > 10 ? 11 : 10, down = shift - bits;
      for (int i = tid; i < kEvBins; i += kEvThreads) sh.hist[i] = 0;
      __syncthreads();
      for (int base = 0; base < n; base += kEvTile) {
        if (!once) load(base);
        const int t0 = base + tid * kEvHold;
#pragma unroll
        for (int i = 0; i < kEvHold; ++i) {
          const int t = t0 + i;
          const uint32_t k = order_key(x[i]);
          if (t >= lo && t < hi && (shift == 32 || (k >> shift) == (prefix >> shift)))
            atomicAdd(&sh.hist[(k >> down) & (kEvBins - 1) & ((1u << bits) - 1u)], 1);
        }
      }
      __syncthreads();
      // thread i owns 4 bins, from the top down
      const int b0 = kEvBins - 1 - 4 * tid;
      int own[4], sum = 0, total;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        own[i] = sh.hist[b0 - i];
        sum += own[i];
      }
      int above = block_scan(sum, sh.red, total);
      if (above < need && need <= above + sum) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < need && need <= above + own[i]) {
            sh.prefix = prefix | ((uint32_t)(b0 - i) << down);
            sh.need = need - above;
            sh.count = own[i];
          }
          above += own[i];
        }
      }
      __syncthreads();
      prefix = sh.prefix;
      need = sh.need;
      shift = down;
      if (sh.count == need) break;  // every key of the bin stays
    }
  }

  // ---- the kept slots in order
  int taken = 0, eq_seen = 0;  // over the slots before this tile's
  for (int base = 0; base < n; base += kEvTile) {
    if (!once) load(base);
    const int t0 = base + tid * kEvHold;
    uint32_t keep = 0, eq = 0;
#pragma unroll
    for (int i = 0; i < kEvHold; ++i) {
      const int t = t0 + i;
      if (t >= n) continue;
      if (!cut || t < lo || t >= hi) {
        keep |= 1u << i;
      } else if (want > 0) {
        const uint32_t a = shift == 32 ? 0u : order_key(x[i]) >> shift, z = shift == 32 ? 0u : prefix >> shift;
        if (a > z) keep |= 1u << i;
        if (a == z) eq |= 1u << i;
      }
    }
    int eq_total, keep_total;
    const int eq_before = eq_seen + block_scan(__popc(eq), sh.red, eq_total);
    int left = need - eq_before;  // of this thread's equals
#pragma unroll
    for (int i = 0; i < kEvHold; ++i)
      if (((eq >> i) & 1u) && left-- > 0) keep |= 1u << i;
    int at = taken + block_scan(__popc(keep), sh.red, keep_total);  // (a block barrier after every sum was read)
#pragma unroll
    for (int i = 0; i < kEvHold; ++i)
      if ((keep >> i) & 1u) {
        kept[at] = t0 + i;
        mass_out[at] = x[i];
        ++at;
      }
    taken += keep_total;
    eq_seen += eq_total;
  }
  __syncthreads();  // every sum has been read: mass_out may be mass
  const int out_n = min(n, p.budget);
  for (int j = out_n + tid; j < p.budget; j += kEvThreads) kept[j] = -1;
  for (int64_t t = out_n + tid; t < slots; t += kEvThreads) mass_out[t] = 0.f;
}

template <int ROWV>  // 16-byte vectors per row
__global__ void __launch_bounds__(kEvThreads, 2) evict_kernel(const EvictParams p) {
  __shared__ SelectShared sh;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int C = p.cluster, tid = threadIdx.x;
  const int unit = (int)(blockIdx.x / (unsigned)C), rank = (int)(blockIdx.x - (unsigned)unit * C);
  const int cb = unit / p.Hkv, h = unit - cb * p.Hkv, c = cb / p.B, b = cb - c * p.B;
  const int64_t slots = (int64_t)p.max_pages * p.P;
  int n = __ldg(p.seq_lens + b);
  if (n < 0 || n > slots) {
    if (c == 0 && h == 0 && rank == 0 && tid == 0) report(p.status, WM_ERR_BOUNDS);
    n = 0;
  }
  int32_t* kept = p.kept + (int64_t)unit * p.budget;
  if (rank == 0) {
    if (c == 0 && h == 0 && tid == 0) p.new_lens[b] = min(n, p.budget);
    select_unit(p, n, p.mass + unit * slots, p.mass_out + unit * slots, kept, sh);
  }
  if (n <= p.budget) return;  // nothing moves (the same for the whole cluster)
  auto barrier = [&]() {
    if (C == 1) __syncthreads();
    else cg::this_cluster().sync();
  };
  barrier();  // the list is there

  const int32_t* ptab = p.page_table + (int64_t)b * p.max_pages;
  uint4* kb = reinterpret_cast<uint4*>(p.k_pool);
  uint4* vb = reinterpret_cast<uint4*>(p.v_pool);
  const int64_t total = (int64_t)p.budget * ROWV;
  const int wave = C * kEvThreads * kEvVecs;
  auto vec_of = [&](int t, int v) -> int64_t {  // -1: no such page
    const int pg = __ldg(ptab + (t >> p.log2P));
    if (pg < 0 || pg >= p.num_pages) return -1;
    return ((((int64_t)c * p.num_pages + pg) * p.Hkv + h) * p.P + (t & (p.P - 1))) * ROWV + v;
  };
  int64_t src[kEvVecs], dst[kEvVecs];
  auto look_up = [&](int64_t x0) {
#pragma unroll
    for (int i = 0; i < kEvVecs; ++i) {
      const int64_t x = x0 + ((int64_t)i * C + rank) * kEvThreads + tid;
      src[i] = dst[i] = -1;
      if (x >= total) continue;
      const int j = (int)(x / ROWV), v = (int)(x - (int64_t)j * ROWV);
      const int t = __ldcg(kept + j);
      if (t == j) continue;
      src[i] = vec_of(t, v);
      dst[i] = vec_of(j, v);
      if (src[i] < 0 || dst[i] < 0) {
        report(p.status, WM_ERR_BOUNDS);
        dst[i] = -1;
      }
    }
  };
  look_up(0);
  for (int64_t x0 = 0; x0 < total; x0 += wave) {
    uint4 kv[kEvVecs], vv[kEvVecs];
    int64_t to[kEvVecs];
#pragma unroll
    for (int i = 0; i < kEvVecs; ++i) {
      to[i] = dst[i];
      if (to[i] < 0) continue;
      kv[i] = __ldcg(kb + src[i]);
      vv[i] = __ldcg(vb + src[i]);
    }
    if (x0 + wave < total) look_up(x0 + wave);
    barrier();
#pragma unroll
    for (int i = 0; i < kEvVecs; ++i)
      if (to[i] >= 0) {
        kb[to[i]] = kv[i];
        vb[to[i]] = vv[i];
      }
  }
}

template <int ROWV>
cudaError_t launch_rowv(const EvictParams& p, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.k * (unsigned)p.B * (unsigned)p.Hkv * (unsigned)p.cluster);
  cfg.blockDim = dim3(kEvThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, evict_kernel<ROWV>, p);
}

}  // namespace

cudaError_t launch_cache_evict(EvictParams p, int dtype, int d, int sms, cudaStream_t s) {
  const int rowv = d * (dtype == WM_DT_F32 ? 4 : 2) / 16;
  // CTAs per unit: as many as fit the SMs twice over, and no more than there
  // are waves of a single CTA to share
  const int64_t units = (int64_t)p.k * p.B * p.Hkv, vecs = (int64_t)p.budget * rowv;
  p.cluster = 1;
  while (p.cluster < kEvMaxCluster && units * p.cluster * 2 <= 2 * (int64_t)sms &&
         (int64_t)p.cluster * kEvThreads * kEvVecs < vecs)
    p.cluster *= 2;
  switch (rowv) {
    case 8: return launch_rowv<8>(p, s);
    case 12: return launch_rowv<12>(p, s);
    case 16: return launch_rowv<16>(p, s);
    case 24: return launch_rowv<24>(p, s);
    case 32: return launch_rowv<32>(p, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace wm
