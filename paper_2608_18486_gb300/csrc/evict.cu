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
//    holds 4 consecutive slots (up to 2048 in all) or 16; up to 8192 slots the
//    sums are read once.
//  move (all CTAs): row kept[j] goes to slot j, in waves: every row of a wave
//    is read before any is written.  kept[j] >= j and rises with j, so a wave
//    writes only over slots that no later wave reads, and later waves' rows may
//    be on their way meanwhile: a ring of cp.async copies keeps STAGES - 1
//    waves of 16 KB in flight, so that a wave does not wait for its slowest row.  A row
//    is found through two dependent loads (its slot, its page); each is issued a
//    wave ahead of its use.
// The move is bound by HBM: every kept row behind the first gap is read and
// written once, in runs of one row (128 to 512 bytes), which DRAM serves below
// its sequential rate (reads alone, rows of 256 bytes, every fourth kept: 3.2
// TB/s; of 192 bytes, every second: 4.7).  The select is bound by its chain of
// block-wide steps (about 8 us); units in different phases share an SM, so that
// one covers the other: more units than two per SM take three CTAs per SM with
// rings of 4 waves, fewer take two with rings of 6 (768 units of 2048 to 1024
// slots of 192 bytes: 115 against 127 us; 256 units of 32768 to 8192 slots of
// 256 bytes: 574 against 458).
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
constexpr int kEvBins = 2048;
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

__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

struct SelectShared {
  int hist[kEvBins];
  int red[kEvWarps];
  uint32_t prefix;
  int need, count;
};

// Lists the kept slots of a unit of n slots and compacts its sums; a thread holds
// HOLD consecutive ones.
template <int HOLD>
__device__ __forceinline__ void select_unit(const EvictParams& p, int n, const float* mass, float* mass_out, int32_t* kept,
                            SelectShared& sh) {
  constexpr int TILE = kEvThreads * HOLD;
  const int tid = threadIdx.x;
  const int64_t slots = (int64_t)p.max_pages * p.P;
  const bool cut = n > p.budget;
  const int lo = cut ? p.sinks : 0, hi = cut ? n - p.recent : 0;  // the middle slots
  const int want = cut ? p.budget - p.sinks - p.recent : 0;       // of which this many stay
  const bool once = n <= TILE;
  float x[HOLD];
  auto load = [&](int base) {
    const int t0 = base + tid * HOLD;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) x[i] = t0 + i < n ? mass[t0 + i] : 0.f;
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
      for (int base = 0; base < n; base += TILE) {
        if (!once) load(base);
        const int t0 = base + tid * HOLD;
#pragma unroll
        for (int i = 0; i < HOLD; ++i) {
          const int t = t0 + i;
          const uint32_t k = order_key(x[i]);
          if (t >= lo && t < hi && (shift == 32 || (k >> shift) == (prefix >> shift)))
            atomicAdd(&sh.hist[(k >> down) & (kEvBins - 1) & ((1u << bits) - 1u)], 1);
        }
      }
      __syncthreads();
      // a thread owns kOwn bins, from the top down
      constexpr int kOwn = kEvBins / kEvThreads;
      const int b0 = kEvBins - 1 - kOwn * tid;
      int own[kOwn], sum = 0, total;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        own[i] = sh.hist[b0 - i];
        sum += own[i];
      }
      int above = block_scan(sum, sh.red, total);
      if (above < need && need <= above + sum) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
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
  for (int base = 0; base < n; base += TILE) {
    if (!once) load(base);
    const int t0 = base + tid * HOLD;
    uint32_t keep = 0, eq = 0;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
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
    for (int i = 0; i < HOLD; ++i)
      if (((eq >> i) & 1u) && left-- > 0) keep |= 1u << i;
    int at = taken + block_scan(__popc(keep), sh.red, keep_total);  // (a block barrier after every sum was read)
#pragma unroll
    for (int i = 0; i < HOLD; ++i)
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

template <int ROWV, int STAGES, int CTAS>  // 16-byte vectors per row; waves in the ring; CTAs per SM
__global__ void __launch_bounds__(kEvThreads, CTAS) evict_kernel(const EvictParams p) {
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
    const float* mass = p.mass + unit * slots;
    float* mass_out = p.mass_out + unit * slots;
    if (n <= 4 * kEvThreads) select_unit<4>(p, n, mass, mass_out, kept, sh);
    else select_unit<16>(p, n, mass, mass_out, kept, sh);
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
  // A thread moves vector v of one K and one V row per wave; the threads past
  // the last whole row rest.
  constexpr int kRows = kEvThreads / ROWV;  // rows per wave of a CTA
  const int lr = tid / ROWV, v = tid - lr * ROWV;
  const int wave = C * kRows, waves = (p.budget + wave - 1) / wave;
  // (slot -1: no row; page -1: no such page)
  auto slot_of = [&](int w) -> int { return w * wave + rank * kRows + lr; };
  auto kept_of = [&](int w) -> int {
    const int j = slot_of(w);
    return w < waves && j < p.budget && lr < kRows ? __ldcg(kept + j) : -1;
  };
  auto page_of = [&](int t) -> int { return t >= 0 ? __ldg(ptab + (t >> p.log2P)) : -1; };
  auto row_of = [&](int t, int pg) -> int {  // cache row (32 bits: checked on the host)
    if (pg < 0 || pg >= p.num_pages) return -1;
    return ((c * p.num_pages + pg) * p.Hkv + h) * p.P + (t & (p.P - 1));
  };
  int n_wave = 0;                                      // the next wave to load
  int t = kept_of(0), t_next = kept_of(1);             // its kept slot, and that of the wave after
  int pg_s = page_of(t), pg_d = page_of(t >= 0 ? slot_of(0) : -1);  // pages of the row, and of its new place
  extern __shared__ uint4 ring[];  // [STAGES][2][kEvThreads]: each thread reads back its own copies
  int to[STAGES];  // rows the ring's waves go to (-1: nothing moves)
  auto load = [&](int s) {
    const int j = slot_of(n_wave);
    to[s] = -1;
    if (t >= 0 && t != j) {
      const int src = row_of(t, pg_s), dst = row_of(j, pg_d);
      if (src < 0 || dst < 0) {
        report(p.status, WM_ERR_BOUNDS);
      } else {
        to[s] = dst;
        const int64_t at = (int64_t)src * ROWV + v;
        cp_async16(ring + (2 * s) * kEvThreads + tid, kb + at);
        cp_async16(ring + (2 * s + 1) * kEvThreads + tid, vb + at);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ++n_wave;
    t = t_next;
    pg_s = page_of(t);
    pg_d = page_of(t >= 0 ? slot_of(n_wave) : -1);
    t_next = kept_of(n_wave + 1);
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) load(s);
  for (int w0 = 0; w0 < waves; w0 += STAGES) {
#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
      const int w = w0 + s;
      if (w >= waves) break;
      load((s + STAGES - 1) % STAGES);  // wave w + STAGES - 1
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
      barrier();  // every row of wave w has been read
      if (to[s] >= 0) {
        const int64_t at = (int64_t)to[s] * ROWV + v;
        kb[at] = ring[(2 * s) * kEvThreads + tid];
        vb[at] = ring[(2 * s + 1) * kEvThreads + tid];
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <int ROWV, int STAGES, int CTAS>
cudaError_t launch_t(const EvictParams& p, cudaStream_t s) {
  static size_t smem_set[kSmemOptDevices] = {};
  auto kern = evict_kernel<ROWV, STAGES, CTAS>;
  constexpr size_t smem = (size_t)STAGES * 2 * kEvThreads * sizeof(uint4);
  if (cudaError_t e = opt_in_smem(kern, smem, smem_set); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.dynamicSmemBytes = smem;
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
  return cudaLaunchKernelEx(&cfg, kern, p);
}

template <int ROWV>
cudaError_t launch_rowv(const EvictParams& p, bool many, cudaStream_t s) {
  return many ? launch_t<ROWV, 4, 3>(p, s) : launch_t<ROWV, 6, 2>(p, s);
}

}  // namespace

cudaError_t launch_cache_evict(EvictParams p, int dtype, int d, int sms, cudaStream_t s) {
  const int rowv = d * (dtype == WM_DT_F32 ? 4 : 2) / 16;
  // CTAs per unit: as many as are resident at once, and no more than there are
  // pairs of waves of a single CTA to share
  const int64_t units = (int64_t)p.k * p.B * p.Hkv, vecs = (int64_t)p.budget * rowv;
  p.cluster = 1;
  while (p.cluster < kEvMaxCluster && units * p.cluster * 2 <= 2 * (int64_t)sms &&
         (int64_t)p.cluster * kEvThreads * 2 < vecs)
    p.cluster *= 2;
  const bool many = units > 2 * (int64_t)sms;
  switch (rowv) {
    case 8: return launch_rowv<8>(p, many, s);
    case 12: return launch_rowv<12>(p, many, s);
    case 16: return launch_rowv<16>(p, many, s);
    case 24: return launch_rowv<24>(p, many, s);
    case 32: return launch_rowv<32>(p, many, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace wm
