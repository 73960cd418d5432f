// Eviction: cuts every (channel, sequence, kv head) unit of the cache to
// `budget` slots.  The sinks (the first slots), the most recent slots and, of
// the rest, those with the largest sums of attention weight stay; rows keep
// their order.
//
// One kernel, one cluster of C CTAs per unit (C = 1 where the units alone fill
// the SMs):
//  select: the middle slots' sums, mapped to unsigned keys of the same order, are
//    cut by a radix select from the top (at most 11 bits a pass, ending as soon as
//    the threshold's bin is taken whole) to the threshold and the number of slots
//    taken among its equals, lowest slots first.  An ordered pass then lists the
//    kept slots and compacts the sums.  Up to 2048 slots are the first CTA's, 4
//    per thread.  More are shared by the cluster's CTAs, up to 16 per thread, each
//    counting its own part of the slots; the counts are joined through distributed
//    shared memory, over bins of the range that the sums cover (over the bins of
//    all floats most sums meet in a few counters).  Still more than that are read
//    by the first CTA, pass by pass (a unit of 65536 slots of 256 bytes cut to half
//    99 us, of 131072 310).
//  move (all CTAs): row kept[j] goes to slot j, in waves: every row of a group of
//    GROUP waves is read before any is written.  kept[j] >= j and rises with j, so
//    a group writes only over slots that no later one reads, and later groups'
//    rows may be on their way meanwhile: a ring of cp.async copies keeps STAGES -
//    GROUP waves of 16 KB in flight, so that a group does not wait for its slowest
//    row.  A row is found through two dependent loads (its slot, its page); each is
//    issued a group ahead of its use.
// The move is bound by HBM: every kept row behind the first gap is read and
// written once, in runs of one row (128 to 512 bytes), which DRAM serves below
// its sequential rate (reads alone, rows of 256 bytes, every fourth kept: 3.2
// TB/s; of 192 bytes, every second: 4.7); with few units, by the latency of a
// group and its barrier.  The select is bound by its chain of block- or
// cluster-wide steps.  More units than two per SM take three CTAs per SM with
// rings of 4 waves, so that one's select covers another's move (768 units of 2048
// to 1024 slots of 192 bytes: 111 us; with two and rings of 6 127).  Fewer
// take two with 6 (256 units of 32768 to 8192 slots of 256 bytes 386, with three
// 574; 60 units of 25847 to 10818 slots of 128 bytes 84, with a barrier per
// wave 113), and units that leave a CTA an SM of its own rings of 12 where their
// waves fill them (one unit of 9230 to 9164 slots of 512 bytes 45; by one CTA's
// select and a barrier per wave 92).
#include <cooperative_groups.h>
#include <math.h>

#include <type_traits>

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
template <typename V>
__device__ __forceinline__ V block_scan(V v, V* red, V& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  V incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += u;
  }
  __syncthreads();  // the last scan's sums have been read
  if (lane == 31) red[warp] = incl;
  __syncthreads();
  V before = 0;
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
  unsigned long long red[kEvWarps];
  uint32_t kmin, kmax;  // over this CTA's middle slots
  int prefix, need, count;
  int kept, equals;     // of this CTA's slots: kept whatever happens to the equals, and those
};

// Slots of each of `ranks` CTAs that share a unit of n.
__device__ __forceinline__ int slice_of(int n, int ranks) { return ((n + ranks - 1) / ranks + 3) & ~3; }

// Lists the kept slots of a unit of n slots and compacts its sums.  Each of
// `ranks` CTAs (1, or the whole cluster) takes the slots [s0, s1), s0 a multiple
// of 4, which fit one tile if there are several; a thread holds SUB times four
// consecutive ones.  hist: [2][kEvBins].
template <int SUB>
__device__ __forceinline__ void select_unit(const EvictParams& p, int n, int rank, int ranks, const float* mass,
                                            float* mass_out, int32_t* kept, SelectShared& sh, int* hist) {
  // a count for each of the SUB parts of a tile, 16 bits each where there are several
  using Pack = typename std::conditional<SUB == 1, uint32_t, unsigned long long>::type;
  constexpr int HOLD = 4 * SUB, PART = 4 * kEvThreads, TILE = SUB * PART;
  const int tid = threadIdx.x, lane = tid & 31;
  Pack* red = reinterpret_cast<Pack*>(sh.red);
  const int64_t slots = (int64_t)p.max_pages * p.P;
  const int slice = slice_of(n, ranks);
  const int s0 = min(rank * slice, n), s1 = min(s0 + slice, n);
  const bool cut = n > p.budget;
  const int lo = cut ? p.sinks : 0, hi = cut ? n - p.recent : 0;  // the middle slots
  const int want = cut ? p.budget - p.sinks - p.recent : 0;       // of which this many stay
  const bool once = s1 - s0 <= TILE;
  auto sync = [&]() {
    if (ranks == 1) __syncthreads();
    else cg::this_cluster().sync();
  };
  auto peer = [&](auto* x, int r) { return ranks == 1 ? x : cg::this_cluster().map_shared_rank(x, r); };
  float x[HOLD];
  auto slot = [&](int base, int i) { return base + (i >> 2) * PART + tid * 4 + (i & 3); };
  auto load = [&](int base) {
#pragma unroll
    for (int i = 0; i < HOLD; i += 4) {
      const int t = slot(base, i);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (t < s1) {
        if (p.vec4) {
          v = *reinterpret_cast<const float4*>(mass + t);
        } else {
          v.x = mass[t];
          if (t + 1 < s1) v.y = mass[t + 1];
          if (t + 2 < s1) v.z = mass[t + 2];
          if (t + 3 < s1) v.w = mass[t + 3];
        }
      }
      x[i] = v.x;
      x[i + 1] = v.y;
      x[i + 2] = v.z;
      x[i + 3] = v.w;
    }
  };
  auto middle = [&](int t) { return t >= lo && t < min(hi, s1); };
  if (once) load(s0);

  // ---- threshold: keys above it stay, and the first `need` of its equals, both
  // counted from the smallest key of the unit and compared without their low
  // `rem` bits
  uint32_t kmin = 0, cur = 0;
  int need = want, rem = 0;
  int above_here = 0, equals = max(0, min(hi, s1) - max(lo, s0));  // of this CTA (above_here: of this thread's bins)
  if (want > 0) {
    for (int i = tid; i < 2 * kEvBins; i += kEvThreads) hist[i] = 0;
    if (SUB == 1) {
      rem = 32;
      __syncthreads();
    } else {
      // Many sums: bins over the range that they cover, else most would meet in a few.
      if (tid == 0) {
        sh.kmin = 0xFFFFFFFFu;
        sh.kmax = 0u;
      }
      __syncthreads();
      uint32_t a = 0xFFFFFFFFu, z = 0u;
      for (int base = s0; base < s1; base += TILE) {
        if (!once) load(base);
#pragma unroll
        for (int i = 0; i < HOLD; ++i)
          if (middle(slot(base, i))) {
            const uint32_t k = order_key(x[i]);
            a = min(a, k);
            z = max(z, k);
          }
      }
      a = __reduce_min_sync(0xFFFFFFFFu, a);
      z = __reduce_max_sync(0xFFFFFFFFu, z);
      if (lane == 0) {
        atomicMin(&sh.kmin, a);
        atomicMax(&sh.kmax, z);
      }
      sync();
      kmin = __reduce_min_sync(0xFFFFFFFFu, *peer(&sh.kmin, lane < ranks ? lane : 0));
      const uint32_t kmax = __reduce_max_sync(0xFFFFFFFFu, *peer(&sh.kmax, lane < ranks ? lane : 0));
      rem = 32 - __clz(kmax - kmin);
    }
    bool first = true;
    int buf = 0;
    while (rem > 0) {
      const int bits = min(rem, 11), down = rem - bits;
      int* own_hist = hist + buf * kEvBins;
      for (int base = s0; base < s1; base += TILE) {
        if (!once) load(base);
#pragma unroll
        for (int i = 0; i < HOLD; ++i)
          if (middle(slot(base, i))) {
            const uint32_t k = order_key(x[i]) - kmin;
            if (first || (k >> rem) == cur) atomicAdd(&own_hist[(k >> down) & ((1u << bits) - 1u)], 1);
          }
      }
      sync();
      // a thread owns four bins, from the top down
      static_assert(kEvBins == 4 * kEvThreads, "four bins per thread");
      const int b0 = kEvBins - 1 - 4 * tid;
      const int4 mine = reinterpret_cast<const int4*>(own_hist)[kEvThreads - 1 - tid];
      const int here[4] = {mine.w, mine.z, mine.y, mine.x};
      int own[4] = {0, 0, 0, 0};
      for (int r = 0; r < ranks; ++r) {
        const int4 o = peer(reinterpret_cast<int4*>(own_hist), r)[kEvThreads - 1 - tid];
        own[0] += o.w;
        own[1] += o.z;
        own[2] += o.y;
        own[3] += o.x;
      }
      const int sum = own[0] + own[1] + own[2] + own[3];
      Pack total;
      int above = (int)block_scan<Pack>((Pack)sum, red, total);
      if (above < need && need <= above + sum) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < need && need <= above + own[i]) {
            sh.prefix = b0 - i;
            sh.need = need - above;
            sh.count = own[i];
          }
          above += own[i];
        }
      }
      __syncthreads();
      const int bin = sh.prefix;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (b0 - i > bin) above_here += here[i];
      equals = own_hist[bin];
      cur = (first ? 0u : cur << bits) | (uint32_t)bin;
      need = sh.need;
      rem = down;
      first = false;
      if (sh.count == need) break;  // every key of the bin stays
      // (the other buffer's last counts were read before this pass's sync)
      buf ^= 1;
      for (int i = tid; i < kEvBins; i += kEvThreads) hist[buf * kEvBins + i] = 0;
      __syncthreads();
    }
  }

  // ---- the kept slots in order, behind those of the CTAs before
  int taken = 0, eq_seen = 0;
  if (ranks > 1 && !cut) {
    taken = s0;
  } else if (ranks > 1) {
    Pack total;
    block_scan<Pack>((Pack)above_here, red, total);
    if (tid == 0) {
      const int fixed = (s1 - s0) - max(0, min(hi, s1) - max(lo, s0));
      sh.kept = fixed + (int)total;
      sh.equals = equals;
    }
    sync();  // (and every CTA holds its sums: mass_out may be mass)
    for (int r = 0; r < rank; ++r) {
      taken += *peer(&sh.kept, r);
      eq_seen += *peer(&sh.equals, r);
    }
    if (want > 0) taken += min(need, eq_seen);
  }
  for (int base = s0; base < s1; base += TILE) {
    if (!once) load(base);
    uint32_t keep = 0, eq = 0;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
      const int t = slot(base, i);
      if (t >= s1) continue;
      if (!cut || t < lo || t >= hi) {
        keep |= 1u << i;
      } else if (want > 0) {
        const uint32_t k = (order_key(x[i]) - kmin) >> rem;
        if (k > cur) keep |= 1u << i;
        if (k == cur) eq |= 1u << i;
      }
    }
    // counts of the tile's parts in one sum; `before` gets those of slots before
    // the thread's, part by part
    auto count = [&](uint32_t bits, int (&before)[SUB]) -> int {
      Pack v = 0, total;
#pragma unroll
      for (int u = 0; u < SUB; ++u) v |= (Pack)__popc((bits >> (4 * u)) & 15u) << (16 * u);
      const Pack at = block_scan<Pack>(v, red, total);
      int sum = 0;
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        before[u] = sum + (int)((at >> (16 * u)) & 0xFFFFu);
        sum += (int)((total >> (16 * u)) & 0xFFFFu);
      }
      return sum;
    };
    int before[SUB];
    const int eq_total = count(eq, before);
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      int left = need - eq_seen - before[u];  // of this thread's equals
#pragma unroll
      for (int i = 4 * u; i < 4 * u + 4; ++i)
        if (((eq >> i) & 1u) && left-- > 0) keep |= 1u << i;
    }
    const int keep_total = count(keep, before);  // (a block barrier after every sum was read)
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      int at = taken + before[u];
#pragma unroll
      for (int i = 4 * u; i < 4 * u + 4; ++i)
        if ((keep >> i) & 1u) {
          kept[at] = slot(base, i);
          mass_out[at] = x[i];
          ++at;
        }
    }
    taken += keep_total;
    eq_seen += eq_total;
  }
  if (ranks == 1) __syncthreads();  // every sum has been read: mass_out may be mass
  const int out_n = min(n, p.budget), me = rank * kEvThreads + tid, all = ranks * kEvThreads;
  for (int j = out_n + me; j < p.budget; j += all) kept[j] = -1;
  for (int64_t t = out_n + me; t < slots; t += all) mass_out[t] = 0.f;
}

// ROWV: 16-byte vectors per row; STAGES: waves in the ring, GROUP of which are
// written between two barriers; CTAS: per SM
template <int ROWV, int STAGES, int GROUP, int CTAS>
__global__ void __launch_bounds__(kEvThreads, CTAS) evict_kernel(const EvictParams p) {
  __shared__ SelectShared sh;
  extern __shared__ uint4 ring[];  // [STAGES][2][kEvThreads]: each thread reads back its own copies
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
  if (c == 0 && h == 0 && rank == 0 && tid == 0) p.new_lens[b] = min(n, p.budget);
  {
    const float* mass = p.mass + unit * slots;
    float* mass_out = p.mass_out + unit * slots;
    int* hist = reinterpret_cast<int*>(ring);
    // the whole cluster selects where there is enough to share and its CTAs hold
    // all the sums; else the first CTA
    const bool share = n > 4 * kEvThreads && slice_of(n, C) <= 16 * kEvThreads;
    if (n <= 4 * kEvThreads) {
      if (rank == 0) select_unit<1>(p, n, 0, 1, mass, mass_out, kept, sh, hist);
    } else if (share || rank == 0) {
      select_unit<4>(p, n, rank, share ? C : 1, mass, mass_out, kept, sh, hist);
    }
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
  constexpr int kGroups = STAGES / GROUP;
  static_assert(STAGES % GROUP == 0 && kGroups >= 2, "whole groups");
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
  // The kept slots of the next group to load and of the one after; the pages of
  // the next one's rows and of their new places.
  int t[GROUP], t_next[GROUP], pg_s[GROUP], pg_d[GROUP];
  int w_load = 0;  // the next group's first wave
#pragma unroll
  for (int u = 0; u < GROUP; ++u) t[u] = kept_of(u);
#pragma unroll
  for (int u = 0; u < GROUP; ++u) t_next[u] = kept_of(GROUP + u);
#pragma unroll
  for (int u = 0; u < GROUP; ++u) {
    pg_s[u] = page_of(t[u]);
    pg_d[u] = page_of(t[u] >= 0 ? slot_of(u) : -1);
  }
  int to[STAGES];  // rows the ring's waves go to (-1: nothing moves)
  auto load = [&](int g) {
#pragma unroll
    for (int u = 0; u < GROUP; ++u) {
      const int s = g * GROUP + u, j = slot_of(w_load + u);
      to[s] = -1;
      if (t[u] >= 0 && t[u] != j) {
        const int src = row_of(t[u], pg_s[u]), dst = row_of(j, pg_d[u]);
        if (src < 0 || dst < 0) {
          report(p.status, WM_ERR_BOUNDS);
        } else {
          to[s] = dst;
          const int64_t at = (int64_t)src * ROWV + v;
          cp_async16(ring + (2 * s) * kEvThreads + tid, kb + at);
          cp_async16(ring + (2 * s + 1) * kEvThreads + tid, vb + at);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    w_load += GROUP;
#pragma unroll
    for (int u = 0; u < GROUP; ++u) {
      t[u] = t_next[u];
      pg_s[u] = page_of(t[u]);
      pg_d[u] = page_of(t[u] >= 0 ? slot_of(w_load + u) : -1);
    }
#pragma unroll
    for (int u = 0; u < GROUP; ++u) t_next[u] = kept_of(w_load + GROUP + u);
  };
#pragma unroll
  for (int g = 0; g < kGroups - 1; ++g) load(g);
  for (int w0 = 0; w0 < waves; w0 += STAGES) {
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      if (w0 + g * GROUP >= waves) break;
      load((g + kGroups - 1) % kGroups);  // the group kGroups - 1 further on
      asm volatile("cp.async.wait_group %0;" ::"n"(kGroups - 1) : "memory");
      barrier();  // every row of this group has been read
#pragma unroll
      for (int s = g * GROUP; s < (g + 1) * GROUP; ++s) {
        if (to[s] < 0) continue;
        const int64_t at = (int64_t)to[s] * ROWV + v;
        kb[at] = ring[(2 * s) * kEvThreads + tid];
        vb[at] = ring[(2 * s + 1) * kEvThreads + tid];
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <int ROWV, int STAGES, int GROUP, int CTAS>
cudaError_t launch_t(const EvictParams& p, cudaStream_t s) {
  static size_t smem_set[kSmemOptDevices] = {};
  auto kern = evict_kernel<ROWV, STAGES, GROUP, CTAS>;
  constexpr size_t smem = (size_t)STAGES * 2 * kEvThreads * sizeof(uint4);
  static_assert(smem >= 2 * kEvBins * sizeof(int), "the select's counts lie in the ring");
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
cudaError_t launch_rowv(const EvictParams& p, int64_t units, int sms, cudaStream_t s) {
  if (units > 2 * (int64_t)sms) return launch_t<ROWV, 4, 1, 3>(p, s);
  const int wave = p.cluster * (kEvThreads / ROWV);
  if (units * p.cluster > sms || p.budget <= 6 * wave) return launch_t<ROWV, 6, 3, 2>(p, s);
  return launch_t<ROWV, 12, 4, 1>(p, s);
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
  p.vec4 = (int64_t)p.max_pages * p.P % 4 == 0 && ((uintptr_t)p.mass & 15) == 0 ? 1 : 0;
  switch (rowv) {
    case 8: return launch_rowv<8>(p, units, sms, s);
    case 12: return launch_rowv<12>(p, units, sms, s);
    case 16: return launch_rowv<16>(p, units, sms, s);
    case 24: return launch_rowv<24>(p, units, sms, s);
    case 32: return launch_rowv<32>(p, units, sms, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace wm
