// Tensor-core attention of many query rows over part of the cache (bf16):
//
//  window: causal attention of query positions under a sliding window with
//    sinks; row at position i sees the slots t <= i with t < sinks or
//    t > i - window.  Rows are the positions of one query head.
//  prefix: the query rows of a whole batch over a prefix that its sequences
//    share, computed once; rows are the (sequence, query head) pairs of one kv
//    head.  The result of every row stays unnormalised, as (max, sum, O), for
//    the kernel that adds the row's own suffix.
//
// Both are dense contractions around a softmax and run on the tcgen05 tensor
// cores like the causal prefill attention (prefill_attn.cu): 128-row query
// tiles, 128-slot KV tiles, S and O in TMEM, P written over S as bf16 for the
// second product, the running max raised only when it grows by more than 2^8.
// What differs is the shape of the work.  A window makes every item short
// (about window / 128 + 2 KV tiles), so the CTA is persistent (one per SM) and
// its warps run ahead of each other across items: the TMA warp loads the next
// item's queries and first K tiles, and the MMA warp issues its first S, while
// the softmax warps still write the previous item's rows.
//
//  * warps 0-7, 8-15: softmax of query tile 0, 1, two threads per row, each over
//    64 columns (one thread's chain of a whole row was longer than the products
//    of both tiles);
//  * warp 16: each item's ranges (from its rows' positions), passed on through
//    shared memory, and the TMA loads of Q and K;
//  * warp 17: MMA issue, by its elected lane;
//  * warp 18: passes each V tile on to the MMA warp, its unseen rows zeroed
//    where there are any;
//  * warp 19: the TMA loads of V.
//
// The two query tiles of an item are two query heads of one kv head over the
// same rows where the group size is even, else consecutive rows of one head.
// A prefix with at most 128 rows per kv head has one query tile, and the two
// softmax groups take its even and odd KV tiles instead.
//
// A KV tile whose visible slots end early (the sinks, the end of a prefix) is
// only multiplied as far as they go, in steps of 64 columns.  Slots that no
// row of an item sees are never used: their pages are not fetched where a
// whole box is unseen, their V rows are zeroed, their scores replaced.
//
// Measured: 8192 rows of 32 heads of 128 under a window of 1024: 155 us, 838
// TFLOP/s of visible products (the tensor pipe 46% active, instruction issue
// 43%); a prefix of 32768 slots under 64 sequences of 32 query / 8 kv heads of
// 128: 38 us, 3.6 TB/s.  A step's chain bounds it: S, the softmax's reads and
// exponentials, P V, per query tile one after the other.  Two S and two O tiles
// fill tensor memory at a head size of 128; at 64 a further S would fit, but all
// sizes use the layout of 128 (the same rows with heads of 64: 138 us).
// Positions in no order (Item::sparse) make the load and V warps look through the
// item's positions, up to 256 for every box and every V row: 2048 such rows 214 us,
// in order 50.
#include <math.h>

#include "internal.h"
#include "range_attn.h"
#include "tc.cuh"

namespace wm {
namespace {

constexpr int kTM = 128;                  // query rows per tile (MMA M)
constexpr int kTN = 128;                  // slots per KV tile
constexpr int kQT = 2;                    // query tiles per item
constexpr int kTileWarps = 8;             // softmax warps per query tile: two threads per row
constexpr int kSoftWarps = kTileWarps * kQT;
constexpr int kLoadWarp = kSoftWarps;
constexpr int kMmaWarp = kSoftWarps + 1;
constexpr int kFixWarp = kSoftWarps + 2;
constexpr int kVWarp = kSoftWarps + 3;
constexpr int kTThreads = (kSoftWarps + 4) * 32;
constexpr uint32_t kBlock = 128u * 128u;  // bytes of a 64-column block of a 128-row tile
constexpr uint32_t kTmemCols = 512;       // S_i at 128 i (P_i at its columns 0-31 and 64-95), O_i at 256 + 128 i
constexpr float kStaleMax = 8.f;          // log2 headroom before O is rescaled

template <int HD>
struct TShape {
  static constexpr int CB = (HD + 63) / 64;  // 64-column blocks of a head row
  static constexpr int NSK = HD <= 64 ? 4 : 3;
  static constexpr int NSV = HD <= 64 ? 4 : 2;
  static constexpr uint32_t TILE_BYTES = CB * kBlock;  // one Q, K or V tile
  static constexpr uint32_t TILES = (kQT + NSK + NSV) * TILE_BYTES;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }
__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}

// The MMA warp runs as a whole, with every tensor instruction predicated on its
// elected lane: inside a branch of one lane the operands would not stay in
// uniform registers.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate,
                                       uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 e, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate,
                                       uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 e, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "setp.ne.b32 e, %1, 0;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)),
      "r"(lead)
      : "memory");
}

// Wait for this thread's TMEM loads; the registers of the one that is used next
// are operands, so that no use moves up across the wait.
__device__ __forceinline__ void tmem_wait_for(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                 "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                 "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]),
                 "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}

__device__ __forceinline__ void tmem_wait_for(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                 "+r"(r[15])::"memory");
}

// 32 bytes to global memory (wide: dst is 32-byte aligned).
__device__ __forceinline__ void store32(void* dst, const uint32_t (&u)[8], int wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(u[0]), "r"(u[1]),
                 "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(dst)[0] = make_uint4(u[0], u[1], u[2], u[3]);
    reinterpret_cast<uint4*>(dst)[1] = make_uint4(u[4], u[5], u[6], u[7]);
  }
}

// KV tiles of a query tile, or of the whole item: [0, sn) and [wf, we).
struct Span {
  int sn, wf, we;
  __device__ __forceinline__ bool has(int kt) const { return kt < sn || (kt >= wf && kt < we); }
};

// What the warps of a CTA need to know of an item.
struct Item {
  Span tile[kQT], all;
  int steps;   // KV tiles of the item
  int top;     // largest visible slot (-1: none)
  int wlo;     // smallest window start of a row
  int sparse;  // rows may leave slots between wlo and top that none of them sees
};

// Boxes of a step whose page does not exist, bit per box: K tile j + NSK is
// loaded once S of step j is there, and S runs at most two steps ahead of the
// softmax, so a ring of kBadRing is enough.
constexpr int kBadRing = 8;

// Shared memory behind the tiles.  (Nothing is static, so that the tiles start
// at the 1024-byte boundary that the swizzle needs: there is no room to align.)
template <int NSK, int NSV>
struct Shared {
  uint64_t qfull[2], qempty, mfull[2], mfree[2], kfull[NSK], kempty[NSK], vfull[NSV], vready[NSV], vempty[NSV];
  uint64_t sfull[kQT], pfull[2 * kQT], odone[kQT];
  uint64_t xbar[kQT * 4];       // the two warps of a quadrant of a tile
  float xval[kQT][2][kTM];      // what their threads tell each other
  Item items[2];
  uint32_t bad_boxes[kBadRing];
  uint32_t tmem_base;
};

struct Work {  // place of an item
  int b, h, row0, split;  // row0: first row of query tile 0
};

template <bool WIN>
__device__ __forceinline__ Work work_of(const TileParams& p, int it) {
  Work w;
  if (WIN) {
    const int ny = p.pair ? p.Hq / kQT : p.Hq;
    const int x = it % p.blocks, y = it / p.blocks;
    w.b = y / ny;
    w.h = (y - w.b * ny) * (p.pair ? kQT : 1);  // query head of tile 0
    w.row0 = x * (p.pair ? kTM : kQT * kTM);
    w.split = 0;
  } else {
    const int y = it / p.splits;
    w.split = it - y * p.splits;
    w.h = y % p.Hkv;  // kv head
    w.row0 = y / p.Hkv * (p.pair ? kTM : kQT * kTM);
    w.b = 0;
  }
  return w;
}

// Largest slot row r of the item's list sees (-1: none; bad: out of range).
template <bool WIN>
__device__ __forceinline__ int top_of(const TileParams& p, const Work& w, int r, bool& bad) {
  bad = false;
  const int max_slots = p.max_pages * p.P;
  if (WIN) {
    if (r >= p.rows) return -1;
    const int v = __ldg(p.pos + (int64_t)w.b * p.rows + r);
    bad = v < 0 || v >= max_slots;
    return bad ? -1 : v;
  }
  if (r >= p.rows) return -1;
  const int n = __ldg(p.pos + r / p.G);  // the sequence's slots
  bad = n < 0 || n > max_slots;
  return bad ? -1 : min(n, p.prefix_slots) - 1;
}

__device__ __forceinline__ int warp_max(int v) { return __reduce_max_sync(0xFFFFFFFFu, v); }
__device__ __forceinline__ int warp_min(int v) { return __reduce_min_sync(0xFFFFFFFFu, v); }

// The item's ranges (one warp).
template <bool WIN>
__device__ __forceinline__ Item item_of(const TileParams& p, const Work& w, int lane) {
  Item I;
  I.sparse = 0;
  I.wlo = WIN ? INT32_MAX : 0;
  I.top = -1;
  const int nt = p.pair ? 1 : kQT;  // tiles with rows of their own
  int tops[kQT], los[kQT];
#pragma unroll
  for (int i = 0; i < kQT; ++i) {
    tops[i] = -1;
    los[i] = INT32_MAX;
    if (i >= nt) continue;
    int mx = -1, mn = INT32_MAX;
    bool gap = false, bad;
#pragma unroll
    for (int x = 0; x < kTM / 32; ++x) {
      const int r = w.row0 + i * kTM + x * 32 + lane;
      const int t = top_of<WIN>(p, w, r, bad);
      mx = max(mx, t);
      if (t >= 0) mn = min(mn, t);
      if (WIN && r + 1 < p.rows && (i + 1 < nt || x * 32 + lane + 1 < kTM)) {
        // consecutive rows whose positions rise by at most the window see every
        // slot between them
        const int z = top_of<WIN>(p, w, r + 1, bad);
        gap = gap || t < 0 || z < t || z - t > p.window;
      }
    }
    tops[i] = warp_max(mx);
    mn = warp_min(mn);
    los[i] = WIN && tops[i] >= 0 && p.window > 0 ? max(mn - p.window + 1, 0) : INT32_MAX;
    if (WIN && __any_sync(0xFFFFFFFFu, gap)) I.sparse = 1;
    I.top = max(I.top, tops[i]);
    if (WIN) I.wlo = min(I.wlo, los[i]);
  }
  if (nt == 1) {
    tops[1] = tops[0];
    los[1] = los[0];
  }
  auto span = [&](int top, int lo) {
    Span s;
    s.sn = (min(p.sinks, top + 1) + kTN - 1) / kTN;
    s.wf = max(lo / kTN, s.sn);
    s.we = p.window > 0 ? max(top / kTN + 1, s.wf) : s.wf;
    if (top < 0) s.sn = s.wf = s.we = 0;
    return s;
  };
  if (WIN) {
#pragma unroll
    for (int i = 0; i < kQT; ++i) I.tile[i] = span(tops[i], los[i]);
    I.all = span(I.top, I.wlo);
  } else {
    const int n = I.top / kTN + 1, tiles = I.top >= 0 ? n : 0;
    I.all.sn = 0;
    I.all.wf = (int)((int64_t)w.split * tiles / p.splits);
    I.all.we = (int)((int64_t)(w.split + 1) * tiles / p.splits);
#pragma unroll
    for (int i = 0; i < kQT; ++i) {
      I.tile[i] = I.all;
      if (tops[i] < 0) I.tile[i].we = I.tile[i].wf;  // no row of this tile sees anything
    }
  }
  I.steps = I.all.sn + I.all.we - I.all.wf;
  return I;
}

template <bool WIN>
__device__ __forceinline__ int tile_at(const Item& I, int j) {
  return WIN && j < I.all.sn ? j : I.all.wf + j - I.all.sn;
}
// Query tile i takes part in step j.
template <bool WIN>
__device__ __forceinline__ bool active(const TileParams& p, const Item& I, int i, int j) {
  if (!WIN && p.pair) return (j & 1) == i;
  return I.tile[i].has(tile_at<WIN>(I, j));
}
// Columns of step j that may be seen: 64 or 128.
template <bool WIN>
__device__ __forceinline__ int columns(const TileParams& p, const Item& I, int kt) {
  int hi = I.top + 1 - kt * kTN;
  if (WIN && kt < I.all.sn && (kt + 1) * kTN <= I.wlo) hi = min(hi, p.sinks - kt * kTN);
  return hi > kTN / 2 ? kTN : kTN / 2;
}
// No row of the item sees a slot of t0 .. t1.
template <bool WIN>
__device__ __forceinline__ bool unseen(const TileParams& p, const Item& I, const Work& w, int t0, int t1) {
  if (t0 > I.top) return true;
  if (!WIN || t0 < p.sinks) return false;
  if (t1 < I.wlo) return true;
  if (!I.sparse) return false;
  const int n = min(p.rows - w.row0, p.pair ? kTM : kQT * kTM);
  for (int x = 0; x < n; ++x) {
    bool bad;
    const int t = top_of<WIN>(p, w, w.row0 + x, bad);
    if (t >= t0 && t - p.window < t1) return false;
  }
  return true;
}

template <int HD, bool WIN>
__global__ void __launch_bounds__(kTThreads, 1)
    tile_attn_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                     const __grid_constant__ CUtensorMap tmV, const TileParams p) {
  using SH = TShape<HD>;
  constexpr int CB = SH::CB, NSK = SH::NSK, NSV = SH::NSV;
  constexpr uint32_t TB = SH::TILE_BYTES;
  constexpr unsigned FULL = 0xFFFFFFFFu;
  static_assert(NSK + 3 <= kBadRing, "bad-page ring");
  using Sh = Shared<NSK, NSV>;
  static_assert(SH::TILES + sizeof(Sh) <= 227 * 1024, "shared memory");
  extern __shared__ __align__(1024) uint8_t smem_dyn[];
  Sh& sh = *reinterpret_cast<Sh*>(smem_dyn + SH::TILES);
  if ((smem_u32(smem_dyn) & 1023u) != 0) {  // (cannot happen)
    report(p.status, WM_ERR_CUDA);
    return;
  }
  auto& qfull = sh.qfull;
  auto& mfull = sh.mfull;
  auto& mfree = sh.mfree;
  auto& kfull = sh.kfull;
  auto& kempty = sh.kempty;
  auto& vfull = sh.vfull;
  auto& vready = sh.vready;
  auto& vempty = sh.vempty;
  auto& sfull = sh.sfull;
  auto& pfull = sh.pfull;
  auto& odone = sh.odone;
  auto& xbar = sh.xbar;
  uint64_t& qempty = sh.qempty;
  auto& items = sh.items;
  auto& bad_boxes = sh.bad_boxes;

  const int tid = threadIdx.x, lane = tid & 31;
  // Warp-uniform by construction (here and wherever a value of the MMA warp's
  // schedule comes from memory): the tensor instructions take their operands
  // from uniform registers, and a value the compiler cannot prove uniform costs
  // a move each, about 85 cycles per MMA against the 64 it takes to run.
  const int warp = uniform(tid >> 5);
  uint8_t* Qs = smem_dyn;
  uint8_t* Ks = Qs + kQT * TB;
  uint8_t* Vs = Ks + NSK * TB;

  if (tid == 0) {
    mbar_init(&qempty, 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&qfull[s], 1);
      mbar_init(&mfull[s], 1);
      mbar_init(&mfree[s], kSoftWarps + 3);
    }
    for (int s = 0; s < NSK; ++s) {
      mbar_init(&kfull[s], 1);
      mbar_init(&kempty[s], 1);
    }
    for (int s = 0; s < NSV; ++s) {
      mbar_init(&vfull[s], 1);
      mbar_init(&vready[s], 1);
      mbar_init(&vempty[s], 1);
    }
    for (int i = 0; i < kQT; ++i) {
      mbar_init(&sfull[i], 1);
      mbar_init(&pfull[i], kTileWarps);
      mbar_init(&pfull[kQT + i], kTileWarps / 2);
      for (int x = 0; x < 4; ++x) mbar_init(&xbar[4 * i + x], 2);
      mbar_init(&odone[i], 1);
    }
    fence_mbar_init();
    tc::prefetch_tensormap(&tmQ);
    tc::prefetch_tensormap(&tmK);
    tc::prefetch_tensormap(&tmV);
  }
  if (warp == 0) {
    tc::tmem_alloc(&sh.tmem_base, kTmemCols);
    tc::tmem_relinquish();
  }
  // Dependents may start once this grid has waited for the work before it:
  // what that work wrote is then visible to them as well.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = (uint32_t)uniform((int)sh.tmem_base);
  const int stride = (int)gridDim.x;
  bool ok = true;

  if (warp == kLoadWarp || warp == kVWarp) {
    // ================================================================ TMA
    // Lane t owns box t of every KV tile (one box per page, or one per 128
    // slots of a longer page) and fetches its page id one tile ahead.
    const int boxes = p.P >= kTN ? 1 : kTN >> p.log2P;  // <= 16 for pages of >= 8 slots
    const int brows = p.P >= kTN ? kTN : p.P;
    const bool kq = warp == kLoadWarp;
    const CUtensorMap* tm = kq ? &tmK : &tmV;
    int n_tile = 0;  // tiles loaded
    int no = 0;      // items of this CTA
    for (int it = (int)blockIdx.x; it < p.items && ok; it += stride, ++no) {
      const Work w = work_of<WIN>(p, it);
      Item I;
      if (kq) {
        I = item_of<WIN>(p, w, lane);
        if (no >= 2) ok = __all_sync(FULL, mbar_wait(&mfree[no & 1], ((no >> 1) - 1) & 1));
        if (!ok) break;
        if (lane == 0) {
          items[no & 1] = I;
          mbar_arrive(&mfull[no & 1]);
        }
        __syncwarp();
      } else {
        ok = __all_sync(FULL, mbar_wait(&mfull[no & 1], (no >> 1) & 1));
        if (!ok) break;
        I = items[no & 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(&mfree[no & 1]);
      }
      const int hkv = WIN ? w.h / p.G : w.h;
      // tensor-map row of this lane's box of step j (-brows: read zeros; below
      // that: zeros, and the box has no page)
      auto box_row = [&](int j) -> int {
        const int s = tile_at<WIN>(I, j) * kTN + lane * brows;  // first slot of the box
        const int lp = s >> p.log2P;                            // logical page
        int row = -brows;
        if (lane < boxes && lp < p.max_pages && !unseen<WIN>(p, I, w, s, s + brows - 1)) {
          const int pg = __ldg(p.page_table + (int64_t)w.b * p.max_pages + lp);
          if (pg >= 0 && pg < p.num_pages)
            row = (int)((((int64_t)p.chan * p.num_pages + pg) * p.Hkv + hkv) * p.P + (s & (p.P - 1)));
          else
            row = -2 * brows;
        }
        return row;
      };
      // the queries go out behind the first two K tiles (whose slots free up
      // before the previous item's queries do), but first of all in the first item
      auto load_q = [&]() {
        if (no >= 1) ok = __all_sync(FULL, mbar_wait(&qempty, (no - 1) & 1));
        if (!ok || lane != 0) return;
        const int nq = !WIN && p.pair ? 1 : kQT;
        if (I.steps == 0) {
          mbar_arrive(&qfull[no & 1]);
          return;
        }
        mbar_arrive_expect_tx(&qfull[no & 1], nq * TB);
        for (int i = 0; i < nq; ++i)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            if (WIN)
              tc::tma_load_2d(Qs + i * TB + cb * kBlock, &tmQ, (w.h + (p.pair ? i : 0)) * HD + cb * 64,
                              w.b * p.rows + w.row0 + (p.pair ? 0 : i * kTM), &qfull[no & 1]);
            else
              tc::tma_load_3d(Qs + i * TB + cb * kBlock, &tmQ, cb * 64, w.h * p.G, (w.row0 + i * kTM) / p.G,
                              &qfull[no & 1]);
          }
      };
      const int q_at = no == 0 ? 0 : min(2, I.steps);
      int row_next = I.steps > 0 ? box_row(0) : 0;
      for (int j = 0; j < I.steps; ++j, ++n_tile) {
        if (kq && j == q_at) {
          load_q();
          ok = __all_sync(FULL, ok);
          if (!ok) break;
        }
        const int row = row_next;
        if (j + 1 < I.steps) row_next = box_row(j + 1);
        const int depth = kq ? NSK : NSV, slot = n_tile % depth, turn = n_tile / depth;
        if (turn > 0) ok = __all_sync(FULL, mbar_wait(kq ? &kempty[slot] : &vempty[slot], (turn - 1) & 1));
        if (!ok) break;
        uint64_t* bar = kq ? &kfull[slot] : &vfull[slot];
        uint8_t* dst = (kq ? Ks : Vs) + slot * TB;
        if (kq) {
          const uint32_t gone = __ballot_sync(FULL, row < -brows);
          if (lane == 0) {
            bad_boxes[n_tile % kBadRing] = gone;
            if (gone) report(p.status, WM_ERR_BOUNDS);
          }
        }
        if (lane == 0) mbar_arrive_expect_tx(bar, TB);
        __syncwarp();
        if (lane < boxes)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) tc::tma_load_2d(dst + cb * kBlock + lane * brows * 128, tm, cb * 64, row, bar);
      }
      if (kq && ok && I.steps <= q_at) load_q();
      ok = __all_sync(FULL, ok);
    }
    if (!ok && lane == 0) {
      report(p.status, WM_ERR_TIMEOUT);
      // the copies still on their way to this CTA's shared memory (bounded)
      const int depth = kq ? NSK : NSV;
      for (int x = max(0, n_tile - depth); x < n_tile; ++x)
        mbar_wait(kq ? &kfull[x % depth] : &vfull[x % depth], (x / depth) & 1);
      if (kq && no > 0) mbar_wait(&qfull[(no - 1) & 1], ((no - 1) >> 1) & 1);
    }
  } else if (warp == kFixWarp) {
    // ================================================================ V tiles
    int vs = 0, no = 0;
    for (int it = (int)blockIdx.x; it < p.items && ok; it += stride, ++no) {
      ok = __all_sync(FULL, mbar_wait(&mfull[no & 1], (no >> 1) & 1));
      if (!ok) break;
      const Item I = items[no & 1];
      const Work w = work_of<WIN>(p, it);
      __syncwarp();  // every lane has read the item's ranges
      if (lane == 0) mbar_arrive(&mfree[no & 1]);
      for (int j = 0; j < I.steps; ++j, ++vs) {
        const int sv = vs % NSV, kt = tile_at<WIN>(I, j), s0 = kt * kTN;
        const int cols = columns<WIN>(p, I, kt);
        ok = __all_sync(FULL, mbar_wait(&vfull[sv], (vs / NSV) & 1));
        if (!ok) break;
        if (s0 + cols - 1 > I.top || (WIN && s0 + cols > p.sinks && (s0 < I.wlo || I.sparse))) {
          // slots that no row sees may hold anything: zero their V rows
          uint8_t* vt = Vs + sv * TB;
          for (int row = lane; row < cols; row += 32) {
            if (!unseen<WIN>(p, I, w, s0 + row, s0 + row)) continue;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
              for (int u = 0; u < 8; ++u)
                *reinterpret_cast<uint4*>(vt + cb * kBlock + row * 128 + u * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_shared();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&vready[sv]);
      }
    }
    if (!ok && lane == 0) report(p.status, WM_ERR_TIMEOUT);
  } else if (warp == kMmaWarp) {
    // ================================================================ MMA
    const uint32_t idesc_o = tc::idesc_bf16_f32(kTM, HD) | tc::kIdescBMajorMN;
    const int la = !WIN && p.pair ? 2 : 1;  // steps that S runs ahead of P V
    const uint32_t lead = elect_one();
    // descriptors of the first tiles (a tile further on: plus its bytes / 16)
    const uint64_t qd = tc::sdesc_kmajor_sw128(smem_u32(Qs)), kd0 = tc::sdesc_kmajor_sw128(smem_u32(Ks)),
                   vd0 = tc::sdesc_mnmajor_sw128(smem_u32(Vs), kBlock, 1024);
    auto all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(FULL, mbar_wait(bar, parity)) != 0; };
    int ks = 0, vs = 0;      // K tiles multiplied, V tiles multiplied
    int cnt0 = 0, cnt1 = 0;  // P V products of each query tile
    int no = 0;
    for (int it = (int)blockIdx.x; it < p.items && ok; it += stride, ++no) {
      ok = __all_sync(FULL, mbar_wait(&qfull[no & 1], (no >> 1) & 1));
      if (!ok) break;
      Item I;
      {
        const int* src = reinterpret_cast<const int*>(&items[no & 1]);
        int* to = reinterpret_cast<int*>(&I);
#pragma unroll
        for (int x = 0; x < (int)(sizeof(Item) / sizeof(int)); ++x) to[x] = uniform(src[x]);
      }
      const int steps = I.steps;
      __syncwarp();  // every lane has read the item's ranges
      if (lead) {
        mbar_arrive(&mfree[no & 1]);
        if (steps == 0) mbar_arrive(&qempty);
      }
      __syncwarp();
      {  // (a scope of its own: the item's schedule)
        auto issue_s = [&](int i, int cols) {  // S_i = Q_i K^T with the next K tile
          const uint64_t qi = qd + (!WIN && p.pair ? 0 : i) * (TB >> 4), kd = kd0 + (ks % NSK) * (TB >> 4);
          const uint32_t idesc = tc::idesc_bf16_f32(kTM, cols);
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t off = ((kk >> 2) * kBlock + (kk & 3) * 32) >> 4;
            mma_ss(tmem + 128 * i, qi + off, kd + off, idesc, kk > 0, lead);
          }
          commit(&sfull[i], lead);
        };
        // O_i += P_i V; the second half of P follows on its own barrier
        auto issue_pv = [&](int i, int cols, uint64_t vd, bool begun, uint32_t parity) -> bool {
          const uint32_t o = tmem + 256 + 128 * i, pa = tmem + 128 * i;
#pragma unroll
          for (int kk = 0; kk < kTN / 32; ++kk)
            mma_ts(o, pa + 8 * kk, vd + kk * (16 * 128 >> 4), idesc_o, begun || kk > 0, lead);
          if (cols == kTN) {
            if (!all(&pfull[kQT + i], parity)) return false;
            tc::fence_after_sync();
#pragma unroll
            for (int kk = kTN / 32; kk < kTN / 16; ++kk)
              mma_ts(o, pa + 64 + 8 * (kk - kTN / 32), vd + kk * (16 * 128 >> 4), idesc_o, 1, lead);
          } else if (!all(&pfull[kQT + i], parity)) {
            return false;
          }
          commit(&odone[i], lead);
          return true;
        };
        auto wait_k = [&]() -> bool { return all(&kfull[ks % NSK], (ks / NSK) & 1); };
        // the K tile of step j is free once the S issued so far are done
        auto free_k = [&](int j) {
          commit(&kempty[ks % NSK], lead);
          if (j == steps - 1) commit(&qempty, lead);
          ++ks;
        };
        for (int j = 0; j < la && j < steps && ok; ++j) {
          ok = wait_k();
          if (!ok) break;
          tc::fence_after_sync();
          const int cols = columns<WIN>(p, I, tile_at<WIN>(I, j));
#pragma unroll
          for (int i = 0; i < kQT; ++i)
            if (active<WIN>(p, I, i, j)) issue_s(i, cols);
          free_k(j);
        }
        bool begun0 = false, begun1 = false;  // O_i holds this item's products
        for (int j = 0; j < steps && ok; ++j, ++vs) {
          const int sv = vs % NSV;
          const int cols = columns<WIN>(p, I, tile_at<WIN>(I, j));
          const bool more = j + la < steps;
          const int cols_next = more ? columns<WIN>(p, I, tile_at<WIN>(I, j + la)) : 0;
          ok = all(&vready[sv], (vs / NSV) & 1) && (!more || wait_k());
          if (!ok) break;
          const uint64_t vd = vd0 + sv * (TB >> 4);
#pragma unroll
          for (int i = 0; i < kQT; ++i) {
            if (active<WIN>(p, I, i, j)) {
              int& cnt = i == 0 ? cnt0 : cnt1;
              bool& begun = i == 0 ? begun0 : begun1;
              ok = all(&pfull[i], cnt & 1);
              if (!ok) break;
              tc::fence_after_sync();
              ok = issue_pv(i, cols, vd, begun, cnt & 1);
              if (!ok) break;
              begun = true;
              ++cnt;
            }
            if (more && active<WIN>(p, I, i, j + la)) issue_s(i, cols_next);
          }
          if (!ok) break;
          commit(&vempty[sv], lead);
          if (more) free_k(j + la);
        }
      }
    }
    if (!ok && lead) report(p.status, WM_ERR_TIMEOUT);
  } else {
    // ================================================================ softmax
    const int i = warp / kTileWarps;     // query tile
    const int half = (warp >> 2) & 1;    // columns 64 half .. 64 half + 63
    const int lr = (warp & 3) * 32 + lane;  // row in the tile: the warp's quadrant of TMEM lanes
    const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t scol = 128 * i + 64 * half, ocol = 256 + 128 * i + HD / 2 * half;
    // The other half's value of the row: written to shared memory, then a barrier
    // of the two warps.  A step's value is overwritten only after the next S is
    // there, which was issued after both warps handed on this step's P.
    uint64_t* xb = &xbar[4 * i + (warp & 3)];
    int xn = 0;  // barriers passed
    auto meet = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(xb);
      return __all_sync(FULL, mbar_wait(xb, xn++ & 1));
    };
    auto exchange = [&](float mine, float& other) -> bool {
      sh.xval[i][half][lr] = mine;
      if (!meet()) return false;
      other = sh.xval[i][half ^ 1][lr];
      return true;
    };
    int cnt = 0;                         // steps of this tile, over all items
    int done = 0;                        // steps of the CTA before this item
    const int log2b = p.P >= kTN ? 7 : p.log2P;  // slots per box
    int no = 0;
    // largest slot this thread's row of item `it` sees, fetched an item ahead
    auto row_top = [&](int it) -> int {
      const Work w = work_of<WIN>(p, it);
      bool bad;
      const int t = top_of<WIN>(p, w, w.row0 + (p.pair ? 0 : i * kTM) + lr, bad);
      if (bad) report(p.status, WM_ERR_BOUNDS);
      return t;
    };
    int top_next = (int)blockIdx.x < p.items ? row_top((int)blockIdx.x) : -1;
    // tcgen05.ld / st are warp-collective: every lane of the warp issues each
    // one, and the wait outcomes are made warp-uniform before any branch
    for (int it = (int)blockIdx.x; it < p.items && ok; it += stride, ++no) {
      const int mytop = top_next;  // largest slot this thread's row sees
      if (it + stride < p.items) top_next = row_top(it + stride);
      ok = __all_sync(FULL, mbar_wait(&qfull[no & 1], (no >> 1) & 1));
      if (!ok) break;
      const Item& I = items[no & 1];
      const Span mine = i == 0 ? I.tile[0] : I.tile[1];
      const int steps = I.steps;
      float m = -INFINITY, l = 0.f;  // max used for P (log2 units) and running sum
      int x = 0;                     // steps of this tile in the item
      for (int j = 0; j < steps && ok; ++j) {
        const int kt = tile_at<WIN>(I, j), s0 = kt * kTN;
        if (!WIN && p.pair ? (j & 1) != i : !mine.has(kt)) continue;
        ok = __all_sync(FULL, mbar_wait(&sfull[i], cnt & 1));
        if (!ok) break;
        tc::fence_after_sync();
        const int nc = columns<WIN>(p, I, kt) / 32;  // 32-column parts of the step: 2 or 4
        // Visible columns of this row: e < vis, and under a window e < es (sinks)
        // or e >= el (the row's window).  Masked scores become -inf.
        const int vis = mytop - s0 + 1;
        int es = 0, el = 0;
        if (WIN) {
          es = p.sinks - s0;
          el = mytop - p.window + 1 - s0;
          if (es >= el) el = 0;
        }
        const uint32_t gone = bad_boxes[(done + j) % kBadRing];
        const bool masked = __any_sync(FULL, vis < 32 * nc || el > 0 || gone != 0);
        // The warp's two parts of 32 columns: nothing of one is seen (0), some (1) or
        // all of it (2); a diagonal or a window's edge leaves most of them whole.
        uint32_t see[2] = {0xFFFFFFFFu, 0xFFFFFFFFu};  // bit per column
        int kind[2] = {2, 2};
        if (masked) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int c0 = 64 * half + 32 * c;
            auto below = [&](int n) -> uint32_t {  // columns e < n
              return n >= c0 + 32 ? 0xFFFFFFFFu : n <= c0 ? 0u : (1u << (n - c0)) - 1u;
            };
            see[c] = below(vis) & (below(es) | ~below(el));
            if (gone)
              for (int e = 0; e < 32; ++e)
                if ((gone >> ((c0 + e) >> log2b)) & 1u) see[c] &= ~(1u << e);
            kind[c] = __all_sync(FULL, see[c] == 0xFFFFFFFFu) ? 2 : __any_sync(FULL, see[c] != 0u) ? 1 : 0;
          }
        }
        auto mask_part = [&](uint32_t bits, uint32_t (&v)[32]) {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = (bits >> e) & 1u ? v[e] : 0xFF800000u;
        };
        // The thread's part of the row is read from TMEM twice, 32 columns at a
        // time: for its maximum, then for the probabilities.  (Unrolled loops, or
        // separate ones for masked steps, cost more in the instruction cache than
        // they save.)
        const bool mine_too = nc > 2 * half;  // (a step of 64 columns is the lower half's)
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (mine_too) {
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            const int k = c == 0 ? kind[0] : kind[1];
            if (k == 0) continue;
            uint32_t v[32];
            tc::tmem_ld32(lane_base + scol + 32 * c, v);
            tmem_wait_for(v);
            if (k == 1) mask_part(c == 0 ? see[0] : see[1], v);
#pragma unroll
            for (int e = 0; e < 32; ++e) mx[e & 3] = fmaxf(mx[e & 3], __uint_as_float(v[e]));
          }
        }
        float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), mo = 0.f;
        ok = exchange(mt, mo);
        if (!ok) break;
        mt = fmaxf(mt, mo) * p.qscale;  // qscale > 0: the max commutes with the scale
        float scale = 1.f;
        const bool raise = (m == -INFINITY) ? (mt != -INFINITY) : (mt > m + kStaleMax);
        if (raise) {
          scale = (m == -INFINITY) ? 0.f : ex2(m - mt);
          m = mt;
        }
        if (__any_sync(FULL, raise && x > 0)) {
          // a row's max grew past the headroom: rescale O (every lane of the
          // warp takes part; rows that did not raise their max scale by 1)
          // once P V of the previous step has landed in it
          const float fac = raise && x > 0 ? scale : 1.f;
          ok = __all_sync(FULL, mbar_wait(&odone[i], (cnt - 1) & 1));
          if (!ok) break;
          tc::fence_after_sync();
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t o[16];
            tc::tmem_ld16(lane_base + ocol + 16 * c, o);
            tmem_wait_for(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fac);
            tc::tmem_st16(lane_base + ocol + 16 * c, o);
          }
          tc::tmem_st_wait();
        }
        // P V of the first 64 slots starts while the others' P is computed; it
        // needs the lower half's P, and O rescaled by both.
        tc::fence_before_sync();
        __syncwarp();
        if (half == 1 && lane == 0) mbar_arrive(&pfull[i]);
        // p = 2^(s * qscale - m) in pairs; masked slots give 0, and so do rows
        // that have seen nothing yet.  P enters the product as bf16 (the tensor
        // cores' operand); the row sum is kept in fp32 from the unrounded values.
        const float nm = m == -INFINITY ? 0.f : -m;
        const float2 qs2 = make_float2(p.qscale, p.qscale), nm2 = make_float2(nm, nm);
        float2 sum2 = make_float2(0.f, 0.f);
        float2 sum2b = make_float2(0.f, 0.f);
        if (mine_too) {
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            const int k = c == 0 ? kind[0] : kind[1];
            uint32_t v[32], pk[16];
            if (k == 0) {
#pragma unroll
              for (int e = 0; e < 16; ++e) pk[e] = 0u;
              tc::tmem_st16(lane_base + scol + 16 * c, pk);
              continue;
            }
            tc::tmem_ld32(lane_base + scol + 32 * c, v);
            tmem_wait_for(v);
            if (k == 1) mask_part(c == 0 ? see[0] : see[1], v);
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float2 y = __ffma2_rn(make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), qs2, nm2);
              const float2 pr = make_float2(ex2(y.x), ex2(y.y));
              if (e & 2) sum2b = __fadd2_rn(sum2b, pr);
              else sum2 = __fadd2_rn(sum2, pr);
              const __nv_bfloat162 h = __floats2bfloat162_rn(pr.x, pr.y);
              pk[e / 2] = *reinterpret_cast<const uint32_t*>(&h);
            }
            // P over this thread's own S columns that have been read
            tc::tmem_st16(lane_base + scol + 16 * c, pk);
          }
          tc::tmem_st_wait();
          tc::fence_before_sync();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&pfull[half == 0 ? i : kQT + i]);
        sum2 = __fadd2_rn(sum2, sum2b);
        l = l * scale + (sum2.x + sum2.y);
        ++cnt;
        ++x;
      }
      if (ok && x > 0) ok = __all_sync(FULL, mbar_wait(&odone[i], (cnt - 1) & 1));
      if (ok && x > 0) {  // both halves' sums (the same in both threads: addition commutes)
        float lo = 0.f;
        ok = exchange(l, lo) && meet();  // (the next item's first value waits for both reads)
        l += lo;
      }
      if (!ok) break;
      __syncwarp();  // every lane is done with the item's ranges
      if (lane == 0) mbar_arrive(&mfree[no & 1]);
      // ---- this row's result.  The next item's first P V overwrites O only
      // after this thread has arrived on pfull again.
      tc::fence_after_sync();
      done += steps;
      const Work w = work_of<WIN>(p, it);
      const int r = w.row0 + (p.pair ? 0 : i * kTM) + lr;
      const bool live = r < p.rows;
      const float inv = WIN ? (l > 0.f ? 1.f / l : 0.f) : 1.f;
      __nv_bfloat16* dst = nullptr;
      float* rec = nullptr;
      if (WIN)
        dst = reinterpret_cast<__nv_bfloat16*>(p.out) +
              (((int64_t)w.b * p.rows + r) * p.Hq + w.h + (p.pair ? i : 0)) * HD;
      else
        rec = p.part + (((int64_t)w.h * p.rows + r) * p.records + (p.pair ? w.split * kQT + i : w.split)) * tile_rec(HD);
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {  // 16 columns of this thread's half
        uint32_t o[16];
        if (x > 0) {  // the same for the whole warp group
          tc::tmem_ld16(lane_base + ocol + 16 * c, o);
          tmem_wait_for(o);
        }
        if (!live) continue;
        const int col = HD / 2 * half + 16 * c;
        if (WIN) {
          uint32_t u[8];
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const float f0 = x > 0 ? __uint_as_float(o[2 * t]) * inv : 0.f;
            const float f1 = x > 0 ? __uint_as_float(o[2 * t + 1]) * inv : 0.f;
            const __nv_bfloat162 h = __floats2bfloat162_rn(f0, f1);
            u[t] = *reinterpret_cast<const uint32_t*>(&h);
          }
          store32(dst + col, u, p.wide_out);
        } else if (x > 0) {
#pragma unroll
          for (int e = 0; e < 16; e += 8) {
            uint32_t u[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) u[t] = o[e + t];
            store32(rec + col + e, u, 1);
          }
        }
      }
      if (!WIN && live && half == 0) *reinterpret_cast<float2*>(rec + HD) = make_float2(m, l);
      tc::fence_before_sync();
    }
    if (!ok) report(p.status, WM_ERR_TIMEOUT);
  }
  // Every MMA this CTA issued has completed (each item's last products were
  // waited on, or the CTA gave up after a bounded wait); release TMEM.
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, kTmemCols);
  }
}

template <int HD, bool WIN>
cudaError_t launch_t(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const TileParams& p, int sms,
                     cudaStream_t s) {
  static size_t smem_set[kSmemOptDevices] = {};
  auto kern = tile_attn_kernel<HD, WIN>;
  constexpr size_t smem = TShape<HD>::TILES + sizeof(Shared<TShape<HD>::NSK, TShape<HD>::NSV>);
  if (cudaError_t e = opt_in_smem(kern, smem, smem_set); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.items < sms ? p.items : sms));
  cfg.blockDim = dim3(kTThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, q, k, v, p);
}

}  // namespace

cudaError_t launch_tile_attn(TileParams p, const TileInputs& in, int sms, cudaStream_t s) {
  const bool win = p.part == nullptr;
  p.wide_out = ((uintptr_t)p.out & 31) == 0 ? 1 : 0;
  CUtensorMap tq, tk, tv;
  const uint64_t pool_rows = (uint64_t)in.k * p.num_pages * p.Hkv * p.P;
  const uint32_t box_rows = p.P >= kTN ? (uint32_t)kTN : (uint32_t)p.P;
  const bool q_ok = win ? tma_map_bf16_2d(&tq, in.q, (uint64_t)in.B * p.rows, (uint64_t)p.Hq * in.d,
                                          (uint64_t)p.Hq * in.d, (uint32_t)kTM)
                        : tma_map_bf16_3d(&tq, in.q, (uint64_t)in.B, (uint64_t)p.Hq, (uint64_t)in.d,
                                          (uint32_t)(kTM / p.G), (uint32_t)p.G);
  if (!q_ok || !tma_map_bf16_2d(&tk, in.k_pool, pool_rows, in.d, in.d, box_rows) ||
      !tma_map_bf16_2d(&tv, in.v_pool, pool_rows, in.d, in.d, box_rows))
    return cudaErrorInvalidValue;
  switch (in.d) {
    case 64: return win ? launch_t<64, true>(tq, tk, tv, p, sms, s) : launch_t<64, false>(tq, tk, tv, p, sms, s);
    case 96: return win ? launch_t<96, true>(tq, tk, tv, p, sms, s) : launch_t<96, false>(tq, tk, tv, p, sms, s);
    case 128: return win ? launch_t<128, true>(tq, tk, tv, p, sms, s) : launch_t<128, false>(tq, tk, tv, p, sms, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace wm
