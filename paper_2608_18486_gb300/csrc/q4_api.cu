// C ABI of the cache held in 4 bits (declared in include/wm.h): its layout, rows
// of a cache to 4 bits and back, the pool appended in 4 bits, and attention over
// it.  Argument checks, work splits and kernel dispatch; all device memory
// belongs to the caller.
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include "api_util.h"
#include "internal.h"
#include "q4.h"
#include "range_attn.h"
#include "wm.h"

namespace wm {

cudaError_t launch_q4_attn_bf16(const Q4AttnParams& p, int d, cudaStream_t s);
cudaError_t launch_q4_attn_f32(const Q4AttnParams& p, int d, cudaStream_t s);

cudaError_t launch_q4_attn(const Q4AttnParams& p, int dtype, int d, cudaStream_t s) {
  return dtype == WM_DT_F32 ? launch_q4_attn_f32(p, d, s) : launch_q4_attn_bf16(p, d, s);
}

}  // namespace wm

namespace {

using namespace wm;

constexpr int kMaxBatch = 4096;

wm_status cuda_status(cudaError_t e) { return e == cudaSuccess ? WM_OK : WM_ERR_CUDA; }

// The 4-bit cache belongs to the config and is usable.
wm_status check_q4(const wm_config& c, const wm_q4_cache* q4) {
  if (!q4 || !q4->pool || q4->num_pages < 1 || !aligned(q4->pool, 16)) return WM_ERR_INVALID_ARG;
  if (q4->k != c.k || q4->Hkv != c.Hkv || q4->page_size != c.page_size || q4->d != c.d) return WM_ERR_INVALID_ARG;
  // 32-bit tiles per channel
  if ((int64_t)q4->num_pages * c.Hkv * (c.page_size / q4_tile_slots(c.page_size)) > INT32_MAX) return WM_ERR_UNSUPPORTED;
  return WM_OK;
}

// Checks of every call that takes a 4-bit cache, its page table and a batch.
wm_status check_call(const wm_config* c, const wm_q4_cache* q4, int32_t B, int32_t max_pages) {
  wm_status st = wm_config_check(c);
  if (st != WM_OK) return st;
  if ((st = check_q4(*c, q4)) != WM_OK) return st;
  if (B < 0 || max_pages < 1) return WM_ERR_INVALID_ARG;
  if ((int64_t)max_pages * c->page_size > INT32_MAX / 2) return WM_ERR_INVALID_ARG;
  return WM_OK;
}

size_t channel_bytes(const wm_config& c, int32_t num_pages) {
  return (size_t)num_pages * c.Hkv * q4_page_bytes(c.page_size, c.d);
}

// K (or V) rows of one token of each of B sequences, all channels
size_t row_bytes(const wm_config& c, int32_t B) {
  return align256((size_t)c.k * B * c.Hkv * c.d * elem_size(c.dtype));
}

Q4CopyParams copy_params(const wm_config& c, const wm_q4_cache& q4, int32_t B, int32_t max_pages, int32_t span,
                         int32_t* dev_status) {
  Q4CopyParams p{};
  p.pool = (uint8_t*)q4.pool;
  p.status = dev_status;
  p.page_bytes = q4_page_bytes(c.page_size, c.d);
  p.B = B;
  p.k = c.k;
  p.Hkv = c.Hkv;
  p.P = c.page_size;
  p.log2P = ilog2(c.page_size);
  p.tile = q4_tile_slots(c.page_size);
  p.log2tile = ilog2(p.tile);
  p.tile_bytes = (int32_t)q4_tile_bytes(c.page_size, c.d);
  p.q4_pages = q4.num_pages;
  p.max_pages = max_pages;
  p.span = span;
  p.steps = (span + 2 * kQ4Step - 2) / kQ4Step;  // a range may start and end inside a tile
  return p;
}

wm_status copy_ranges(bool write, const wm_config* c, const wm_cache* cache, const int32_t* table,
                      const wm_q4_cache* q4, const int32_t* q4_table, const int32_t* first, const int32_t* last,
                      int32_t span, int32_t B, int32_t max_pages, int32_t* dev_status, void* stream) {
  wm_status st = check_call(c, q4, B, max_pages);
  if (st != WM_OK) return st;
  if ((st = check_cache(*c, cache)) != WM_OK) return st;
  if (span < 0) return WM_ERR_INVALID_ARG;
  if (B == 0 || span == 0) return WM_OK;
  if (!table || !q4_table || !first || !last) return WM_ERR_INVALID_ARG;
  const int32_t slots = max_pages * c->page_size;
  Q4CopyParams p = copy_params(*c, *q4, B, max_pages, span < slots ? span : slots, dev_status);
  if ((int64_t)p.k * B * p.steps * p.Hkv > INT32_MAX / 2) return WM_ERR_UNSUPPORTED;
  p.k_rows = cache->k_pool;
  p.v_rows = cache->v_pool;
  p.row_table = table;
  p.q4_table = q4_table;
  p.first = first;
  p.last = last;
  p.rows_at = kQ4Paged;
  p.row_pages = cache->num_pages;
  return cuda_status(write ? launch_q4_write(p, c->dtype, c->d, sm_count(), (cudaStream_t)stream)
                           : launch_q4_read(p, c->dtype, c->d, sm_count(), (cudaStream_t)stream));
}

// Clusters of C CTAs that are resident at once where an SM takes k CTAs (a GPC's SMs
// are not always taken whole).  0: unknown.
__global__ void __launch_bounds__(kQ4Warps * 32) q4_places_kernel() {}  // (asked about, never launched)

int cluster_places(int C, int k) {
  static int known[kSmemOptDevices][kQ4MaxCtas][kQ4MaxCluster] = {};
  static size_t smem_set[kSmemOptDevices] = {};
  int dev = 0, per_sm = 0, reserved = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kSmemOptDevices) return 0;
  int& slot = known[dev][k - 1][C - 1];
  if ((n = __atomic_load_n(&slot, __ATOMIC_RELAXED)) != 0) return n;
  if (cudaDeviceGetAttribute(&per_sm, cudaDevAttrMaxSharedMemoryPerMultiprocessor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&reserved, cudaDevAttrReservedSharedMemoryPerBlock, dev) != cudaSuccess)
    return 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)C);
  cfg.blockDim = dim3(kQ4Warps * 32);
  cfg.dynamicSmemBytes = (size_t)((per_sm / k - reserved) / 128 * 128);  // k of them, not k + 1
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)C;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (opt_in_smem(q4_places_kernel, cfg.dynamicSmemBytes, smem_set) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, q4_places_kernel, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();
    return 0;
  }
  __atomic_store_n(&slot, n, __ATOMIC_RELAXED);
  return n;
}

// CTAs per unit, at most `most`, where an SM takes per_sm of them.  The units of an SM that
// has k CTAs take k / C of a CTA's time each, with k small a little more: fewer
// loads in flight.  One cluster more than are resident at once takes a second wave.  us by C
// (bf16, 4 query heads of 128, 4096 slots): 60 units 1: 20.7, 2: 17.0, 4: 13.5, 7: 14.5, 8: 13.7;
// 84 units 2: 21.2, 4: 16.8, 5: 15.3, 6: 16.2, 7 (two waves): 22.1; 120 units 1: 31.3, 2: 22.6,
// 4: 22.1, 5 (two waves): 27.8; 152 units 1: 28.4, 2: 23.0, 3: 27.0.
int cluster_size(int64_t units, int most, int per_sm) {
  constexpr double load[kQ4MaxCtas] = {1.5, 2.2, 3.1, 4.};
  double least = 1e30;
  int best = 1;
  for (int C = 1; C <= most; ++C)
    for (int k = 1; k <= per_sm; ++k)
      if (units <= cluster_places(C, k)) {
        if (load[k - 1] / C < least) {
          least = load[k - 1] / C;
          best = C;
        }
        break;
      }
  return best;
}

// Split of an attention call.  Short units are one cluster each, joined on chip; the
// steps of long ones are spread evenly over the resident CTAs, whatever the lengths,
// and a second kernel joins the units that were cut.
struct Q4Plan {
  int nb, col_blocks;
  int pieces;    // CTAs per unit at most, or of the spread
  int per_sm;    // CTAs
  bool spread;
  size_t total;  // workspace
};

constexpr double kWideMb = 55.;  // MB of codes times groups of 8 columns
constexpr int kLongSteps = 14;    // steps of a warp from which they are spread, with few CTAs,
constexpr int kFilledSteps = 32;  // and so many more where the CTAs fill the SMs

Q4Plan attn_plan(const wm_config& c, int32_t B, int32_t Tq, int32_t max_pages) {
  const int64_t cols = (int64_t)Tq * (c.Hq / c.Hkv);
  Q4Plan pl{};
  // 16 columns per unit read the codes once for both eights, but run half the warps: for
  // enough work only.  us with 16 / 8 columns per unit (32 query, 8 kv heads of 128): 1 sequence
  // of 512 slots, 4 rows 10.1 / 9.0; of 8192, 8 rows 17.6 / 14.2, 32 rows 28.1 / 34.7; 8 of
  // 32768, 4 rows 86 / 114; 16 of 2048, 4 rows 20.7 / 22.9; 8 of 4096, 12 heads of 64, 16 rows
  // 15.5 / 17.2.  What the rule does not see is a second wave of the fewer CTAs that 16 columns
  // leave on an SM; it takes the slower form of 1 of 16384, 8 rows 25.9 / 21.6, 16 of 2048, 12 heads
  // of 64, 16 rows 17.4 / 16.7 and 20 rows 31.6 / 20.5.
  const double mb = (double)B * max_pages * c.page_size * c.Hkv * (c.d + c.d / 8) * 1e-6;
  pl.nb = cols > 8 && c.dtype == WM_DT_BF16 && mb * (double)((cols + 7) / 8) > kWideMb ? 2 : 1;
  pl.col_blocks = (int)((cols + 8 * pl.nb - 1) / (8 * pl.nb));
  const int64_t units = (int64_t)B * c.Hkv * pl.col_blocks;
  const int64_t steps = ((int64_t)max_pages * c.page_size + kQ4Slots - 1) / kQ4Slots;
  pl.per_sm = q4_ctas_per_sm(c.dtype == WM_DT_BF16, pl.nb, c.dtype == WM_DT_F32 && cols <= kQ4Fold);
  const int resident = sm_count() * pl.per_sm;
  // at most as many CTAs per unit as are resident, a step per warp at least
  int64_t C = resident / units;
  if (C > steps / kQ4Warps) C = steps / kQ4Warps;
  C = C < 1 ? 1 : C > kQ4MaxCluster ? kQ4MaxCluster : C;
  pl.pieces = (int)C;
  pl.total = 256;
  // The spread has a start (a scan of the lengths), a second kernel, and a share of it drains its
  // rings at each unit's end: for long units, the sooner the fewer CTAs these would make
  // otherwise, and not where a CTA would take several units.  us, spread / not, heads of 128,
  // lengths from half of the largest to it: 32 heads: 16 x 16384 slots 147 / 151, 32 x 8192 148 / 152, 48 x
  // 5461 151 / 141, 128 x 2048 169 / 145; 32/8 heads: 16 x 8192 39 / 28, 64 x 4096 63 / 46,
  // 1 x 32768 19 / 28; 8/2 heads: 1 x 16384 14.4 / 16.3, 8 x 32768 24 / 35, 8 x 16384 20.4 / 20.3.
  // Of 168 sizes (half of them with equal lengths) 8 take the slower form, by 13% at most: 8 x 16384,
  // 8/2 heads, equal lengths 18.1 / 20.5 (not spread); 48 x 5461, 32/8 heads 58 / 51 (spread).
  const double fill = (double)(units * C) / resident;
  const double longest = kLongSteps + kFilledSteps * (fill < 1. ? fill : 1.);
  if (pl.col_blocks == 1 && units <= 2 * resident && (double)steps > (double)(C * kQ4Warps) * longest) {
    pl.pieces = resident;
    pl.spread = true;
    pl.total = align256(sizeof(float) * 2 * (size_t)resident * q4_rec(8 * pl.nb, c.d));
  }
  return pl;
}

wm_status attn(const wm_config& c, const wm_q4_cache& q4, int32_t layer, const void* q, const int32_t* page_table,
               const int32_t* lens, int32_t len_add, int32_t B, int32_t Tq, int32_t max_pages, void* out,
               void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream) {
  if (!q || !page_table || !lens || !out || !workspace) return WM_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256)) return WM_ERR_INVALID_ARG;
  const Q4Plan pl = attn_plan(c, B, Tq, max_pages);
  if (ws_bytes < pl.total) return WM_ERR_INVALID_ARG;
  Q4AttnParams p{};
  p.pool = (const uint8_t*)q4.pool + c.chan_of_layer[layer] * channel_bytes(c, q4.num_pages);
  p.q = q;
  p.out = out;
  p.page_table = page_table;
  p.lens = lens;
  p.status = dev_status;
  p.part = pl.spread ? (float*)workspace : nullptr;
  p.len_add = len_add;
  p.B = B;
  p.Tq = Tq;
  p.Hq = c.Hq;
  p.Hkv = c.Hkv;
  p.G = c.Hq / c.Hkv;
  p.P = c.page_size;
  p.log2P = ilog2(c.page_size);
  p.tile = q4_tile_slots(c.page_size);
  p.log2tile = ilog2(p.tile);
  p.tile_bytes = (int32_t)q4_tile_bytes(c.page_size, c.d);
  p.num_pages = q4.num_pages;
  p.max_pages = max_pages;
  p.col_blocks = pl.col_blocks;
  p.nb = pl.nb;
  p.pieces = pl.spread ? pl.pieces : cluster_size((int64_t)B * c.Hkv * pl.col_blocks, pl.pieces, pl.per_sm);
  p.qscale = (float)(1.4426950408889634 / sqrt((double)c.d));
  return cuda_status(launch_q4_attn(p, c.dtype, c.d, (cudaStream_t)stream));
}

// Many rows: a group of sequences is read back into the workspace (bf16 rows of one
// channel) and attended to by the tensor-core kernel.  Where the group's rows alone make
// too few items for the SMs, its KV tiles are cut as well, by the form of that kernel
// for a prefix that rows of unequal lengths share: the rows of a sequence are such.
struct RowsPlan {
  bool tiles;
  int group;                       // sequences read back at once
  bool cut;
  int pair, blocks, splits, records;
  int joined;                      // cut: sequences whose partial records are held, and joined, at once
  size_t off_v, off_table, off_last, off_lens, off_part, total;
};

// Estimates in us that choose between the two forms, and whether the KV tiles are cut.
// Streaming: 16 columns take as long as the codes' stream, and every CTA has a start
// and an end.  Tensor cores: reading back (codes in, rows out, rows in again), one step
// of 2 x 128 rows over a KV tile, the launches, the partial records' way to their join.
// Measured (streaming / tensor cores; heads of 128, 32 query and 8 kv heads): 1 sequence of 8192
// slots, 32 rows 28 / 33, 64 rows 47 / 35, 256 rows 157 / 50; 8 of 32768, 16 rows 296 / 532, 32
// rows 587 / 553, 64 rows 1059 / 557; 32 of 1024, 16 rows 63 / 123, 32 rows 116 / 97.  Whole
// KV ranges / cut ones: 16 of 4096, 256 rows 293 / 520; 32 of 8192, 300 rows, 32/4 heads 1480 /
// 1720; 1 of 131072, 64 rows 1790 / 225.  The constants fit 100 sizes; of 60 others, drawn, 3 take
// a form that is more than 5% behind the best one (1 of 3053 slots, 97 rows, 256/32 heads
// of 64: 72 and 62).  Several groups have to be faster by kSeveral: their rounds take as long
// for sequences that fill little of their page table, which streaming does not (32 of 1024
// in tables of 131072, 32 rows: 1028 / 116).
constexpr double kCallUs = 6., kCtaUs = 0.022, kReadUs = 0.9, kGroupUs = 10., kCutUs = 6., kLeastTileUs = 15.;
constexpr double kRecordUs = 0.1;  // per MB
constexpr double kSeveral = 0.85;
constexpr double stream_us(int d) { return d == 64 ? 0.33 : d == 96 ? 0.27 : 0.23; }  // per MB of codes and 16 columns
constexpr double tile_step_us(int d) { return d == 64 ? 1.4 : 1.9; }
// Rows read back at once, beyond one sequence.  Fewer and larger groups leave less of their
// last waves empty: 64 sequences of 2048 slots, 64 rows, up to 64 MB 467 us, 128 407, 256 386,
// 512 321 (57 and 7), all in one 313; 16 of 4096, 256 rows 439, 363, 350, 287 (weights in bf16).
constexpr size_t kGroupBytes = 512 << 20;
// Partial records held at once: as many sequences' as fit are joined together, and a
// sequence is cut into no more parts than fit (1 of 32048 slots, 2048 rows, 32/8 heads of 128,
// 7 parts 249 MB: 849 us, 890 whole).
constexpr size_t kRecordBytes = 256 << 20;

RowsPlan rows_plan(const wm_config& c, int32_t B, int32_t Tq, int32_t max_pages) {
  RowsPlan pl{};
  const int G = c.Hq / c.Hkv, sms = sm_count();
  const int64_t rows = (int64_t)Tq * G, slots = (int64_t)max_pages * c.page_size;
  if (c.dtype != WM_DT_BF16 || c.page_size < 8 || !tma_available()) return pl;
  if (slots * c.Hkv >= INT32_MAX || (int64_t)B * Tq >= INT32_MAX || rows >= INT32_MAX / 2) return pl;
  const size_t one = (size_t)slots * c.Hkv * c.d * 2 * 2;
  int64_t group = kGroupBytes / one;
  if (group > (INT32_MAX - 1) / (slots * c.Hkv)) group = (INT32_MAX - 1) / (slots * c.Hkv);
  group = group < 1 ? 1 : group > B ? B : group;
  const int64_t tiles = (slots + kTileSlots - 1) / kTileSlots;
  const double step = tile_step_us(c.d);
  // whole items: two heads of 128 rows, or one of 256; an item's start as one KV tile
  const int64_t items = G % 2 == 0 ? (int64_t)c.Hq / 2 * ((Tq + kTileRows - 1) / kTileRows)
                                   : (int64_t)c.Hq * ((Tq + 2 * kTileRows - 1) / (2 * kTileRows));
  auto whole = [&](int64_t n) { return (double)((n * items + sms - 1) / sms) * (double)(tiles + 1) * step; };
  auto all = [&](int64_t n) {
    return (double)(B / n) * (kGroupUs + whole(n)) + (B % n ? kGroupUs + whole(B % n) : 0.);
  };
  pl.group = (int)group;
  for (int64_t n = group - 1; group < B && n > group / 2; --n)  // (whichever fills the waves best)
    if (all(n) < all(pl.group)) pl.group = (int)n;
  // cut ones: the count of parts with the shortest last CTA, its start again as one KV tile
  pl.pair = rows <= kTileRows ? 1 : 0;
  pl.blocks = pl.pair ? 1 : (int)((rows + 2 * kTileRows - 1) / (2 * kTileRows));
  const int64_t units = (int64_t)pl.blocks * c.Hkv;
  const size_t part = sizeof(float) * (size_t)c.Hkv * rows * (pl.pair ? 2 : 1) * tile_rec(c.d);  // a part's records
  double least = 1e30, one_cut = 1e30;
  int splits = 1;
  for (int n = 1; n <= 32 && n <= tiles && part * n <= kRecordBytes; ++n) {
    const double us = step * ((double)((units * n + sms - 1) / sms) * ((double)((tiles + n - 1) / n) + 1.) + 0.05 * n);
    const double run = us > kLeastTileUs ? us : kLeastTileUs, join = kRecordUs * 1e-6 * (double)(part * n);
    if (run + 0.5 * join < least) {  // (half: of 62 MB of records a third gets to HBM)
      least = run + 0.5 * join;
      one_cut = run + join;
      splits = n;
    }
  }
  const double cut = kCutUs + pl.group * one_cut;
  pl.cut = cut < whole(pl.group);
  pl.splits = pl.cut ? splits : 1;
  const size_t most = kRecordBytes / (part * pl.splits);
  pl.joined = !pl.cut ? 0 : most < (size_t)pl.group ? (int)most : pl.group;
  const double mb = (double)B * slots * c.Hkv * (c.d + c.d / 8) * 1e-6, blocks = (double)((rows + 15) / 16);
  const double tensor = kReadUs * mb + (pl.cut ? (double)((B + pl.group - 1) / pl.group) * (kGroupUs + cut) : all(pl.group));
  const double stream = kCallUs + blocks * (mb * stream_us(c.d) + kCtaUs * B * c.Hkv);
  if (stream * (B > pl.group ? kSeveral : 1.) <= tensor) return pl;
  pl.tiles = true;
  pl.records = pl.splits * (pl.pair ? 2 : 1);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += align256(bytes);
    return at;
  };
  take(one / 2 * pl.group);
  pl.off_v = take(one / 2 * pl.group);
  pl.off_table = take(sizeof(int32_t) * (size_t)pl.group * max_pages);
  pl.off_last = take(sizeof(int32_t) * (size_t)pl.group);
  pl.off_lens = take(sizeof(int32_t) * (size_t)pl.group * Tq);
  pl.off_part = take(part * pl.splits * pl.joined);
  pl.total = off;
  return pl;
}

wm_status rows_on_tiles(const RowsPlan& pl, const wm_config& c, const wm_q4_cache& q4, int32_t layer, const void* q,
                        const int32_t* pos, const int32_t* page_table, int32_t B, int32_t Tq, int32_t max_pages,
                        void* out, char* ws, int32_t* dev_status, cudaStream_t s) {
  const int G = c.Hq / c.Hkv, chan = c.chan_of_layer[layer];
  int32_t* const table = (int32_t*)(ws + pl.off_table);
  int32_t* const last = (int32_t*)(ws + pl.off_last);
  int32_t* const lens = (int32_t*)(ws + pl.off_lens);
  float* const part = (float*)(ws + pl.off_part);
  const size_t row_elems = (size_t)Tq * c.Hq * c.d;
  for (int32_t b0 = 0; b0 < B; b0 += pl.group) {
    const int32_t n = B - b0 < pl.group ? B - b0 : pl.group;
    Q4RowsPrep prep{};
    prep.pos = pos + (size_t)b0 * Tq;
    prep.q4_table = page_table + (size_t)b0 * max_pages;
    prep.last = last;
    prep.lens = lens;
    prep.table = table;
    prep.Tq = Tq;
    prep.max_pages = max_pages;
    prep.P = c.page_size;
    prep.q4_pages = q4.num_pages;
    if (launch_q4_rows_prep(prep, n, s) != cudaSuccess) return WM_ERR_CUDA;
    Q4CopyParams r = copy_params(c, q4, n, max_pages, max_pages * c.page_size, dev_status);
    r.pool += chan * channel_bytes(c, q4.num_pages);
    r.k = 1;
    r.k_rows = ws;
    r.v_rows = ws + pl.off_v;
    r.q4_table = prep.q4_table;
    r.last = last;
    r.rows_at = kQ4Dense;
    r.row_pages = INT32_MAX;
    if (launch_q4_read(r, c.dtype, c.d, sm_count(), s) != cudaSuccess) return WM_ERR_CUDA;
    TileParams t{};
    t.status = dev_status;
    t.page_table = table;
    t.Hq = c.Hq;
    t.G = G;
    t.Hkv = c.Hkv;
    t.num_pages = n * max_pages;
    t.max_pages = max_pages;
    t.P = c.page_size;
    t.log2P = ilog2(c.page_size);
    t.qscale = (float)(1.4426950408889634 / sqrt((double)c.d));
    t.splits = pl.splits;
    t.v_half = 1;
    __nv_bfloat16* const o = (__nv_bfloat16*)out + b0 * row_elems;
    const __nv_bfloat16* const x = (const __nv_bfloat16*)q + b0 * row_elems;
    if (!pl.cut) {
      t.pos = prep.pos;
      t.out = o;
      t.rows = Tq;
      t.window = max_pages * c.page_size;
      t.pair = G % 2 == 0 ? 1 : 0;
      const int block = t.pair ? kTileRows : 2 * kTileRows;
      t.blocks = (Tq + block - 1) / block;
      t.items = n * (t.pair ? c.Hq / 2 : c.Hq) * t.blocks;
      const TileInputs in{x, ws, ws + pl.off_v, n, 1, c.d};
      if (launch_tile_attn(t, in, sm_count(), s) != cudaSuccess) return WM_ERR_CUDA;
      continue;
    }
    for (int32_t i = 0, first = 0; i < n; ++i) {  // first: of the sequences that are joined next
      t.pos = lens + (size_t)i * Tq;
      t.page_table = table + (size_t)i * max_pages;
      t.part = part + (size_t)(i - first) * c.Hkv * Tq * G * pl.records * tile_rec(c.d);
      t.rows = Tq * G;
      t.prefix_slots = max_pages * c.page_size;
      t.pair = pl.pair;
      t.records = pl.records;
      t.items = pl.blocks * c.Hkv * pl.splits;
      const TileInputs in{x + i * row_elems, ws, ws + pl.off_v, Tq, 1, c.d};
      if (launch_tile_attn(t, in, sm_count(), s) != cudaSuccess) return WM_ERR_CUDA;
      if (i + 1 < n && i + 1 - first < pl.joined) continue;
      const Q4RowsJoin j{part, o + first * row_elems, i + 1 - first, Tq, c.Hq, c.Hkv, G, pl.records};
      if (launch_q4_rows_join(j, c.d, s) != cudaSuccess) return WM_ERR_CUDA;
      first = i + 1;
    }
  }
  return WM_OK;
}

}  // namespace

extern "C" {

size_t wm_q4_cache_bytes(const wm_config* c, int32_t num_pages) {
  if (wm_config_check(c) != WM_OK || num_pages < 1) return 0;
  return align256(c->k * channel_bytes(*c, num_pages));
}

wm_status wm_q4_cache_alloc(const wm_config* c, void* dev_buf, size_t bytes, int32_t num_pages, wm_q4_cache* out) {
  wm_status st = wm_config_check(c);
  if (st != WM_OK) return st;
  if (!dev_buf || !out || num_pages < 1 || !aligned(dev_buf, 256)) return WM_ERR_INVALID_ARG;
  // (the padding behind the last channel is not read)
  if (bytes < c->k * channel_bytes(*c, num_pages)) return WM_ERR_INVALID_ARG;
  memset(out, 0, sizeof *out);
  out->pool = dev_buf;
  out->num_pages = num_pages;
  out->k = c->k;
  out->Hkv = c->Hkv;
  out->page_size = c->page_size;
  out->d = c->d;
  return WM_OK;
}

wm_status wm_q4_write(const wm_config* c, const wm_cache* cache, const int32_t* page_table, const wm_q4_cache* q4,
                      const int32_t* q4_table, const int32_t* first, const int32_t* last, int32_t span, int32_t B,
                      int32_t max_pages, int32_t* dev_status, void* stream) {
  return copy_ranges(true, c, cache, page_table, q4, q4_table, first, last, span, B, max_pages, dev_status, stream);
}

wm_status wm_q4_read(const wm_config* c, const wm_q4_cache* q4, const int32_t* q4_table, const wm_cache* cache,
                     const int32_t* page_table, const int32_t* first, const int32_t* last, int32_t span, int32_t B,
                     int32_t max_pages, int32_t* dev_status, void* stream) {
  return copy_ranges(false, c, cache, page_table, q4, q4_table, first, last, span, B, max_pages, dev_status, stream);
}

size_t wm_q4_kv_mix_workspace(const wm_config* c, int32_t B) {
  const size_t mix = wm_kv_mix_workspace(c, B);
  return mix == 0 ? 0 : mix + 2 * row_bytes(*c, B);
}

wm_status wm_q4_kv_mix(const wm_config* c, const wm_q4_cache* q4, const wm_mix_weights* w, const void* h,
                       const int32_t* page_table, const int32_t* slot, const int32_t* pos, int32_t B,
                       int32_t max_pages, void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream) {
  wm_status st = check_call(c, q4, B, max_pages);
  if (st != WM_OK) return st;
  if (!w) return WM_ERR_INVALID_ARG;
  if (B == 0) return WM_OK;
  if (!page_table || !workspace || ws_bytes < wm_q4_kv_mix_workspace(c, B)) return WM_ERR_INVALID_ARG;
  if ((int64_t)c->k * B * c->Hkv > INT32_MAX / 2) return WM_ERR_UNSUPPORTED;
  const size_t mix = wm_kv_mix_workspace(c, B), rows = row_bytes(*c, B);
  char* const ws = (char*)workspace;
  st = kv_mix_to_rows(c, w, h, slot, pos, B, max_pages * c->page_size, ws + mix, ws + mix + rows, workspace, mix,
                      dev_status, stream);
  if (st != WM_OK) return st;
  Q4CopyParams p = copy_params(*c, *q4, B, max_pages, 1, dev_status);
  p.k_rows = ws + mix;
  p.v_rows = ws + mix + rows;
  p.rows_at = kQ4Staged;
  p.row_pages = B;
  p.q4_table = page_table;
  p.first = slot;
  p.steps = 1;
  return cuda_status(launch_q4_write(p, c->dtype, c->d, sm_count(), (cudaStream_t)stream));
}

size_t wm_q4_decode_attn_workspace(const wm_config* c, int32_t B, int32_t max_pages) {
  if (wm_config_check(c) != WM_OK || B < 0 || max_pages < 1) return 0;
  return B == 0 ? 256 : attn_plan(*c, B, 1, max_pages).total;
}

wm_status wm_q4_decode_attn(const wm_config* c, const wm_q4_cache* q4, int32_t layer, const void* q,
                            const int32_t* page_table, const int32_t* seq_lens, int32_t B, int32_t max_pages,
                            void* out, void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream) {
  wm_status st = check_call(c, q4, B, max_pages);
  if (st != WM_OK) return st;
  if (layer < 0 || layer >= c->L) return WM_ERR_INVALID_ARG;
  if (B == 0) return WM_OK;
  if (B > kMaxBatch || (int64_t)B * c->Hq > INT32_MAX / 2) return WM_ERR_UNSUPPORTED;
  return attn(*c, *q4, layer, q, page_table, seq_lens, 0, B, 1, max_pages, out, workspace, ws_bytes, dev_status, stream);
}

size_t wm_q4_rows_attn_workspace(const wm_config* c, int32_t B, int32_t Tq, int32_t max_pages) {
  if (wm_config_check(c) != WM_OK || B < 0 || Tq < 0 || max_pages < 1) return 0;
  if (B == 0 || Tq == 0) return 256;
  const RowsPlan pl = rows_plan(*c, B, Tq, max_pages);
  return pl.tiles ? pl.total : attn_plan(*c, B, Tq, max_pages).total;
}

wm_status wm_q4_rows_attn(const wm_config* c, const wm_q4_cache* q4, int32_t layer, const void* q, const int32_t* pos,
                          const int32_t* page_table, int32_t B, int32_t Tq, int32_t max_pages, void* out,
                          void* workspace, size_t ws_bytes, int32_t* dev_status, void* stream) {
  wm_status st = check_call(c, q4, B, max_pages);
  if (st != WM_OK) return st;
  if (layer < 0 || layer >= c->L || Tq < 0) return WM_ERR_INVALID_ARG;
  if (B == 0 || Tq == 0) return WM_OK;
  if (B > kMaxBatch || (int64_t)B * Tq > INT32_MAX / 2 / c->Hq) return WM_ERR_UNSUPPORTED;
  const RowsPlan pl = rows_plan(*c, B, Tq, max_pages);
  if (pl.tiles) {
    if (!q || !pos || !page_table || !out || !workspace) return WM_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256) || ws_bytes < pl.total)
      return WM_ERR_INVALID_ARG;
    return rows_on_tiles(pl, *c, *q4, layer, q, pos, page_table, B, Tq, max_pages, out, (char*)workspace, dev_status,
                         (cudaStream_t)stream);
  }
  return attn(*c, *q4, layer, q, page_table, pos, 1, B, Tq, max_pages, out, workspace, ws_bytes, dev_status, stream);
}

}  // extern "C"
