// C ABI of the long-context operators (declared in include/wm.h): attention
// over a sliding window with sinks, over a shared prefix, decode attention
// that sums each slot's weight, and eviction by those sums.  Argument checks,
// work splits and kernel dispatch; all device memory belongs to the caller.
#include <math.h>

#include "api_util.h"
#include "common.cuh"
#include "internal.h"
#include "range_attn.h"
#include "wm.h"

namespace {

using namespace wm;

constexpr int kMaxBatch = 4096;

// Work a warp of a split launch is left with at least, in stages.
constexpr int kMinStagesPerWarp = 4;

int clamp_int(int64_t x, int64_t lo, int64_t hi) { return (int)(x < lo ? lo : x > hi ? hi : x); }

// CTAs per unit of a launch whose partial records a later kernel joins: enough
// for about `waves` waves of resident CTAs, so that sequences of unequal length
// still fill the SMs, while each warp keeps kMinStagesPerWarp stages.
int split_pieces(int64_t units, int64_t stages, int waves) {
  const int64_t by_work = stages / (kRangeWarps * kMinStagesPerWarp);
  const int64_t by_sms = ((int64_t)sm_count() * kRangeCtasPerSm * waves + units - 1) / units;
  return clamp_int(by_work < by_sms ? by_work : by_sms, 1, kMassMaxPieces);
}

int64_t stages_of(const wm_config& c, int64_t slots) {
  const int ss = range_stage_slots(c.dtype, c.d);
  return (slots + ss - 1) / ss;
}

// CTAs per unit (one cluster, joined on chip) of a launch that writes its
// outputs itself: as many as keep every CTA resident and leave each warp a stage.
int range_cluster(const wm_config& c, int64_t units, int64_t visible) {
  const int64_t stages = stages_of(c, visible) + 1;
  int C = 1;
  while (C < kRangeMaxCluster && units * C * 2 <= (int64_t)sm_count() * kRangeCtasPerSm &&
         (int64_t)C * kRangeWarps < stages)
    C *= 2;
  return C;
}

// Checks every attention call of this file makes.
wm_status check_attn(const wm_config* c, const wm_cache* cache, int32_t layer, int32_t B, int32_t max_pages) {
  wm_status st = wm_config_check(c);
  if (st != WM_OK) return st;
  if ((st = check_cache(*c, cache)) != WM_OK) return st;
  if (layer < 0 || layer >= c->L || B < 0 || max_pages < 1) return WM_ERR_INVALID_ARG;
  if ((int64_t)max_pages * c->page_size > INT32_MAX / 2) return WM_ERR_INVALID_ARG;
  // 32-bit cache rows per channel
  if ((int64_t)cache->num_pages * c->Hkv * c->page_size > INT32_MAX) return WM_ERR_UNSUPPORTED;
  return WM_OK;
}

RangeParams range_params(const wm_config& c, const wm_cache& cache, int32_t layer, const void* q,
                         const int32_t* page_table, const int32_t* lens, int32_t B, int32_t max_pages,
                         int32_t* dev_status) {
  const size_t chan = (size_t)c.chan_of_layer[layer] * cache.num_pages * c.Hkv * c.page_size * c.d * elem_size(c.dtype);
  RangeParams p{};
  p.k_pool = (const char*)cache.k_pool + chan;
  p.v_pool = (const char*)cache.v_pool + chan;
  p.q = q;
  p.page_table = page_table;
  p.seq_lens = lens;
  p.status = dev_status;
  p.B = B;
  p.Hq = c.Hq;
  p.Hkv = c.Hkv;
  p.G = c.Hq / c.Hkv;
  p.P = c.page_size;
  p.log2P = ilog2(c.page_size);
  p.num_pages = cache.num_pages;
  p.max_pages = max_pages;
  p.rows = p.G;
  p.pieces = 1;
  p.rows_per_seq = 1;
  p.qscale = (float)(1.4426950408889634 / sqrt((double)c.d));
  return p;
}

// The tensor-core kernel is built for bf16 and pages of at least 8 slots (a TMA
// box is a whole 8-row swizzle atom); its tensor maps take 32-bit rows over all
// channels.  Everything else runs on the range kernel.
bool tiles_ok(const wm_config& c, int32_t num_pages) {
  return c.dtype == WM_DT_BF16 && c.page_size >= 8 && tma_available() &&
         (int64_t)c.k * num_pages * c.Hkv * c.page_size < INT32_MAX;
}

TileParams tile_params(const wm_config& c, const wm_cache& cache, int32_t layer, const int32_t* page_table,
                       int32_t max_pages, int32_t* dev_status) {
  TileParams p{};
  p.page_table = page_table;
  p.status = dev_status;
  p.Hq = c.Hq;
  p.G = c.Hq / c.Hkv;
  p.Hkv = c.Hkv;
  p.chan = c.chan_of_layer[layer];
  p.num_pages = cache.num_pages;
  p.max_pages = max_pages;
  p.P = c.page_size;
  p.log2P = ilog2(c.page_size);
  p.splits = 1;
  p.qscale = (float)(1.4426950408889634 / sqrt((double)c.d));
  return p;
}

wm_status launch_tiles(const TileParams& p, const wm_config& c, const wm_cache& cache, const void* q, int32_t B,
                       void* stream) {
  const TileInputs in{q, cache.k_pool, cache.v_pool, B, c.k, c.d};
  const cudaError_t e = launch_tile_attn(p, in, sm_count(), (cudaStream_t)stream);
  if (e == cudaErrorInvalidValue) return WM_ERR_INVALID_ARG;  // the tensor-map encoder refused
  return e == cudaSuccess ? WM_OK : WM_ERR_CUDA;
}

// Split of a shared-prefix call and its workspace.  The prefix runs either on
// the tensor cores (row blocks of 256, or of 128 if there are no more, times
// `splits` parts of its KV tiles) or on the range kernel (groups of 8 rows,
// times prefix_pieces).
struct PrefixPlan {
  int blocks, pair, splits, records;  // tensor cores
  int groups, prefix_pieces;          // range kernel
  int suffix_cluster;
  size_t total;
};

// Which kernel reads the prefix.  The range kernel reads it once per 8 rows, from
// L2 after the first, and starts in about 5 us less; the tensor-core kernel reads
// it once.  Measured side by side (us per call, range / tensor): 4.7 MB of K/V
// and 8 rows 11.0 / 15.4, 37 MB and 8 rows 22.2 / 28.3, 5.9 MB and 16 rows 11.2 /
// 14.8, 5.9 MB and 32 rows 18.6 / 17.8, 49 MB and 16 rows 32.8 / 25.5, 134 MB and
// 8 rows 44.5 / 39.3.
constexpr int64_t kPrefixRangeBytes = 40 << 20;

bool prefix_on_tiles(const wm_config& c, int32_t num_pages, int32_t shared_pages, int groups) {
  const int64_t bytes = (int64_t)shared_pages * c.page_size * c.Hkv * c.d * 2 * (int64_t)elem_size(c.dtype);
  return tiles_ok(c, num_pages) && bytes * groups > kPrefixRangeBytes;
}

// Pieces of a unit of the range kernel's prefix: streaming takes time as
// stages / pieces, the join behind it as pieces, so about sqrt(stages) of them
// within the SMs' residency.  More than half the SMs' worth of CTAs keeps the
// suffix from starting beside them: then no more (bf16) than leave each warp 4
// stages.  Measured (us per call, 3 / 8 pieces): 16 sequences of 12 heads behind
// 1920 slots 11.3 / 12.5; 4 sequences of 3 heads behind 512 slots, 2 / 6 pieces,
// 9.4 / 8.0.
int prefix_pieces(const wm_config& c, int64_t units, int64_t slots) {
  const int64_t stages = stages_of(c, slots), sms = sm_count();
  int64_t n = (int64_t)(sqrt((double)stages) + 0.5);
  if (n > kRangeCtasPerSm * sms / units) n = kRangeCtasPerSm * sms / units;
  if (c.dtype == WM_DT_BF16 && 2 * units * n > sms) {
    const int64_t by_work = stages / (kRangeWarps * kMinStagesPerWarp), beside = sms / 2 / units;
    const int64_t most = by_work > beside ? by_work : beside;
    if (n > most) n = most;
  }
  return clamp_int(n, 1, 64);
}

// KV parts of the tensor-core prefix: the count with the shortest last CTA,
// counting a CTA's fixed cost as two KV tiles and each further record's join.
int prefix_splits(int64_t units, int64_t tiles, int sms) {
  int best = 1;
  double least = 1e30;
  for (int n = 1; n <= 64 && n <= tiles; ++n) {
    const double waves = (double)((units * n + sms - 1) / sms);
    const double cost = waves * ((double)((tiles + n - 1) / n) + 2.0) + 0.05 * n;
    if (cost < least) {
      least = cost;
      best = n;
    }
  }
  return best;
}

PrefixPlan prefix_plan(const wm_config& c, int32_t B, int32_t max_pages, int32_t shared_pages) {
  const int G = c.Hq / c.Hkv;
  PrefixPlan pl{};
  pl.groups = (int)(((int64_t)B * G + kRangeRows - 1) / kRangeRows);
  pl.prefix_pieces = prefix_pieces(c, (int64_t)pl.groups * c.Hkv, (int64_t)shared_pages * c.page_size);
  pl.suffix_cluster = range_cluster(c, (int64_t)B * c.Hkv, (int64_t)(max_pages - shared_pages) * c.page_size);
  const int64_t rows = (int64_t)B * G;
  pl.pair = rows <= kTileRows ? 1 : 0;
  pl.blocks = pl.pair ? 1 : (int)((rows + 2 * kTileRows - 1) / (2 * kTileRows));
  pl.splits = prefix_splits((int64_t)pl.blocks * c.Hkv,
                            ((int64_t)shared_pages * c.page_size + kTileSlots - 1) / kTileSlots, sm_count());
  pl.records = pl.splits * (pl.pair ? 2 : 1);
  const size_t tile_bytes = sizeof(float) * (size_t)c.Hkv * rows * pl.records * tile_rec(c.d);
  const size_t range_bytes =
      sizeof(float) * (size_t)pl.groups * c.Hkv * pl.prefix_pieces * range_rec(kRangeRows, c.d);
  // (room for either: which one runs depends on the cache too)
  pl.total = align256(tile_bytes > range_bytes ? tile_bytes : range_bytes);
  if (pl.total == 0) pl.total = 256;
  return pl;
}

// Split of a mass call.  Where a CTA's scores fit beside its ring without
// costing the SM its second CTA, one launch does it all (clusters join on chip
// and add their own slots' weights); else partial records and scores go through
// the workspace to a second kernel.
struct MassPlan {
  int cluster, mass_slots;  // one launch: CTAs per unit (0: two launches), slots per CTA
  int pieces;
  int64_t score_stride;
  size_t off_scores, total;
};
constexpr int kMassSmemBytes = 4096;

MassPlan mass_plan(const wm_config& c, int32_t B, int32_t max_pages) {
  const int G = c.Hq / c.Hkv;
  const int64_t slots = (int64_t)max_pages * c.page_size, units = (int64_t)B * c.Hkv;
  MassPlan pl{};
  const int64_t stages = stages_of(c, slots);
  const int C = range_cluster(c, units, slots);
  const int64_t per_cta = (stages + C * kRangeWarps - 1) / (C * kRangeWarps) * kRangeWarps * range_stage_slots(c.dtype, c.d);
  if (per_cta * G * (int64_t)sizeof(float) <= kMassSmemBytes) {
    pl.cluster = C;
    pl.mass_slots = (int)per_cta;
    pl.total = 256;
    return pl;
  }
  pl.pieces = split_pieces(units, stages, 6);
  pl.score_stride = (slots + 31) / 32 * 32;
  pl.off_scores = align256(sizeof(float) * (size_t)units * pl.pieces * range_rec(G, c.d));
  pl.total = pl.off_scores + align256(sizeof(float) * (size_t)units * G * pl.score_stride);
  return pl;
}

wm_status cuda_status(cudaError_t e) { return e == cudaSuccess ? WM_OK : WM_ERR_CUDA; }

}  // namespace

extern "C" {

wm_status wm_window_attn(const wm_config* c, const wm_cache* cache, int32_t layer, const void* q,
                         const int32_t* page_table, const int32_t* seq_lens, int32_t sinks, int32_t window,
                         int32_t B, int32_t max_pages, void* out, int32_t* dev_status, void* stream) {
  wm_status st = check_attn(c, cache, layer, B, max_pages);
  if (st != WM_OK) return st;
  if (sinks < 0 || window < 0) return WM_ERR_INVALID_ARG;
  if (B == 0) return WM_OK;
  if (B > kMaxBatch || (int64_t)B * c->Hq > INT32_MAX / 2) return WM_ERR_UNSUPPORTED;
  if (!q || !page_table || !seq_lens || !out) return WM_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16)) return WM_ERR_INVALID_ARG;
  const int64_t slots = (int64_t)max_pages * c->page_size, visible = (int64_t)sinks + window;
  RangeParams p = range_params(*c, *cache, layer, q, page_table, seq_lens, B, max_pages, dev_status);
  p.mode = kRangeWindow;
  p.out = out;
  p.sinks = sinks;
  p.window = window;
  p.pieces = range_cluster(*c, (int64_t)B * c->Hkv, visible < slots ? visible : slots);
  return cuda_status(launch_range_attn(p, c->dtype, c->d, B * c->Hkv, (cudaStream_t)stream));
}

wm_status wm_window_prefill_attn(const wm_config* c, const wm_cache* cache, int32_t layer, const void* q,
                                 const int32_t* pos, const int32_t* page_table, int32_t sinks, int32_t window,
                                 int32_t B, int32_t Tq, int32_t max_pages, void* out, int32_t* dev_status,
                                 void* stream) {
  wm_status st = check_attn(c, cache, layer, B, max_pages);
  if (st != WM_OK) return st;
  if (Tq < 0 || sinks < 0 || window < 0) return WM_ERR_INVALID_ARG;
  if (B == 0 || Tq == 0) return WM_OK;
  if ((int64_t)B * Tq > INT32_MAX / 2 / c->Hq) return WM_ERR_UNSUPPORTED;
  if (!q || !pos || !page_table || !out) return WM_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16)) return WM_ERR_INVALID_ARG;
  if (tiles_ok(*c, cache->num_pages)) {
    const int64_t slots = (int64_t)max_pages * c->page_size;
    TileParams t = tile_params(*c, *cache, layer, page_table, max_pages, dev_status);
    t.pos = pos;
    t.out = out;
    t.rows = Tq;
    t.sinks = (int32_t)(sinks < slots ? sinks : slots);
    t.window = (int32_t)(window < slots ? window : slots);
    t.pair = t.G % 2 == 0 ? 1 : 0;
    const int block = t.pair ? kTileRows : 2 * kTileRows;
    t.blocks = (Tq + block - 1) / block;
    t.items = B * (t.pair ? c->Hq / 2 : c->Hq) * t.blocks;
    return launch_tiles(t, *c, *cache, q, B, stream);
  }
  RangeParams p = range_params(*c, *cache, layer, q, page_table, pos, B * Tq, max_pages, dev_status);
  p.mode = kRangeWindow;
  p.out = out;
  p.sinks = sinks;
  p.window = window;
  p.rows_per_seq = Tq;
  p.len_add = 1;  // the query at position i sees slots up to i
  return cuda_status(launch_range_attn(p, c->dtype, c->d, B * Tq * c->Hkv, (cudaStream_t)stream));
}

size_t wm_prefix_attn_workspace(const wm_config* c, int32_t B, int32_t max_pages, int32_t shared_pages) {
  if (wm_config_check(c) != WM_OK || B < 0 || max_pages < 1 || shared_pages < 0 || shared_pages > max_pages) return 0;
  if (B == 0) return 256;
  return prefix_plan(*c, B, max_pages, shared_pages).total;
}

wm_status wm_prefix_attn(const wm_config* c, const wm_cache* cache, int32_t layer, const void* q,
                         const int32_t* page_table, const int32_t* seq_lens, int32_t shared_pages, int32_t B,
                         int32_t max_pages, void* out, void* workspace, size_t ws_bytes, int32_t* dev_status,
                         void* stream) {
  wm_status st = check_attn(c, cache, layer, B, max_pages);
  if (st != WM_OK) return st;
  if (shared_pages < 0 || shared_pages > max_pages) return WM_ERR_INVALID_ARG;
  if (B == 0) return WM_OK;
  if (B > kMaxBatch || (int64_t)B * c->Hq > INT32_MAX / 2) return WM_ERR_UNSUPPORTED;
  if (!q || !page_table || !seq_lens || !out || !workspace) return WM_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256)) return WM_ERR_INVALID_ARG;
  const PrefixPlan pl = prefix_plan(*c, B, max_pages, shared_pages);
  if (ws_bytes < pl.total) return WM_ERR_INVALID_ARG;
  RangeParams p = range_params(*c, *cache, layer, q, page_table, seq_lens, B, max_pages, dev_status);
  p.begin = shared_pages * c->page_size;
  const bool tiles = prefix_on_tiles(*c, cache->num_pages, shared_pages, pl.groups);
  if (shared_pages > 0 && tiles) {
    TileParams t = tile_params(*c, *cache, layer, page_table, max_pages, dev_status);
    t.pos = seq_lens;
    t.part = (float*)workspace;
    t.rows = B * p.G;
    t.prefix_slots = p.begin;
    t.pair = pl.pair;
    t.splits = pl.splits;
    t.records = pl.records;
    t.items = pl.blocks * c->Hkv * pl.splits;
    if ((st = launch_tiles(t, *c, *cache, q, B, stream)) != WM_OK) return st;
  } else if (shared_pages > 0) {  // every other form of the prefix
    p.part = (float*)workspace;
    p.mode = kRangePrefix;
    p.rows = kRangeRows;
    p.pieces = pl.prefix_pieces;
    if (launch_range_attn(p, c->dtype, c->d, pl.groups * c->Hkv, (cudaStream_t)stream) != cudaSuccess)
      return WM_ERR_CUDA;
  }
  p.part = nullptr;
  p.mode = kRangeSuffix;
  p.out = out;
  p.prefix = (const float*)workspace;
  p.records = shared_pages == 0 ? 0 : tiles ? pl.records : pl.prefix_pieces;
  p.tile_records = tiles ? 1 : 0;
  p.rows = p.G;
  p.pieces = pl.suffix_cluster;
  return cuda_status(launch_range_attn(p, c->dtype, c->d, B * c->Hkv, (cudaStream_t)stream));
}

size_t wm_decode_attn_mass_workspace(const wm_config* c, int32_t B, int32_t max_pages) {
  if (wm_config_check(c) != WM_OK || B < 0 || max_pages < 1) return 0;
  if (B == 0) return 256;
  return mass_plan(*c, B, max_pages).total;
}

wm_status wm_decode_attn_mass(const wm_config* c, const wm_cache* cache, int32_t layer, const void* q,
                              const int32_t* page_table, const int32_t* seq_lens, float* mass, int32_t B,
                              int32_t max_pages, void* out, void* workspace, size_t ws_bytes,
                              int32_t* dev_status, void* stream) {
  wm_status st = check_attn(c, cache, layer, B, max_pages);
  if (st != WM_OK) return st;
  if (B == 0) return WM_OK;
  if (B > kMaxBatch || (int64_t)B * c->Hq > INT32_MAX / 2) return WM_ERR_UNSUPPORTED;
  if (!q || !page_table || !seq_lens || !mass || !out || !workspace) return WM_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(mass, 4) || !aligned(workspace, 256)) return WM_ERR_INVALID_ARG;
  const MassPlan pl = mass_plan(*c, B, max_pages);
  if (ws_bytes < pl.total) return WM_ERR_INVALID_ARG;
  RangeParams p = range_params(*c, *cache, layer, q, page_table, seq_lens, B, max_pages, dev_status);
  p.mode = kRangeScores;
  const int32_t max_slots = max_pages * c->page_size;
  float* chan_mass = mass + (size_t)c->chan_of_layer[layer] * B * c->Hkv * max_slots;
  if (pl.cluster > 0) {
    p.out = out;
    p.mass = chan_mass;
    p.mass_slots = pl.mass_slots;
    p.pieces = pl.cluster;
    return cuda_status(launch_range_attn(p, c->dtype, c->d, B * c->Hkv, (cudaStream_t)stream));
  }
  p.pieces = pl.pieces;
  p.part = (float*)workspace;
  p.scores = (float*)((char*)workspace + pl.off_scores);
  p.score_stride = pl.score_stride;
  const cudaError_t e = launch_range_attn(p, c->dtype, c->d, B * c->Hkv, (cudaStream_t)stream);
  if (e != cudaSuccess) return WM_ERR_CUDA;
  MassParams m{};
  m.part = p.part;
  m.scores = p.scores;
  m.seq_lens = seq_lens;
  m.max_slots = max_slots;
  m.mass = chan_mass;
  m.out = out;
  m.score_stride = pl.score_stride;
  m.B = B;
  m.Hq = c->Hq;
  m.Hkv = c->Hkv;
  m.G = p.G;
  m.pieces = pl.pieces;
  return cuda_status(launch_mass_add(m, c->dtype, c->d, (cudaStream_t)stream));
}

wm_status wm_cache_evict(const wm_config* c, const wm_cache* cache, const float* mass, float* mass_out,
                         const int32_t* page_table, const int32_t* seq_lens, int32_t budget, int32_t sinks,
                         int32_t recent, int32_t B, int32_t max_pages, int32_t* kept, int32_t* new_lens,
                         int32_t* dev_status, void* stream) {
  wm_status st = check_attn(c, cache, 0, B, max_pages);
  if (st != WM_OK) return st;
  if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget) return WM_ERR_INVALID_ARG;
  if (budget > max_pages * c->page_size) return WM_ERR_INVALID_ARG;
  if (B == 0) return WM_OK;
  if ((int64_t)c->k * B * c->Hkv > INT32_MAX / 8) return WM_ERR_UNSUPPORTED;
  // 32-bit cache rows over all channels
  if ((int64_t)c->k * cache->num_pages * c->Hkv * c->page_size > INT32_MAX) return WM_ERR_UNSUPPORTED;
  if (!mass || !mass_out || !page_table || !seq_lens || !kept || !new_lens) return WM_ERR_INVALID_ARG;
  if (!aligned(mass, 4) || !aligned(mass_out, 4) || new_lens == seq_lens) return WM_ERR_INVALID_ARG;
  EvictParams p{};
  p.k_pool = cache->k_pool;
  p.v_pool = cache->v_pool;
  p.mass = mass;
  p.mass_out = mass_out;
  p.page_table = page_table;
  p.seq_lens = seq_lens;
  p.kept = kept;
  p.new_lens = new_lens;
  p.status = dev_status;
  p.B = B;
  p.k = c->k;
  p.Hkv = c->Hkv;
  p.P = c->page_size;
  p.log2P = ilog2(c->page_size);
  p.num_pages = cache->num_pages;
  p.max_pages = max_pages;
  p.budget = budget;
  p.sinks = sinks;
  p.recent = recent;
  return cuda_status(launch_cache_evict(p, c->dtype, c->d, sm_count(), (cudaStream_t)stream));
}

}  // extern "C"
