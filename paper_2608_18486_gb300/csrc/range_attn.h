// Launch interface of the attention over part of a sequence's slots: sliding
// windows with sinks, shared prefixes and their suffixes, and decode attention
// that keeps its scores (range_attn.cuh, range_attn.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "wm.h"

namespace wm {

// What a unit (one group of query rows that read the same K/V rows) covers.
enum RangeMode : int32_t {
  kRangeWindow = 0,  // (sequence, kv head): the sinks and the window, written to out
  kRangeSuffix = 1,  // (sequence, kv head): slots begin .. S-1, joined with the
                     // prefix's records and written to out
  kRangePrefix = 2,  // (8 query rows of any sequences, kv head): slots 0 .. begin-1 of
                     // sequence 0's pages, partial records
  kRangeScores = 3   // (sequence, kv head): every slot; partial records and scores, or
                     // (mass != NULL) out and the weights added to mass
};

constexpr int kRangeRows = 8;        // most query rows of a unit
constexpr int kRangeWarps = 4;       // warps per CTA
constexpr int kRangeMaxCluster = 8;
constexpr int kRangeMaxRecords = 128;  // most records of a shared prefix per row

struct RangeParams {
  const void* k_pool;         // channel base of the K pool
  const void* v_pool;
  const void* q;              // [B][Hq][d]
  void* out;                  // [B][Hq][d] (kRangeWindow)
  const int32_t* page_table;  // [B][max_pages]
  const int32_t* seq_lens;    // [B]
  int32_t* status;
  const float* prefix;        // kRangeSuffix: records of the shared prefix, tile_rec or
                              // range_rec (8 rows) ones
  int32_t records, tile_records;  // of them per row (0: no prefix), and their layout
  float* mass;                // [units][max_slots] of the channel, or NULL
  int32_t mass_slots;         // mass: most slots of one CTA
  float* part;                // [units][pieces][range_rec(rows, d)]
  float* scores;              // [units][G][score_stride] log2-scaled scores (kRangeScores)
  int64_t score_stride;
  int32_t mode, B, Hq, Hkv, G, P, log2P, num_pages, max_pages;
  int32_t rows_per_seq;       // "sequences" per page-table row (many query positions of one), 1 for decode
  int32_t len_add;            // slots of sequence b: seq_lens[b] + len_add
  int32_t sinks, window;      // kRangeWindow
  int32_t begin;              // kRangeSuffix / kRangePrefix: slots in the shared prefix
  int32_t rows;               // query rows per unit: G, or kRangeRows for kRangePrefix
  int32_t pieces;             // CTAs per unit
  float qscale;               // log2(e) / sqrt(d)
};

// floats of a partial record of the tile kernel: d outputs, (max, sum), padded
// to 32 bytes
constexpr int tile_rec(int d) { return d + 8; }
// floats of one partial record: rows x d unnormalised outputs, then (max, sum)
// per row in log2 units, padded to 16 bytes
constexpr int range_rec(int rows, int d) { return rows * d + (2 * rows + 3) / 4 * 4; }

// Slots of one pipeline stage (the grain the planner splits by).
int range_stage_slots(int dtype, int d);
// CTAs of the kernel that fit one SM (the planner's unit of residency).
constexpr int kRangeCtasPerSm = 2;
cudaError_t launch_range_attn(const RangeParams& p, int dtype, int d, int units, cudaStream_t s);

// Joins the partial records of kRangeScores and adds the weights to mass.
struct MassParams {
  const float* part;     // [B][Hkv][pieces][range_rec(G, d)]
  const float* scores;   // [B][Hkv][G][score_stride]
  const int32_t* seq_lens;
  float* mass;           // [B][Hkv][max_slots], the call's channel
  void* out;             // [B][Hq][d]
  int64_t score_stride;
  int32_t B, Hq, Hkv, G, pieces, max_slots;
  int32_t vec4;          // rows of mass are 16-byte aligned (set by the launch)
};
constexpr int kMassMaxPieces = 64;
cudaError_t launch_mass_add(MassParams p, int dtype, int d, cudaStream_t s);

// Tensor-core attention of many rows (tile_attn.cu; bf16, pages of >= 8 slots):
// under a window with sinks (part == NULL), or over a shared prefix into
// partial records.
struct TileParams {
  const int32_t* pos;         // window: [B][rows] positions; prefix: [B] lengths
  const int32_t* page_table;  // [B][max_pages]
  void* out;                  // window: [B][rows][Hq][d]
  float* part;                // prefix: [Hkv][rows][records][tile_rec(d)]
  int32_t* status;
  int32_t rows;               // window: query positions per sequence; prefix: B * G
  int32_t Hq, G, Hkv, chan, num_pages, max_pages, P, log2P;
  int32_t sinks, window;      // at most the page table's slots
  int32_t prefix_slots;
  int32_t pair;               // window: the two tiles are query heads h, h + 1 of the same
                              // rows; prefix: they are the even and odd KV tiles of one
  int32_t splits;             // prefix: parts of the KV tiles
  int32_t records;            // prefix: partial records per row
  int32_t blocks;             // window: row blocks per head
  int32_t items;
  int32_t wide_out;           // out is 32-byte aligned
  int32_t v_half;             // the V pool holds fp16, and the weights enter P V as fp16
  float qscale;               // log2(e) / sqrt(d)
};
struct TileInputs {
  const void* q;
  const void* k_pool;         // whole pools, all channels
  const void* v_pool;
  int32_t B, k, d;
};
constexpr int kTileRows = 128;
constexpr int kTileSlots = 128;
cudaError_t launch_tile_attn(TileParams p, const TileInputs& in, int sms, cudaStream_t s);
// 3-D map of a bf16 array [n2][n1][n0], boxes of 64 x box1 x box2 elements,
// 128-byte swizzle (rows of a box are its (n2, n1) pairs in order).
bool tma_map_bf16_3d(void* tm, const void* ptr, uint64_t n2, uint64_t n1, uint64_t n0, uint32_t box2, uint32_t box1);

// Cache eviction (evict.cu).
struct EvictParams {
  void* k_pool;               // whole pools: [k][num_pages][Hkv][P][d]
  void* v_pool;
  const float* mass;          // [k][B][Hkv][max_slots]
  float* mass_out;
  const int32_t* page_table;
  const int32_t* seq_lens;
  int32_t* kept;              // [k][B][Hkv][budget]
  int32_t* new_lens;
  int32_t* status;
  int32_t B, k, Hkv, P, log2P, num_pages, max_pages, budget, sinks, recent;
  int32_t cluster, vec4;      // set by the launch: CTAs per unit; sums may be read 16 bytes at a time
};
cudaError_t launch_cache_evict(EvictParams p, int dtype, int d, int sms, cudaStream_t s);

}  // namespace wm
