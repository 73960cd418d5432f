// The 4-bit paged cache: layout and launch interfaces (q4_copy.cu, q4_attn.cuh).
//
// A row of d elements (a key or a value of one slot and kv head) is d signed
// 4-bit floats and a scale per 16 of them; value = code * scale.
//   code    bit 3 the sign, bits 2-0 the magnitude 0, 0.5, 1, 1.5, 2, 3, 4 or 6
//   scale   8 bits, 5 of exponent and 3 of mantissa: the fp16 of bits byte << 7,
//           so 2^-17 .. 10240; 0xFF (NaN) for 16 elements that are not all finite
// The scale is the nearest one (ties to even) to the largest magnitude of the 16
// over 6, each code the nearest (ties to even) to its element over the scale.  A
// code has 2 significant bits and a scale 4, so every value is exact in fp16 and in
// bf16, whatever the element type the row came from.
//
// Slots are held in tiles of n = min(page_size, 16): codes of the K rows [n][d/2]
// (element 2 i in the low half of byte i), codes of the V rows, scales of the K rows
// [n][d/16], scales of the V rows, padded to 16 bytes.  So 16 slots (or a small
// page) of one head are one contiguous piece (2304 bytes for d = 128) that one bulk
// copy fetches, 9/32 of the bf16 cache's bytes.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "wm.h"

namespace wm {

constexpr int kQ4Group = 16;       // elements that share a scale
constexpr int kQ4Step = 16;        // slots of a whole tile
constexpr int kQ4MaxScale = 226;   // byte of 10240: 6 * 10240 is below the largest fp16

inline int q4_tile_slots(int page_size) { return page_size < kQ4Step ? page_size : kQ4Step; }
inline int64_t q4_tile_bytes(int page_size, int d) {
  return ((int64_t)q4_tile_slots(page_size) * 2 * (d / 2 + d / kQ4Group) + 15) / 16 * 16;
}
inline int64_t q4_page_bytes(int page_size, int d) {  // of one kv head
  return page_size / q4_tile_slots(page_size) * q4_tile_bytes(page_size, d);
}

// Where the rows of a copy are.
enum Q4Rows : int32_t {
  kQ4Paged = 0,   // a cache, through row_table
  kQ4Staged = 1,  // [k][B][Hkv][d]: one row per sequence, of its slot `first`
  kQ4Dense = 2    // one channel, pages b * max_pages + t / page_size (bf16: V as fp16)
};

struct Q4CopyParams {
  void* k_rows;               // rows of the element type
  void* v_rows;
  uint8_t* pool;              // 4-bit pool (read: of the first channel copied)
  const int32_t* row_table;   // [B][max_pages] (kQ4Paged)
  const int32_t* q4_table;    // [B][max_pages]
  const int32_t* first;       // [B]: slots first .. last - 1 (NULL: from 0)
  const int32_t* last;        // [B] (NULL: one slot, `first`, at least slot 1)
  int32_t* status;
  int64_t page_bytes;         // of one kv head
  int32_t rows_at;            // Q4Rows
  int32_t B, k, Hkv, P, log2P, tile, log2tile, tile_bytes, row_pages, q4_pages, max_pages;
  int32_t span;               // slots of a range at most
  int32_t steps;              // tiles of 16 slots that a range touches at most
  int32_t wide, heads, items; // set by the launch: rows are 32-byte aligned, kv heads per
                              // item, items
};
cudaError_t launch_q4_write(const Q4CopyParams& p, int dtype, int d, int sms, cudaStream_t s);
cudaError_t launch_q4_read(const Q4CopyParams& p, int dtype, int d, int sms, cudaStream_t s);

// Many rows (bf16): a group of sequences is read back into the workspace and runs on
// the tensor-core kernel of range_attn.h.  V as fp16, in which it is exact as well: the
// weights then enter its product with 11 bits, as in the streaming kernel, and not 8.
struct Q4RowsPrep {
  const int32_t* pos;         // [B][Tq]
  const int32_t* q4_table;    // [B][max_pages]
  int32_t* last;              // [B]: slots that some row sees
  int32_t* lens;              // [B][Tq]: slots that each row sees, -1 for a bad position
  int32_t* table;             // [B][max_pages]: pages of the rows in the workspace (-1: none)
  int32_t Tq, max_pages, P, q4_pages;
};
cudaError_t launch_q4_rows_prep(const Q4RowsPrep& p, int B, cudaStream_t s);

struct Q4RowsJoin {
  const float* part;          // [B][Hkv][Tq * G][records][tile_rec(d)]
  void* out;                  // [B][Tq][Hq][d]
  int32_t B, Tq, Hq, Hkv, G, records;
};
cudaError_t launch_q4_rows_join(const Q4RowsJoin& p, int d, cudaStream_t s);

// ------------------------------------------------------------ attention
constexpr int kQ4Warps = 4;        // warps per CTA
constexpr int kQ4Slots = 32;       // slots of a warp's step
constexpr int kQ4MaxCluster = 8;
constexpr int kQ4MinSteps = 1;     // steps of a warp at least where all steps are spread
// Resident CTAs per SM, by registers.  (fp32 parts among the columns, 16 x 8192 slots of 32
// heads of 128: 3 CTAs 97 us, 2 108, 4 with the tiles of a step one by one 109.)
constexpr int q4_ctas_per_sm(bool bf16, int nb, bool fold) { return fold ? 3 : bf16 && nb == 1 ? 4 : 2; }
constexpr int kQ4MaxCtas = 4;      // the most of q4_ctas_per_sm
constexpr int kQ4Fold = 2;         // fp32: columns of a unit up to which their parts are columns

struct Q4AttnParams {
  const uint8_t* pool;        // channel base
  const void* q;              // [B][Tq][Hq][d]
  void* out;
  const int32_t* page_table;  // [B][max_pages]
  const int32_t* lens;        // [B][Tq]: the row sees slots t < lens + len_add
  int32_t* status;
  float* part;                // not NULL: all steps are spread over `pieces` CTAs, records
                              // [pieces][2][q4_rec] of shared units are joined by a second kernel
  int32_t len_add;
  int32_t B, Tq, Hq, Hkv, G, P, log2P, tile, log2tile, tile_bytes, num_pages, max_pages;
  int32_t col_blocks;         // units per (sequence, kv head): groups of 8 NB (row, head) columns
  int32_t nb;                 // NB
  int32_t pieces;             // CTAs per unit (one cluster), or of the spread
  float qscale;               // log2(e) / sqrt(d)
};
// floats of a partial record: cols x d unnormalised outputs, (reference, sum) per column
constexpr int q4_rec(int cols, int d) { return cols * (d + 2); }
cudaError_t launch_q4_attn(const Q4AttnParams& p, int dtype, int d, cudaStream_t s);

}  // namespace wm
