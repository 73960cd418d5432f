#pragma once
// Attention of a few query rows over a cache held in 4 bits (layout in q4.h):
// decode attention, and several positions per sequence at once.
//
//   out_c = sum_t p_ct v_t,  p_ct = 2^(x_ct - m_c) / l_c,  x_ct = (q_c . k_t) log2(e) / sqrt(d)
//   over the slots t below column c's limit.  A column is one (row, query head) pair
//   that reads a kv head; sums (m, l, sum_t 2^(x - m) v_t) of disjoint slot sets
//   join for any references m.
//
// A unit is one (sequence, kv head) and 8 NB of its columns.  `pieces` CTAs of 4
// warps share a unit; each warp takes a contiguous part of its steps of 32 slots
// through a private ring of cp.async copies, whose issue costs all lanes less than that of
// bulk copies (addresses in uniform registers: lane by lane).
//
// Both products are mma.sync m16n8k16 with the 8 columns as the narrow operand:
//   S^T [16 slots x 8 columns] += K [16 x d] Q^T,   O^T [d x 8] += V^T [d x 16] P^T,
// so 16 slots cost d / 8 of them for up to 8 columns.  The values of the cache are exact
// in fp16: a pair of codes becomes an fp16 pair in one conversion and one product
// with the scale.  For S^T a lane takes consecutive features of one slot, for O^T the same
// features of two slots, whose codes are first interleaved (byte = feature, halves =
// slots).  P^T is the transpose of S^T's accumulators: movmatrix.
//  * bf16: the columns' queries are scaled by a power of two so that they keep all
//    8 bits in fp16; P is rounded to fp16 (11 bits) against a reference 2^8 below
//    the running maximum, so that weights down to 2^-22 of the largest keep
//    them, and the reference moves only when a score passes it by 2^15.
//  * fp32: queries in three fp16 parts and P in two, beside each other among the
//    columns where there is room (see Fill); each feature block's products start at zero
//    and are added with rounding, since a matrix instruction truncates its sums.
// Bound by HBM and, just below it, by instruction issue: 16 slots of a head of 128 are 2304
// bytes and 250 (one column) to 268 instructions, 66 of them conversions; four warps
// per scheduler issue 60 to 64% of the time.  Measured: 32 sequences of 4096 to 8192 slots, 32
// heads of 128: 150 us, 6.0 TB/s of codes (the copies alone, without the products, 136); 8
// of 70001 to 131072, 32/8 heads: 153 us.  Two tiles of 16 slots per step: one, with more
// CTAs, 202 against 169 us.  4 CTAs per SM at 128 registers: 5 at 96, 171 against 162;
// CTAs of 8 warps 165 against 161; three steps in a ring 172 against 169.
#include <cooperative_groups.h>
#include <float.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "q4.h"

namespace wm {
namespace q4_detail {

namespace cg = cooperative_groups;

constexpr int kThreads = kQ4Warps * 32;
constexpr int kSlots = kQ4Slots, kTiles = kSlots / kQ4Step;
constexpr int kStages = 2;         // ring depth per warp, in steps
constexpr float kHead = 8.f;       // log2 of the weight of a new reference maximum
constexpr float kRaise = 15.f;     // log2 of the weight that moves the reference
constexpr unsigned FULL = 0xFFFFFFFFu;

template <int HD>
struct Shape {
  static constexpr int KW = HD / 32;                 // words of 8 codes per lane and K row
  static constexpr int MT = HD / 16;                 // 16-feature blocks
  static constexpr int BYTES16 = 16 * (HD + HD / 8);  // of 16 slots
  // pages of 1 or 2 slots: each tile is padded to 16 bytes
  static constexpr int PADDED16 = 16 * ((HD + HD / 8 + 15) / 16 * 16);
  template <int LT>
  static constexpr int tile() { return BYTES16 >> (4 - LT); }
};
template <typename T>
struct Parts {
  static constexpr int Q = sizeof(T) == 4 ? 3 : 1, P = sizeof(T) == 4 ? 2 : 1;
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The 8 x 8 matrix of 16-bit elements, row lane / 4, columns 2 (lane % 4) + {0, 1}, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(dst),
      "l"(src), "r"((int)on)
      : "memory");
}
// A whole tile, 16 bytes per lane and copy (dst and src at the lane's first); at < 0: none.
// One statement, so that its predicates are made once.
template <int HD>
__device__ __forceinline__ void cp_async_tile(uint32_t dst, const void* src, int at, int lane) {
  constexpr int REST = 16 * (HD + HD / 8) / 16 % 32;  // lanes of the last copy
  static_assert(HD == 64 || HD == 96 || HD == 128, "72, 108 or 144 chunks");
#define WM_Q4_CP(N) "@p cp.async.cg.shared.global [%0 + " #N "], [%1 + " #N "], 16;\n\t"
#define WM_Q4_CP_LAST(N) "@q cp.async.cg.shared.global [%0 + " #N "], [%1 + " #N "], 16;\n\t}"
#define WM_Q4_CP_PRED \
  "{\n\t.reg .pred p, q;\n\tsetp.ge.s32 p, %2, 0;\n\tsetp.lt.and.s32 q, %3, %4, p;\n\t"
  if constexpr (HD == 64)
    asm volatile(WM_Q4_CP_PRED WM_Q4_CP(0) WM_Q4_CP(512) WM_Q4_CP_LAST(1024) ::"r"(dst), "l"(src), "r"(at), "r"(lane),
                 "n"(REST)
                 : "memory");
  else if constexpr (HD == 96)
    asm volatile(WM_Q4_CP_PRED WM_Q4_CP(0) WM_Q4_CP(512) WM_Q4_CP(1024) WM_Q4_CP_LAST(1536) ::"r"(dst), "l"(src),
                 "r"(at), "r"(lane), "n"(REST)
                 : "memory");
  else
    asm volatile(WM_Q4_CP_PRED WM_Q4_CP(0) WM_Q4_CP(512) WM_Q4_CP(1024) WM_Q4_CP(1536) WM_Q4_CP_LAST(2048) ::"r"(dst),
                 "l"(src), "r"(at), "r"(lane), "n"(REST)
                 : "memory");
#undef WM_Q4_CP
#undef WM_Q4_CP_LAST
#undef WM_Q4_CP_PRED
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// The four bytes of w, two codes each, to fp16 pairs (low half first).
__device__ __forceinline__ void codes4(uint32_t w, uint32_t (&r)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "r"(w));
}
__device__ __forceinline__ uint32_t times(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 floats_of(uint32_t h) {
  float2 f;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}"
      : "=f"(f.x), "=f"(f.y)
      : "r"(h));
  return f;
}
// Two neighbouring fp16 of the parts: hi + mid + lo = x to 2^-33 of the largest |x|.
template <int N>
__device__ __forceinline__ void split(float x, float y, uint32_t (&part)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    part[i] = half2_of(x, y);
    if (i + 1 < N) {
      const float2 f = floats_of(part[i]);
      x -= f.x;
      y -= f.y;
    }
  }
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The reference below a largest score x.  Past 2^27 the difference may be rounded to 16,
// and 2^16 is no fp16: the score itself then.
__device__ __forceinline__ float below(float x) {
  const float y = __fsub_rn(x, kHead);
  return __fsub_rn(x, y) > kRaise ? x : y;
}

// First of the two neighbouring features of accumulator block m of lane row g.
template <int HD>
__device__ __forceinline__ int feature(int g, int m) {
  if (HD == 128) return 16 * g + 2 * m;
  if (HD == 64 || m < 4) return 8 * g + 2 * m;
  return 64 + 4 * g + 2 * (m - 4);
}

// What the eight columns of the products hold:
//  * kColumns: the unit's columns.
//  * kOne (bf16, one column): its query fills all eight of S^T's, column n with zeros but
//    for the features of scale group n, so that the product leaves one sum per group:
//    the scales of K then cost two products per slot and lane instead of one per pair
//    of codes (32 x 8192 slots, 32 heads of 128: 151 us against 153).  In O^T's all
//    columns are the same.
//  * kFold (fp32, up to two columns): column 4 i + n the n-th part of column i's query, and of
//    its weights, so that a product is one instruction and not three or two (16 x 8192
//    slots, 32 heads of 128: 97 us against 137).
enum Fill { kColumns, kOne, kFold };
// LT: log2 of a tile's slots, 2 to 4, or 0 for tiles of 1 or 2 slots.
// One warp's columns.  Lane: g = lane / 4, c = lane % 4.
template <typename T, int HD, int NB, int LT, Fill FILL>
struct Math {
  using SH = Shape<HD>;
  static constexpr bool ONE = FILL == kOne, FOLD = FILL == kFold;
  static constexpr bool EXACT = sizeof(T) == 4;  // products start at zero and are added with rounding
  static constexpr int NQ = FOLD ? 1 : Parts<T>::Q, NP = FOLD ? 1 : Parts<T>::P;
  uint32_t q[NB][NQ][SH::MT][2];  // column g: features (HD / 4) c + 8 w + 4 u + {0, 1}, {2, 3} at [2 w + u]
  float o[NB][SH::MT][4];         // features feature(g, m) (+ 1), columns 2 c, 2 c + 1
  float ref[NB][2], l[NB][2];     // columns 2 c, 2 c + 1; l: this lane's slots only
  float mul[NB][2];               // accumulator to score
  int lim[NB][2];

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int m = 0; m < SH::MT; ++m) o[n][m][0] = o[n][m][1] = o[n][m][2] = o[n][m][3] = 0.f;
      ref[n][0] = ref[n][1] = -FLT_MAX;
      l[n][0] = l[n][1] = 0.f;
    }
  }

  // Column g of block n: row (NULL: none) and limit.
  __device__ __forceinline__ void load(int n, const T* row, int limit, int lane, float qscale) {
    const int c = lane & 3;
    float x[HD / 4], top = 0.f;
#pragma unroll
    for (int i = 0; i < HD / 4; i += 16 / (int)sizeof(T)) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (row) v = __ldcg(reinterpret_cast<const uint4*>(row + HD / 4 * c + i));
      Elem<T>::unpack(v, x + i);
    }
#pragma unroll
    for (int i = 0; i < HD / 4; ++i) top = fmaxf(top, fabsf(x[i]));
    top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
    top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
    // largest magnitude to [2^14, 2^15): an exact product, undone by `mul`
    const int field = min(268 - (int)(__float_as_uint(top) >> 23), 253);
    const float up = __uint_as_float((uint32_t)field << 23);
#pragma unroll
    for (int j = 0; j < SH::MT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t part[Parts<T>::Q];
        split(x[4 * j + 2 * i] * up, x[4 * j + 2 * i + 1] * up, part);
        if constexpr (FOLD) {
          const int y = (lane >> 2) & 3;
          part[0] = y == 0 ? part[0] : y == 1 ? part[1] : y == 2 ? part[2] : 0u;
        }
        if (ONE && ((HD / 4 * c + 4 * j) >> 4) != lane >> 2) part[0] = 0u;
#pragma unroll
        for (int y = 0; y < NQ; ++y) q[n][y][j][i] = part[y];
      }
    const float down = qscale * __uint_as_float((uint32_t)(254 - field) << 23);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int from = FOLD ? 16 * (c >> 1) : 4 * (2 * c + i);  // a lane of that column
      mul[n][i] = __shfl_sync(FULL, down, from);
      lim[n][i] = __shfl_sync(FULL, limit, from);
    }
  }

  // Offsets of this lane's slots in a tile (or 16 slots of small pages): codes and
  // scales of K rows g, g + 8 and of V rows 2 c, 2 c + 1, 2 c + 8, 2 c + 9.
  struct At {
    static constexpr int N = LT > 0 ? 1 : 4;
    uint32_t k_[N], ks_[N], v_[N], vs_[N];
    // from a slot to the one 8 further on, codes (PER = HD / 2) or scales (HD / 16)
    static constexpr uint32_t eight(int per) { return LT == 4 ? 8 * per : (8 >> LT) * SH::template tile<LT>(); }
    __device__ __forceinline__ uint32_t k(int i) const { return LT > 0 ? k_[0] + i * eight(HD / 2) : k_[i]; }
    __device__ __forceinline__ uint32_t ks(int i) const { return LT > 0 ? ks_[0] + i * eight(HD / kQ4Group) : ks_[i]; }
    __device__ __forceinline__ uint32_t v(int i) const {
      return LT > 0 ? v_[0] + (i & 1) * (HD / 2) + (i >> 1) * eight(HD / 2) : v_[i];
    }
    __device__ __forceinline__ uint32_t vs(int i) const {
      return LT > 0 ? vs_[0] + (i & 1) * (HD / kQ4Group) + (i >> 1) * eight(HD / kQ4Group) : vs_[i];
    }
  };
  __device__ __forceinline__ static At offsets(int log2tile, int tile_bytes, int lane) {
    const int g = lane >> 2, c = lane & 3;
    At a;
    auto put = [&](int slot, int X, uint32_t& codes, uint32_t& scales) {
      const int l2 = LT > 0 ? LT : log2tile, n = 1 << l2, r = X * n + (slot & (n - 1));
      const uint32_t base = (uint32_t)(slot >> l2) * (LT > 0 ? SH::template tile<LT>() : tile_bytes);
      codes = base + r * (HD / 2) + (X ? (HD == 128 ? 8 * g : 4 * g) : HD / 8 * c);
      scales = base + n * HD + r * (HD / kQ4Group) +
               (X ? (HD == 128 ? g : g >> 1) : ONE ? min(2 * c, HD / kQ4Group - 2) : HD == 128 ? 2 * c : HD == 64 ? c : (3 * c) >> 1);
    };
#pragma unroll
    for (int i = 0; i < (LT > 0 ? 1 : 2); ++i) put(g + 8 * i, 0, a.k_[i], a.ks_[i]);
#pragma unroll
    for (int i = 0; i < (LT > 0 ? 1 : 4); ++i) put(2 * c + (i & 1) + 8 * (i >> 1), 1, a.v_[i], a.vs_[i]);
    return a;
  }

  // The lane's codes of K row g + 8 i.
  __device__ __forceinline__ static void load_codes(const unsigned char* a, uint32_t (&w)[SH::KW]) {
    if constexpr (HD == 128) {
      const uint4 v = *reinterpret_cast<const uint4*>(a);
      w[0] = v.x;
      w[1] = v.y;
      w[2] = v.z;
      w[3] = v.w;
    } else if constexpr (HD == 64) {
      const uint2 v = *reinterpret_cast<const uint2*>(a);
      w[0] = v.x;
      w[1] = v.y;
    } else {
#pragma unroll
      for (int i = 0; i < SH::KW; ++i) w[i] = reinterpret_cast<const uint32_t*>(a)[i];
    }
  }

  // ONE: scores of slots g and g + 8 of the 16 at st, in all four lanes of a slot.
  __device__ __forceinline__ void scores_one(const unsigned char* st, const At& at, float (&s)[2]) {
    uint32_t kw[2][SH::KW];
    float z[4] = {0.f, 0.f, 0.f, 0.f};  // slots g, g + 8; groups 2 c, 2 c + 1
#pragma unroll
    for (int i = 0; i < 2; ++i) load_codes(st + at.k(i), kw[i]);
#pragma unroll
    for (int w = 0; w < SH::KW; ++w) {
      uint32_t r0[4], r1[4];
      codes4(kw[0][w], r0);
      codes4(kw[1][w], r1);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        mma(z, r0[2 * u], r1[2 * u], r0[2 * u + 1], r1[2 * u + 1], q[0][0][2 * w + u][0], q[0][0][2 * w + u][1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 f = floats_of((st[at.ks(i)] | (uint32_t)st[at.ks(i) + 1] << 16) << 7);
      s[i] = fmaf(z[2 * i + 1], f.y, z[2 * i] * f.x);
      s[i] += __shfl_xor_sync(FULL, s[i], 1);
      s[i] += __shfl_xor_sync(FULL, s[i], 2);
    }
  }

  // S^T of the 16 slots at shared address st.
  __device__ __forceinline__ void scores(const unsigned char* st, const At& at, int lane, float (&s)[NB][4]) {
    const int c = lane & 3;
    uint32_t kw[2][SH::KW], sc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      load_codes(st + at.k(i), kw[i]);
      sc[i][0] = st[at.ks(i)] * 0x00800080u;  // an fp16 pair
      sc[i][1] = HD == 64 ? sc[i][0] : st[at.ks(i) + 1] * 0x00800080u;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
    for (int w = 0; w < SH::KW; ++w) {
      uint32_t r0[4], r1[4];
      codes4(kw[0][w], r0);
      codes4(kw[1][w], r1);
      // which of the lane's scales: 96 features per row have 24 per lane, one and a half groups
      uint32_t s0, s1;
      if constexpr (HD == 96) {
        const bool second = ((3 * c + w) >> 1) != ((3 * c) >> 1);
        s0 = second ? sc[0][1] : sc[0][0];
        s1 = second ? sc[1][1] : sc[1][0];
      } else {
        s0 = sc[0][w >> 1];
        s1 = sc[1][w >> 1];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r0[i] = times(r0[i], s0);
        r1[i] = times(r1[i], s1);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const int j = 2 * w + u;
          if constexpr (!EXACT) {
            mma(s[n], r0[2 * u], r1[2 * u], r0[2 * u + 1], r1[2 * u + 1], q[n][0][j][0], q[n][0][j][1]);
          } else {
            float z[4] = {0.f, 0.f, 0.f, 0.f};  // (smallest parts first)
#pragma unroll
            for (int y = NQ - 1; y >= 0; --y)
              mma(z, r0[2 * u], r1[2 * u], r0[2 * u + 1], r1[2 * u + 1], q[n][y][j][0], q[n][y][j][1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[n][i] += z[i];
          }
        }
    }
  }

  // O^T += V^T P^T of the 16 slots at st; live: bit per slot that is there (WHOLE: all).
  template <bool WHOLE>
  __device__ __forceinline__ void values(const unsigned char* st, const At& at, int lane, uint32_t live,
                                         const uint32_t (&p)[NB][NP][2]) {
    const int g = lane >> 2, c = lane & 3;
    uint32_t vs[2][2];  // scales of two slots, for the pairs 2 c + {0, 1} and 8 more
    auto pair_scales = [&](int off, uint32_t (&to)[2]) {
      uint32_t b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i] = st[at.vs(i) + off];
      if (!WHOLE)  // what lies in other slots must not reach the sums: 0 times any code
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!((live >> (2 * c + (i & 1) + 8 * (i >> 1))) & 1u)) b[i] = 0u;
      to[0] = b[0] * 0x80u + b[1] * 0x800000u;
      to[1] = b[2] * 0x80u + b[3] * 0x800000u;
    };
    pair_scales(0, vs[0]);
    if constexpr (HD == 96) {
      pair_scales(4 + (g >> 2) - (g >> 1), vs[1]);
    } else {
      vs[1][0] = vs[0][0];
      vs[1][1] = vs[0][1];
    }
    uint32_t vw[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned char* a = st + at.v(i);
      if constexpr (HD == 128) {
        const uint2 v = *reinterpret_cast<const uint2*>(a);
        vw[i][0] = v.x;
        vw[i][1] = v.y;
      } else {
        vw[i][0] = *reinterpret_cast<const uint32_t*>(a);
        vw[i][1] = HD == 96 ? *reinterpret_cast<const uint16_t*>(a - 4 * g + 32 + 2 * g) : 0u;
      }
    }
#pragma unroll
    for (int w = 0; w < (HD == 64 ? 1 : 2); ++w) {
      constexpr uint32_t M = 0x0F0F0F0Fu;
      uint32_t e[2][4], f[2][4];  // slot pairs: even features, odd features
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t x = vw[2 * h][w], y = vw[2 * h + 1][w];
        codes4((x & M) | (y << 4 & ~M), e[h]);
        codes4((x >> 4 & M) | (y & ~M), f[h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          e[h][i] = times(e[h][i], vs[w][h]);
          f[h][i] = times(f[h][i], vs[w][h]);
        }
      }
#pragma unroll
      for (int i = 0; i < (HD == 96 && w == 1 ? 2 : 4); ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          float(&to)[4] = o[n][4 * w + i];
          if constexpr (!EXACT) {
            mma(to, e[0][i], f[0][i], e[1][i], f[1][i], p[n][0][0], p[n][0][1]);
          } else if constexpr (FOLD) {
            float z[4] = {0.f, 0.f, 0.f, 0.f};
            mma(z, e[0][i], f[0][i], e[1][i], f[1][i], p[n][0][0], p[n][0][1]);
#pragma unroll
            for (int x = 0; x < 4; ++x) to[x] += z[x];
          } else {
            float y[4] = {0.f, 0.f, 0.f, 0.f}, z[4] = {0.f, 0.f, 0.f, 0.f};
            mma(y, e[0][i], f[0][i], e[1][i], f[1][i], p[n][NP - 1][0], p[n][NP - 1][1]);
            mma(z, e[0][i], f[0][i], e[1][i], f[1][i], p[n][0][0], p[n][0][1]);
#pragma unroll
            for (int x = 0; x < 4; ++x) to[x] += fmaf(y[x], 1.f / 2048.f, z[x]);
          }
        }
    }
  }

  // FOLD: scores of slots g and g + 8, of column c / 2.
  __device__ __forceinline__ void scores_fold(const unsigned char* st, const At& at, int lane, float (&s)[2]) {
    float z[NB][4];
    scores(st, at, lane, z);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i] = z[0][2 * i] + z[0][2 * i + 1];
      s[i] += __shfl_xor_sync(FULL, s[i], 1);
    }
  }

  // tiles() where a lane has scores of one column.
  template <bool WHOLE, int NT>
  __device__ __forceinline__ void tiles_one(const unsigned char* st, uint32_t stride, const At& at, int lane, int t0,
                                            uint32_t live) {
    const int g = lane >> 2;
    float s[NT][2], d[NT][2], most = -INFINITY;  // slots t0 + 16 x + g + 8 i
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      if constexpr (ONE) scores_one(st + x * stride, at, s[x]);
      else scores_fold(st + x * stride, at, lane, s[x]);
    }
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int slot = 16 * x + g + 8 * i;
        if (!WHOLE && !(((live >> slot) & 1u) && t0 + slot < lim[0][0])) s[x][i] = -INFINITY;
        d[x][i] = fmaf(s[x][i], mul[0][0], -ref[0][0]);
        most = fmaxf(most, d[x][i]);
      }
    if (__any_sync(FULL, most > kRaise)) {
      float top = -INFINITY;
#pragma unroll
      for (int x = 0; x < NT; ++x) top = fmaxf(top, fmaxf(s[x][0], s[x][1]));
#pragma unroll
      for (int y = 4; y < 32; y *= 2) top = fmaxf(top, __shfl_xor_sync(FULL, top, y));
      const float to = fmaxf(ref[0][0], below(__fmul_rn(top, mul[0][0]))), corr = ex2(ref[0][0] - to);
      ref[0][0] = to;
      l[0][0] *= corr;
#pragma unroll
      for (int m = 0; m < SH::MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[0][m][i] *= corr;
#pragma unroll
      for (int x = 0; x < NT; ++x)  // (two roundings: see tiles())
#pragma unroll
        for (int i = 0; i < 2; ++i) d[x][i] = __fsub_rn(__fmul_rn(s[x][i], mul[0][0]), ref[0][0]);
    }
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      uint32_t p[NB][NP][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float u = ex2(d[x][i]);
        l[0][0] += u;
        uint32_t w = half2_of(u, u);
        if constexpr (FOLD) {  // the rest, 2^11 larger, beside it; the odd lanes' columns are empty
          w = half2_of(u, (u - floats_of(w).x) * 2048.f);
          if (lane & 1) w = 0u;
        }
        p[0][0][i] = transposed(w);
      }
      values<WHOLE>(st + x * stride, at, lane, live >> (16 * x), p);
    }
  }

  // NT tiles, `stride` bytes apart, from shared memory st on; t0: the first slot; live:
  // bit per slot that is there and below the unit's largest limit; WHOLE: every column
  // sees every slot.
  template <bool WHOLE, int NT>
  __device__ __forceinline__ void tiles(const unsigned char* st, uint32_t stride, const At& at, int lane, int t0, uint32_t live) {
    if constexpr (ONE || FOLD) {
      tiles_one<WHOLE, NT>(st, stride, at, lane, t0, live);
      return;
    }
    const int g = lane >> 2;
    float s[NT][NB][4];
#pragma unroll
    for (int x = 0; x < NT; ++x) scores(st + x * stride, at, lane, s[x]);
    if (!WHOLE) {
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int slot = 16 * x + g + 8 * (i >> 1);
            if (!(((live >> slot) & 1u) && t0 + slot < lim[n][i & 1])) s[x][n][i] = -INFINITY;
          }
    }
    // score - reference: slots t0 + 16 x + g + 8 (i / 2), columns 2 c + i % 2 of block n
    float d[NT][NB][4], most = -INFINITY;
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[x][n][i] = fmaf(s[x][n][i], mul[n][i & 1], -ref[n][i & 1]);
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = fmaxf(most, d[x][n][i]);
    if (__any_sync(FULL, most > kRaise)) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float top = -INFINITY;
#pragma unroll
          for (int x = 0; x < NT; ++x) top = fmaxf(top, fmaxf(s[x][n][i], s[x][n][i + 2]));
#pragma unroll
          for (int y = 4; y < 32; y *= 2) top = fmaxf(top, __shfl_xor_sync(FULL, top, y));
          const float to = fmaxf(ref[n][i], below(__fmul_rn(top, mul[n][i]))), corr = ex2(ref[n][i] - to);
          ref[n][i] = to;
          l[n][i] *= corr;
#pragma unroll
          for (int m = 0; m < SH::MT; ++m) {
            o[n][m][i] *= corr;
            o[n][m][i + 2] *= corr;
          }
        }
      // (Two roundings: the rounded score is what the reference is made of.  One would
      // leave scores past 2^24 off it by more than the reference's lead.)
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) d[x][n][i] = __fsub_rn(__fmul_rn(s[x][n][i], mul[n][i & 1]), ref[n][i & 1]);
    }
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      uint32_t p[NB][NP][2];  // column g, slots 2 c + {0, 1} and 8 more
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float u = ex2(d[x][n][2 * h]), v = ex2(d[x][n][2 * h + 1]);
          l[n][0] += u;
          l[n][1] += v;
          p[n][0][h] = half2_of(u, v);
          if constexpr (NP == 2) {  // the rest, 2^11 larger so that it is no subnormal
            const float2 f = floats_of(p[n][0][h]);
            p[n][1][h] = transposed(half2_of((u - f.x) * 2048.f, (v - f.y) * 2048.f));
          }
          p[n][0][h] = transposed(p[n][0][h]);
        }
      values<WHOLE>(st + x * stride, at, lane, live >> (16 * x), p);
    }
  }

  // One step of kTiles tiles, at once but for fp32 in several parts: registers.  16 columns of
  // bf16 heads of 128 (4 drafted rows behind 8 x 32768 slots): both at once, 2 CTAs per
  // SM, 84 us; one by one 85, with 3 CTAs and the queries in shared memory 85.
  static constexpr int kAtOnce = NQ == 1 ? kTiles : 1;
  template <bool WHOLE>
  __device__ __forceinline__ void step(const unsigned char* st, uint32_t stride, const At& at, int lane, int t0,
                                       uint32_t live) {
#pragma unroll
    for (int x = 0; x < kTiles; x += kAtOnce)
      tiles<WHOLE, kAtOnce>(st + x * stride, stride, at, lane, t0 + 16 * x, live >> (16 * x));
  }

  // rec[col][HD], then (reference, sum) per column
  __device__ __forceinline__ void store(float* rec, int cols, int lane) {
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[n][i] += __shfl_xor_sync(FULL, l[n][i], d);
        const int col = FOLD ? (c >> 1) : 8 * n + 2 * c + i;
        if (col >= cols || (FOLD && ((c & 1) || i))) continue;
#pragma unroll
        for (int m = 0; m < SH::MT; ++m) {
          float2 v = make_float2(o[n][m][i], o[n][m][i + 2]);
          if (FOLD) v = make_float2(fmaf(o[n][m][1], 1.f / 2048.f, v.x), fmaf(o[n][m][3], 1.f / 2048.f, v.y));
          *reinterpret_cast<float2*>(rec + col * HD + feature<HD>(g, m)) = v;
        }
        if (g == 0) {
          rec[cols * HD + 2 * col] = ref[n][i];
          rec[cols * HD + 2 * col + 1] = l[n][i];
        }
      }
  }
};

// Slots that row x / G of sequence b sees (0: a bad length).
__device__ __forceinline__ int row_limit(const Q4AttnParams& p, int b, int row, bool& bad) {
  const int n = __ldg(p.lens + (int64_t)b * p.Tq + row);
  bad = n < 0 || n > p.max_pages * p.P - p.len_add;
  return bad ? 0 : n + p.len_add;
}
// Steps of a sequence's units.
__device__ __forceinline__ int seq_steps(const Q4AttnParams& p, int b, bool reporter) {
  int S = 0;
  for (int r = 0; r < p.Tq; ++r) {
    bool bad;
    S = max(S, row_limit(p, b, r, bad));
    if (bad && reporter) report(p.status, WM_ERR_BOUNDS);
  }
  return (S + kSlots - 1) / kSlots;
}

// Where the steps of all units are spread evenly over the CTAs (col_blocks 1): in the
// order (sequence, kv head, step) CTA i of n takes steps T i / n .. T (i + 1) / n - 1.
// All threads of the block (NT) call count and find.
template <int NT>
struct Spread {
  int64_t total;      // steps x Hkv of all sequences
  int64_t mine, own;  // of this thread's sequences: where they begin, how many they are
  int n;              // CTAs
  __device__ __forceinline__ int first_seq(const Q4AttnParams& p) const {
    return (int)threadIdx.x * ((p.B + NT - 1) / NT);
  }
  __device__ __forceinline__ void count(const Q4AttnParams& p, int ctas, bool reporter) {
    __shared__ int64_t sums[NT / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = (p.B + NT - 1) / NT;
    own = 0;
    for (int b = first_seq(p); b < min(first_seq(p) + per, p.B); ++b) own += (int64_t)seq_steps(p, b, reporter) * p.Hkv;
    int64_t incl = own;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int64_t x = __shfl_up_sync(FULL, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    total = 0;
    mine = incl - own;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
      if (w < warp) mine += sums[w];
      total += sums[w];
    }
    const int64_t most = total / (kQ4Warps * kQ4MinSteps);
    n = (int)(most < 1 ? 1 : most < ctas ? most : ctas);
  }
  // Sequence b of step pos < total, and the step's place among the sequence's.
  __device__ __forceinline__ void find(const Q4AttnParams& p, int64_t pos, int& b, int64_t& off) const {
    __shared__ int64_t at_s[2];
    if (pos >= mine && pos < mine + own) {
      int64_t x = pos - mine, w;
      int y = first_seq(p);
      while (x >= (w = (int64_t)seq_steps(p, y, false) * p.Hkv)) {
        x -= w;
        ++y;
      }
      at_s[0] = y;
      at_s[1] = x;
    }
    __syncthreads();
    b = (int)at_s[0];
    off = at_s[1];
  }
  // Steps before sequence b's.
  __device__ __forceinline__ int64_t before(const Q4AttnParams& p, int b) const {
    __shared__ int64_t before_s;
    const int per = (p.B + NT - 1) / NT;
    if (b / per == (int)threadIdx.x) {
      int64_t x = mine;
      for (int y = first_seq(p); y < b; ++y) x += (int64_t)seq_steps(p, y, false) * p.Hkv;
      before_s = x;
    }
    __syncthreads();
    return before_s;
  }
  __device__ __forceinline__ int64_t start(int i) const { return total * i / n; }
  // the CTA that takes step x: the last one that starts at or before it
  __device__ __forceinline__ int cta_of(int64_t x) const { return (int)(((x + 1) * n + total - 1) / total) - 1; }
};

// Where a cluster's (reference, sum) pairs are in a CTA's record space, and its size.
template <int HD, int NB>
constexpr int kMlAt = 8 * NB * HD + kQ4MaxCluster;
template <int HD, int NB>
constexpr int kJoinFloats = kMlAt<HD, NB> + 2 * kQ4MaxCluster * 8 * NB;

template <typename T, int HD, int NB, int LT, Fill FILL>
__global__ void __launch_bounds__(kThreads, q4_ctas_per_sm(sizeof(T) == 2, NB, FILL == kFold))
    q4_attn_kernel(const Q4AttnParams p) {
  using SH = Shape<HD>;
  constexpr int STAGE = kTiles * (LT > 0 ? SH::BYTES16 : SH::PADDED16);
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char* ring = smem_raw + warp * kStages * STAGE;
  float* crec = reinterpret_cast<float*>(smem_raw + kQ4Warps * kStages * STAGE);

  // Dependents start only after this grid's own wait, so that everything before
  // it is visible to them whatever they wait for; and early only where this grid fills
  // the SMs.  Elsewhere CTAs that start beside these would crowd on the SMs that have
  // most room: 400 units of 2048 slots, back to back, 27.3 us instead of 33.4.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (p.part) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  int b, h, x0 = 0, piece = 0, C = 1;
  int64_t off = 0, left = 0;  // spread: step among the sequence's units, steps left to take
  const bool spread = p.part != nullptr;
  if (spread) {
    Spread<kThreads> sp;
    sp.count(p, (int)gridDim.x, blockIdx.x == 0);
    // sequences without steps get their zeros
    for (int y = blockIdx.x; y < p.B; y += (int)gridDim.x)
      if (seq_steps(p, y, false) == 0) {
        T* out = reinterpret_cast<T*>(p.out) + (int64_t)y * p.Tq * p.Hq * HD;
        for (int e = tid; e < p.Tq * p.Hq * HD; e += kThreads) out[e] = Elem<T>::from_f(0.f);
      }
    if ((int)blockIdx.x >= sp.n) return;
    const int64_t pos = sp.start(blockIdx.x);
    left = sp.start(blockIdx.x + 1) - pos;
    if (left == 0) return;
    sp.find(p, pos, b, off);
    h = 0;
  } else {
    C = p.pieces;
    const int unit = (int)(blockIdx.x / (unsigned)C);
    piece = (int)(blockIdx.x - (unsigned)unit * C);
    const int bh = unit / p.col_blocks;
    x0 = (unit - bh * p.col_blocks) * 8 * NB;
    b = bh / p.Hkv;
    h = bh - b * p.Hkv;
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // (this CTA is there)
  }
  const int cols = min(8 * NB, p.Tq * p.G - x0), E = cols * HD;

  for (;;) {  // units (one, unless spread)
  int S = 0, least = INT32_MAX;  // largest and smallest limit of the unit's columns
  {
    bool bad = false;
    if (lane < cols) {
      least = S = row_limit(p, b, (x0 + lane) / p.G, bad);
      if (bad && !spread && h == 0 && piece == 0 && warp == 0) report(p.status, WM_ERR_BOUNDS);
    }
    S = __reduce_max_sync(FULL, S);
    least = __reduce_min_sync(FULL, least);
  }
  const int nsteps = (S + kSlots - 1) / kSlots;
  int from = (int)((int64_t)piece * nsteps / C), steps = (int)((int64_t)(piece + 1) * nsteps / C) - from;
  if (spread) {
    if (off >= (int64_t)nsteps * p.Hkv) {  // on to the next sequence
      off = 0;
      ++b;
      continue;
    }
    h = (int)(off / nsteps);
    from = (int)(off - (int64_t)h * nsteps);
    steps = (int)min((int64_t)(nsteps - from), left);
  }
  const int j0 = from + (int)((int64_t)warp * steps / kQ4Warps);
  const int nmine = from + (int)((int64_t)(warp + 1) * steps / kQ4Warps) - j0;

  // ---- the warp's copies: step i into ring slot i modulo kStages, in 16-byte chunks
  const int32_t* ptab = p.page_table + (int64_t)b * p.max_pages;
  const uint32_t ring_s = smem_u32(ring), to_s = ring_s + lane * 16;
  const uint8_t* pool_lane = p.pool + lane * 16;
  const int log2tile = LT > 0 ? LT : p.log2tile, tiles = kSlots >> log2tile;
  const int per_batch = 1 << log2tile;  // steps whose tiles the lanes hold, one each
  const uint32_t tile_bytes = LT > 0 ? SH::template tile<LT>() : p.tile_bytes;
  const uint32_t stride = LT > 0 ? SH::BYTES16 : kQ4Step / p.tile * tile_bytes;
  // Tiles of `per_batch` steps from step i on, one per lane: its place in the pool (kGone:
  // not seen, or no such page), for tiles below 16 slots less its place in the step, so that
  // a step's chunk y lies y * 16 bytes behind it whichever tile it is of.
  constexpr int kGone = INT32_MIN;
  auto look_up = [&](int i) -> int {
    const int x = i + (lane >> (5 - log2tile)), t = (j0 + i) * kSlots + (lane << log2tile);
    if (x >= nmine || t >= S) return kGone;
    const int pg = __ldg(ptab + (t >> p.log2P));
    if ((unsigned)pg >= (unsigned)p.num_pages) {
      report(p.status, WM_ERR_BOUNDS);
      return kGone;
    }
    const int at = LT == 4 ? (pg * p.Hkv + h) * (p.P / kQ4Step) + (t & (p.P - 1)) / kQ4Step : pg * p.Hkv + h;
    return LT == 4 ? at : at - (lane & (tiles - 1));
  };
  int batch = look_up(0), ahead = look_up(per_batch);
  // Returns which of the step's tiles are there (a bit per tile).
  auto issue = [&](int i, int stage) -> uint32_t {
    const int first = (i & (per_batch - 1)) * tiles;  // lane that holds the step's first tile
    const uint32_t to = to_s + stage * STAGE;
    uint32_t there;
    if constexpr (LT == 4) {
      there = 0;
#pragma unroll
      for (int x = 0; x < kTiles; ++x) {
        const int at = __shfl_sync(FULL, batch, first + x);
        if (at >= 0) there |= 1u << x;
        cp_async_tile<HD>(to + x * SH::BYTES16, pool_lane + (int64_t)at * SH::BYTES16, at, lane);
      }
    } else {
      there = __ballot_sync(FULL, batch != kGone) >> first;
      if (tiles < 32) there &= (1u << tiles) - 1;
      if constexpr (LT > 0) {
        constexpr int CH = SH::template tile<LT>() / 16, ALL = kTiles * SH::BYTES16 / 16;
#pragma unroll
        for (int y = 0; y < ALL; y += 32) {
          const int x = min((y + lane) / CH, (kSlots >> LT) - 1), at = __shfl_sync(FULL, batch, first + x);
          cp_async16(to + y * 16, pool_lane + (int64_t)at * SH::template tile<LT>() + y * 16,
                     at != kGone && (y + 32 <= ALL || y + lane < ALL));
        }
      } else {
        const int chunks = (int)tile_bytes / 16, magic = 65536 / chunks + 1;
        for (int y = 0; y < tiles * chunks; y += 32) {
          const int x = (y + lane) * magic >> 16, at = __shfl_sync(FULL, batch, (first + x) & 31);
          cp_async16(to + y * 16, pool_lane + (int64_t)at * tile_bytes + y * 16, x < tiles && at != kGone);
        }
      }
    }
    if ((i & (per_batch - 1)) == per_batch - 1) {
      batch = ahead;
      ahead = look_up(i + 1 + per_batch);
    }
    return there;
  };
  // one commit group per step, empty ones included, so that group i is step i
  uint32_t there[kStages];  // of the steps in flight, the next one first
#pragma unroll
  for (int i = 0; i < kStages; ++i) {
    there[i] = i < nmine ? issue(i, i) : 0u;
    cp_async_commit();
  }

  // ---- queries
  using Mm = Math<T, HD, NB, LT, FILL>;
  Mm mm;
  mm.init();
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int col = FILL == kOne ? 0 : FILL == kFold ? lane >> 4 : 8 * n + (lane >> 2), x = x0 + col;
    const T* row = nullptr;
    int lim = 0;
    if (col < cols) {
      bool bad;
      row = reinterpret_cast<const T*>(p.q) + (((int64_t)b * p.Tq + x / p.G) * p.Hq + h * p.G + x % p.G) * HD;
      lim = row_limit(p, b, x / p.G, bad);
    }
    mm.load(n, row, lim, lane, p.qscale);
  }
  const typename Mm::At at = Mm::offsets(p.log2tile, p.tile_bytes, lane);

  const uint32_t every = tiles < 32 ? (1u << tiles) - 1 : FULL;
  int t0 = j0 * kSlots, stage = 0;
  for (int i = 0; i < nmine; ++i, t0 += kSlots) {
    cp_async_wait<kStages - 1>();
    __syncwarp();
    const unsigned char* st = ring + stage * STAGE;
    if (there[0] == every && t0 + kSlots <= least) {
      mm.template step<true>(st, stride, at, lane, t0, FULL);
    } else {
      uint32_t live = 0;
      for (int x = 0; x < tiles; ++x)
        if ((there[0] >> x) & 1u) live |= ((1u << (1 << log2tile)) - 1) << (x << log2tile);  // a tile's slots
      if (S - t0 < kSlots) live &= (1u << (S - t0)) - 1;
      mm.template step<false>(st, stride, at, lane, t0, live);
    }
    __syncwarp();  // every lane is done with this ring slot
#pragma unroll
    for (int x = 0; x + 1 < kStages; ++x) there[x] = there[x + 1];
    if (i + kStages < nmine) there[kStages - 1] = issue(i + kStages, stage);
    cp_async_commit();
    stage = stage + 1 < kStages ? stage + 1 : 0;
  }
  cp_async_wait<0>();

  // ---- join the CTA's warps (each warp's state in its idle ring)
  __syncwarp();
  float* wrec = reinterpret_cast<float*>(ring);
  mm.store(wrec, cols, lane);
  __syncthreads();
  auto warp_rec = [&](int w) -> const float* {
    return reinterpret_cast<const float*>(smem_raw + w * kStages * STAGE);
  };
  auto out_row = [&](int col) -> T* {
    const int x = x0 + col;
    return reinterpret_cast<T*>(p.out) + (((int64_t)b * p.Tq + x / p.G) * p.Hq + h * p.G + x % p.G) * HD;
  };
  // a unit that a CTA has to itself is done.  Its part of one that the spread cut goes to
  // the CTA's record 0 (the unit began before its steps) or 1; in a cluster CTA c finishes
  // outputs c * share .. and gets the others' parts of them through distributed shared
  // memory: [C][share], then [C][cols] (reference, sum).
  const bool direct = C == 1 && steps == nsteps;
  float* rec = spread ? p.part + ((int64_t)blockIdx.x * 2 + (from == 0)) * q4_rec(8 * NB, HD) : crec;
  const int share = (E + C - 1) / C;
  cg::cluster_group cluster = cg::this_cluster();
  if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every CTA is there
  auto joined_ml = [&](int r, float& M, float& L) {
    M = -FLT_MAX;
    L = 0.f;
#pragma unroll
    for (int w = 0; w < kQ4Warps; ++w) M = fmaxf(M, warp_rec(w)[E + 2 * r]);
#pragma unroll
    for (int w = 0; w < kQ4Warps; ++w) L = fmaf(exp2f(warp_rec(w)[E + 2 * r] - M), warp_rec(w)[E + 2 * r + 1], L);
  };
  for (int e = tid; e < E; e += kThreads) {
    const int r = e / HD;
    float M, L, O = 0.f;
    joined_ml(r, M, L);
#pragma unroll
    for (int w = 0; w < kQ4Warps; ++w) O = fmaf(exp2f(warp_rec(w)[E + 2 * r] - M), warp_rec(w)[e], O);
    if (direct) {
      out_row(r)[e - r * HD] = Elem<T>::from_f(L == 0.f ? 0.f : O / L);
    } else if (spread) {
      rec[e] = O;
      if (e == r * HD) {
        rec[8 * NB * HD + 2 * r] = M;
        rec[8 * NB * HD + 2 * r + 1] = L;
      }
    } else {
      const int c = e / share;
      cluster.map_shared_rank(crec, c)[piece * share + e - c * share] = O;
    }
  }
  if (spread) {
    left -= steps;
    if (left == 0) return;
    off += steps;
    __syncthreads();  // the rings take copies again
    continue;
  }
  if (C == 1) return;
  for (int x = tid; x < cols * C; x += kThreads) {
    const int r = x / C, c = x - r * C;
    float M, L;
    joined_ml(r, M, L);
    *reinterpret_cast<float2*>(cluster.map_shared_rank(crec, c) + kMlAt<HD, NB> + 2 * (piece * cols + r)) = make_float2(M, L);
  }
  // (nothing is written to a CTA's shared memory behind this, so it may end before the others)
  cluster.sync();
  for (int e = piece * share + tid; e < min((piece + 1) * share, E); e += kThreads) {
    const int r = e / HD;
    float M = -FLT_MAX, L = 0.f, O = 0.f;
    for (int c = 0; c < C; ++c) M = fmaxf(M, crec[kMlAt<HD, NB> + 2 * (c * cols + r)]);
    for (int c = 0; c < C; ++c) {
      const float2 ml = *reinterpret_cast<const float2*>(crec + kMlAt<HD, NB> + 2 * (c * cols + r));
      const float wt = exp2f(ml.x - M);
      L = fmaf(wt, ml.y, L);
      O = fmaf(wt, crec[c * share + e - piece * share], O);
    }
    out_row(r)[e - r * HD] = Elem<T>::from_f(L == 0.f ? 0.f : O / L);
  }
  return;
  }
}

// Joins the records of units whose steps several CTAs took: out = sum_i 2^(m_i - M) O_i /
// sum_i 2^(m_i - M) l_i.  blockIdx.x is the unit, or (fewer CTAs than units) the CTA that
// took such a unit's first steps, blockIdx.y 32 groups of four of its outputs; 8 threads
// share a group's records.
template <typename T, int HD>
__global__ void __launch_bounds__(256) q4_join_kernel(const Q4AttnParams p, int by_unit) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ float4 o_s[8][32];
  __shared__ float l_s[8][32];
  Spread<256> sp;
  sp.count(p, p.pieces, false);
  int b, h, first;
  int64_t unit;  // the unit's first step
  if (by_unit) {
    b = (int)blockIdx.x / p.Hkv;
    h = (int)blockIdx.x - b * p.Hkv;
    const int ns = seq_steps(p, b, false);
    if (ns == 0) return;
    unit = sp.before(p, b) + (int64_t)h * ns;
    first = sp.cta_of(unit);
  } else {
    first = blockIdx.x;
    if (first + 1 >= sp.n) return;
    const int64_t end = sp.start(first + 1);
    int64_t off;
    sp.find(p, end - 1, b, off);  // the unit that the CTA's last step belongs to
    const int ns = seq_steps(p, b, false);
    h = (int)(off / ns);
    unit = end - 1 - (off - (int64_t)h * ns);
    if (unit < sp.start(first)) return;  // begun by another CTA
  }
  const int n = sp.cta_of(unit + seq_steps(p, b, false) - 1) - first + 1;
  if (n == 1) return;  // written by its CTA
  const int cols = p.Tq * p.G, most = 8 * p.nb;
  const int tid = threadIdx.x, lane = tid & 31, grp = tid >> 5, recf = q4_rec(most, HD);
  const int y = blockIdx.y * 32 + lane;  // four outputs
  const bool on = y < cols * HD / 4;
  const int r = on ? y / (HD / 4) : 0, e = on ? (y - r * (HD / 4)) * 4 : 0;
  float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
  float L = 0.f;
  // record i: the first CTA's begins with the unit
  auto rec = [&](int i) -> const float* { return p.part + ((int64_t)(first + i) * 2 + (i == 0)) * recf; };
  float M = -FLT_MAX;
  for (int i = grp; i < n; i += 8) M = fmaxf(M, __ldcg(rec(i) + most * HD + 2 * r));
  l_s[grp][lane] = M;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) M = fmaxf(M, l_s[i][lane]);
  __syncthreads();
  constexpr int NBUF = 4;
  for (int i0 = grp; i0 < n; i0 += 8 * NBUF) {
    float4 v[NBUF];
    float2 ml[NBUF];
#pragma unroll
    for (int i = 0; i < NBUF; ++i)
      if (i0 + 8 * i < n) {
        v[i] = __ldcg(reinterpret_cast<const float4*>(rec(i0 + 8 * i) + r * HD + e));
        ml[i] = __ldcg(reinterpret_cast<const float2*>(rec(i0 + 8 * i) + most * HD + 2 * r));
      }
#pragma unroll
    for (int i = 0; i < NBUF; ++i) {
      if (i0 + 8 * i >= n) continue;
      const float w = exp2f(ml[i].x - M);
      L = fmaf(w, ml[i].y, L);
      O.x = fmaf(w, v[i].x, O.x);
      O.y = fmaf(w, v[i].y, O.y);
      O.z = fmaf(w, v[i].z, O.z);
      O.w = fmaf(w, v[i].w, O.w);
    }
  }
  o_s[grp][lane] = O;
  l_s[grp][lane] = L;
  __syncthreads();
  if (grp > 0 || !on) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const float4 v = o_s[i][lane];
    L += l_s[i][lane];
    O.x += v.x;
    O.y += v.y;
    O.z += v.z;
    O.w += v.w;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  T* out = reinterpret_cast<T*>(p.out) + (((int64_t)b * p.Tq + r / p.G) * p.Hq + h * p.G + r % p.G) * HD + e;
  out[0] = Elem<T>::from_f(O.x * inv);
  out[1] = Elem<T>::from_f(O.y * inv);
  out[2] = Elem<T>::from_f(O.z * inv);
  out[3] = Elem<T>::from_f(O.w * inv);
}

template <typename Kern, typename... Args>
inline cudaError_t launch_chained(Kern kern, dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s,
                                  const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 0 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <typename T, int HD, int NB, int LT, Fill FILL>
inline cudaError_t launch_t(const Q4AttnParams& p, cudaStream_t s) {
  using SH = Shape<HD>;
  static size_t smem_set[kSmemOptDevices] = {};
  auto kern = q4_attn_kernel<T, HD, NB, LT, FILL>;
  constexpr size_t ring = (size_t)kStages * kTiles * (LT > 0 ? SH::BYTES16 : SH::PADDED16), rec = q4_rec(8 * NB, HD) * sizeof(float);
  constexpr size_t join = kJoinFloats<HD, NB> * sizeof(float);
  static_assert(kTiles <= 2, "a bit per slot");
  static_assert(rec <= ring && ring % 16 == 0, "a warp's record goes into its ring");
  const size_t smem = kQ4Warps * ring + (p.part || p.pieces == 1 ? 0 : join);
  if (cudaError_t e = opt_in_smem(kern, smem, smem_set); e != cudaSuccess) return e;
  const unsigned units = (unsigned)p.B * p.Hkv * p.col_blocks;
  if (!p.part) return launch_chained(kern, dim3(units * (unsigned)p.pieces), kThreads, smem, p.pieces, s, p);
  const cudaError_t e = launch_chained(kern, dim3(p.pieces), kThreads, smem, 0, s, p);
  if (e != cudaSuccess) return e;
  const unsigned groups = (unsigned)(p.Tq * p.G * HD / 4 + 31) / 32;
  const bool by_unit = units <= (unsigned)p.pieces;
  return launch_chained(q4_join_kernel<T, HD>, dim3(by_unit ? units : (unsigned)p.pieces, groups), 256, 0, 0, s, p, (int)by_unit);
}

template <typename T, int HD, int NB, Fill FILL>
inline cudaError_t launch_lt(const Q4AttnParams& p, cudaStream_t s) {
  switch (p.log2tile) {
    case 4: return launch_t<T, HD, NB, 4, FILL>(p, s);
    case 3: return launch_t<T, HD, NB, 3, FILL>(p, s);
    case 2: return launch_t<T, HD, NB, 2, FILL>(p, s);
    default: return launch_t<T, HD, NB, 0, FILL>(p, s);
  }
}

template <typename T, int HD>
inline cudaError_t launch_d(const Q4AttnParams& p, cudaStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (p.Tq * p.G == 1) return launch_lt<T, HD, 1, kOne>(p, s);
    if (p.nb == 2) return launch_lt<T, HD, 2, kColumns>(p, s);
  } else {
    if (p.Tq * p.G <= kQ4Fold) return launch_lt<T, HD, 1, kFold>(p, s);
  }
  return launch_lt<T, HD, 1, kColumns>(p, s);
}

}  // namespace q4_detail

// Per-dtype dispatch (one translation unit each, compiled in parallel).
cudaError_t launch_q4_attn_bf16(const Q4AttnParams& p, int d, cudaStream_t s);
cudaError_t launch_q4_attn_f32(const Q4AttnParams& p, int d, cudaStream_t s);

}  // namespace wm
