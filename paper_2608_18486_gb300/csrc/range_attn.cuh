#pragma once
// Attention of a few query rows over part of a sequence's cached slots: a
// sliding window and the first slots (sinks), a shared prefix, the suffix
// behind it, or every slot with the scores kept.
//
//   out_r = sum_t p_rt v_t,  p_rt = 2^(s_rt - m_r) / l_r,  s_rt = (q_r . k_t) log2(e) / sqrt(d)
//   over the visible slots t; (m, l, sum_t 2^(s - m) v_t) of disjoint slot
//   sets join as in the decode attention.
//
// A unit is one group of at most 8 query rows that read the same K/V rows: the
// G query heads of a (sequence, kv head), or 8 rows of any sequences over a
// shared prefix.  `pieces` CTAs of 4 warps share a unit; each warp streams a
// contiguous part of its stages through a private ring of cp.async copies
// (16 bytes per lane, rows of masked slots filled with zeros, so that nothing
// stored there reaches the sums).  The work reads about one byte per FLOP and
// is bound by HBM, so the math only has to stay out of the way:
//  * bf16: mma.sync m16n8k16 with the query rows as the 16-row operand (8 used)
//    for both products (in P V the 8 others carry the low parts of the
//    probabilities), K and V read from shared memory with ldmatrix (chunks
//    of 16 bytes XOR-swizzled by the slot, so that no read conflicts); the
//    cost does not grow with the query heads of a kv head.
//  * fp32, up to 4 rows: CUDA-core FMAs, 8 lanes per slot, queries in shared
//    memory.
//  * fp32, 8 rows: the bf16 products on operands split into three bf16 parts (8
//    bits of the 24 each): x = h + m + l, and q k = (qh + qm)(kh + km + kl) +
//    ql kh up to 2^-23 of |q||k|.  h and m of the query rows fill the 16 rows of
//    one operand, so four matrix instructions do what one does for bf16; the
//    splitting of K and V bounds it (about 4.4 TB/s whatever the rows).  us per
//    call over 1028 slots of 32 sequences, 32 query heads of 128 (FMAs / split): 1
//    row per unit 159 / 229, 2 rows 87 / 123, 4 rows 56 / 63, 8 rows 64 / 40.
// Measured, bf16: windows of 1028 slots, 32 sequences of 32 heads of 128: 88 us,
// 6.1 TB/s; with mass, 8 sequences of 32768 slots of 32 heads of 128: 613 us, 6.8
// TB/s.  CTAs of 4 warps, two per SM: of 2 warps, four per SM, take 94 and 615, of
// 8, one per SM, 93 and 627 (8 windows of 4112 slots of 8 kv heads 27 / 38 / 27).
#include <cooperative_groups.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "range_attn.h"

namespace wm {
namespace range_detail {

namespace cg = cooperative_groups;

constexpr int kThreads = kRangeWarps * 32;
constexpr int kStages = 3;  // ring depth per warp

template <typename T, int HD>
struct Shape {
  static constexpr int VEC = Elem<T>::kVec;
  static constexpr int ROWV = HD * (int)sizeof(T) / 16;  // 16-byte chunks of a row
  static constexpr int SS = sizeof(T) == 2 ? (HD == 64 ? 32 : 16) : (HD == 64 ? 16 : 8);
  static constexpr int ROW_BYTES = ROWV * 16;
  static constexpr int HALF_BYTES = SS * ROW_BYTES;      // K (or V) of one stage
  static constexpr int STAGE_BYTES = 2 * HALF_BYTES;
  static constexpr int CHUNKS = SS * ROWV;
  static_assert(CHUNKS % 32 == 0, "whole warp copies");
};

// Place of 16-byte chunk c of slot row `slot`.  bf16: any 8 consecutive slots have
// a given chunk on 8 different 16-byte bank groups (ldmatrix).  fp32: so have
// two neighbouring slots with 4 chunks each, and 4 slots two apart with 2.
template <typename T, int HD>
__device__ __forceinline__ int swz(int slot, int c) {
  if (sizeof(T) == 4) return c ^ (slot & 6) ^ ((slot & 1) << 2);
  if (HD == 96) return c ^ ((slot >> 1) & 3);  // rows of 192 bytes alternate halves already
  return c ^ (slot & 7);
}

__device__ __forceinline__ void cp_async16_zfill(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
               "r"(live ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// c (rows 0-7 of the 16 x 8 tile) += A B with rows 8-15 of A zero
__device__ __forceinline__ void mma_rows8(float (&c)[2], uint32_t a0, uint32_t a2, uint32_t b0, uint32_t b1) {
  [[maybe_unused]] float x, y;
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %5}, {%7, %8}, "
      "{%0, %1, %9, %9};"
      : "+f"(c[0]), "+f"(c[1]), "=f"(x), "=f"(y)
      : "r"(a0), "r"(0u), "r"(a2), "r"(b0), "r"(b1), "f"(0.f));
}

// c += A B, all 16 rows
__device__ __forceinline__ void mma_rows16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                           uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two neighbouring scores of a row (t even) that has `lim` slots.
__device__ __forceinline__ void put_scores(float* row, int t, int lim, float a, float b) {
  if (t + 1 < lim) *reinterpret_cast<float2*>(row + t) = make_float2(a, b);
  else if (t < lim) row[t] = a;
}

// The visible slots of a unit: [0, a) and [w0, S), as stages of SS slots.
struct Range {
  int S, a, w0, n0, f, n;  // n0 stages of the first part, then from stage f on; n in all
};
template <int SS>
__device__ __forceinline__ Range make_range(int S, int a, int w0) {
  Range r;
  r.S = S;
  r.a = min(a, S);
  r.w0 = min(max(w0, r.a), S);
  const int ns = (S + SS - 1) / SS;
  r.n0 = (r.a + SS - 1) / SS;
  r.f = max(r.w0 / SS, r.n0);
  r.n = r.n0 + (r.w0 < S ? max(ns - r.f, 0) : 0);
  return r;
}

// ------------------------------------------------------------ bf16: matrix instructions
template <int HD>
struct MmaMath {
  using T = __nv_bfloat16;
  using SH = Shape<T, HD>;
  static constexpr int SS = SH::SS, NT = SS / 8;
  uint32_t qa[HD / 16][2];  // A operand: row lane / 4, features 16 kk + 2 (lane % 4) (+ 8)
  float acc[HD / 8][4];     // features 8 j + 2 (lane % 4) + {0, 1} of row lane / 4: from the
                            // probabilities' high parts, then from their low parts
  float m, l;               // of row lane / 4 (l: this lane's slots only)
  int lim;                  // slots of the row: t < lim

  // qrow: this lane's row (lane / 4), or NULL
  __device__ __forceinline__ void init(const T* qrow, int lane, int lim_) {
    const int c = lane & 3;
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk) {
      qa[kk][0] = qrow ? __ldcg(reinterpret_cast<const uint32_t*>(qrow + 16 * kk + 2 * c)) : 0u;
      qa[kk][1] = qrow ? __ldcg(reinterpret_cast<const uint32_t*>(qrow + 16 * kk + 8 + 2 * c)) : 0u;
    }
#pragma unroll
    for (int j = 0; j < HD / 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
    m = -INFINITY;
    l = 0.f;
    lim = lim_;
  }

  // One stage; t0: slot of its first row; live: bit per slot that may be seen.
  // srow (NULL: none): the row's scores, written at t.
  template <bool SCORES>
  __device__ __forceinline__ void stage(uint32_t ks, uint32_t vs, int lane, int t0, uint32_t live, float qscale,
                                        float* srow) {
    const int c = lane & 3;
    float s[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      s[nt][0] = s[nt][1] = 0.f;
      const int slot = nt * 8 + (lane & 7);
#pragma unroll
      for (int q = 0; q < HD / 32; ++q) {
        uint32_t b[4];
        ldsm4(b, ks + slot * SH::ROW_BYTES + swz<T, HD>(slot, 4 * q + (lane >> 3)) * 16);
        mma_rows8(s[nt], qa[2 * q][0], qa[2 * q][1], b[0], b[1]);
        mma_rows8(s[nt], qa[2 * q + 1][0], qa[2 * q + 1][1], b[2], b[3]);
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int slot = nt * 8 + 2 * c + i;
        const bool see = ((live >> slot) & 1u) && t0 + slot < lim;
        s[nt][i] = see ? s[nt][i] * qscale : -INFINITY;
        mx = fmaxf(mx, s[nt][i]);
      }
    if (SCORES && srow)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) put_scores(srow, t0 + nt * 8 + 2 * c, lim, s[nt][0], s[nt][1]);
    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
    const float mnew = fmaxf(m, mx);
    if (__any_sync(0xFFFFFFFFu, mnew > m)) {
      const float corr = m == -INFINITY ? 0.f : exp2f(m - mnew);
      l *= corr;
#pragma unroll
      for (int j = 0; j < HD / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] *= corr;
      m = mnew;
    }
    // Probabilities enter P V as two bf16 parts, p = hi + lo (16 bits of p): the
    // low parts fill rows 8-15 of the A operand, which the query rows leave
    // empty, so they cost no product.  The row sum is kept from p itself.
    uint32_t hi[NT], lo[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float p0 = s[nt][0] == -INFINITY ? 0.f : exp2f(s[nt][0] - m);
      const float p1 = s[nt][1] == -INFINITY ? 0.f : exp2f(s[nt][1] - m);
      l += p0 + p1;
      const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
      const __nv_bfloat162 g = __floats2bfloat162_rn(p0 - __low2float(h), p1 - __high2float(h));
      hi[nt] = *reinterpret_cast<const uint32_t*>(&h);
      lo[nt] = *reinterpret_cast<const uint32_t*>(&g);
    }
#pragma unroll
    for (int kt = 0; kt < NT / 2; ++kt) {
      const int slot = kt * 16 + (lane & 15);
#pragma unroll
      for (int u = 0; u < HD / 16; ++u) {
        uint32_t b[4];
        ldsm4_t(b, vs + slot * SH::ROW_BYTES + swz<T, HD>(slot, 2 * u + (lane >> 4)) * 16);
        mma_rows16(acc[2 * u], hi[2 * kt], lo[2 * kt], hi[2 * kt + 1], lo[2 * kt + 1], b[0], b[1]);
        mma_rows16(acc[2 * u + 1], hi[2 * kt], lo[2 * kt], hi[2 * kt + 1], lo[2 * kt + 1], b[2], b[3]);
      }
    }
  }

  // rec[row][HD], rec[rows * HD + 2 row]: (max, sum)
  __device__ __forceinline__ void store(float* rec, int rows, int lane) {
    l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
    l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
    const int r = lane >> 2, c = lane & 3;
    if (r >= rows) return;
#pragma unroll
    for (int j = 0; j < HD / 8; ++j)
      *reinterpret_cast<float2*>(rec + r * HD + 8 * j + 2 * c) = make_float2(acc[j][0] + acc[j][2], acc[j][1] + acc[j][3]);
    if (c == 0) {
      rec[rows * HD + 2 * r] = m;
      rec[rows * HD + 2 * r + 1] = l;
    }
  }
};

// ------------------------------------------------------------ fp32: three bf16 parts
// x0 and x1 as packed pairs of parts: h rounded, m the next 8 bits, l the rest.
struct Split {
  uint32_t h, m, l;
};
__device__ __forceinline__ Split split2(float x0, float x1) {
  const uint32_t a = __float_as_uint(x0) + 0x8000u, b = __float_as_uint(x1) + 0x8000u;
  const float r0 = x0 - __uint_as_float(a & 0xFFFF0000u), r1 = x1 - __uint_as_float(b & 0xFFFF0000u);
  const uint32_t c = __float_as_uint(r0), d = __float_as_uint(r1);
  const float l0 = r0 - __uint_as_float(c & 0xFFFF0000u), l1 = r1 - __uint_as_float(d & 0xFFFF0000u);
  Split s;
  s.h = __byte_perm(a, b, 0x7632);
  s.m = __byte_perm(c, d, 0x7632);
  s.l = __byte_perm(__float_as_uint(l0), __float_as_uint(l1), 0x7632);
  return s;
}
__device__ __forceinline__ void mma_k8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t b) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(b));
}
__device__ __forceinline__ float4 lds128(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

template <int HD>
struct SplitMath {
  using T = float;
  using SH = Shape<T, HD>;
  static constexpr int SS = SH::SS, NT = SS / 8;
  Split q0[HD / 16], q1[HD / 16];  // row lane / 4, features 16 j + 4 (lane % 4) + {0, 1} and {2, 3}
  float acc[HD / 8][2];            // tile 4 u + t: features 4 (2 (lane % 4) + {0, 1} + 8 u) + t
  float m, l;
  int lim;

  __device__ __forceinline__ void init(const T* qrow, int lane, int lim_) {
    const int c = lane & 3;
#pragma unroll
    for (int j = 0; j < HD / 16; ++j) {
      const float4 x = qrow ? __ldcg(reinterpret_cast<const float4*>(qrow + 16 * j + 4 * c)) : make_float4(0.f, 0.f, 0.f, 0.f);
      q0[j] = split2(x.x, x.y);
      q1[j] = split2(x.z, x.w);
    }
#pragma unroll
    for (int j = 0; j < HD / 8; ++j) acc[j][0] = acc[j][1] = 0.f;
    m = -INFINITY;
    l = 0.f;
    lim = lim_;
  }

  template <bool SCORES>
  __device__ __forceinline__ void stage(uint32_t ks, uint32_t vs, int lane, int t0, uint32_t live, float qscale,
                                        float* srow) {
    const int c = lane & 3, n = lane >> 2;
    float s[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int slot = nt * 8 + n;
      s[nt][0] = s[nt][1] = 0.f;
#pragma unroll
      for (int j = 0; j < HD / 16; ++j) {
        // A matrix instruction truncates its sums: each group of four starts at
        // zero, smallest terms first, and is added with rounding (in one chain over
        // all features and slots the error of a result reached 1e-6).
        float z[4] = {0.f, 0.f, 0.f, 0.f};
        const float4 k = lds128(ks + slot * SH::ROW_BYTES + swz<T, HD>(slot, c + 4 * j) * 16);
        const Split b0 = split2(k.x, k.y), b1 = split2(k.z, k.w);
        mma_rows16(z, q0[j].h, q0[j].m, q1[j].h, q1[j].m, b0.l, b1.l);
        mma_rows16(z, q0[j].l, 0u, q1[j].l, 0u, b0.h, b1.h);
        mma_rows16(z, q0[j].h, q0[j].m, q1[j].h, q1[j].m, b0.m, b1.m);
        mma_rows16(z, q0[j].h, q0[j].m, q1[j].h, q1[j].m, b0.h, b1.h);
        s[nt][0] += z[0] + z[2];
        s[nt][1] += z[1] + z[3];
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int slot = nt * 8 + 2 * c + i;
        const bool see = ((live >> slot) & 1u) && t0 + slot < lim;
        s[nt][i] = see ? s[nt][i] * qscale : -INFINITY;
        mx = fmaxf(mx, s[nt][i]);
      }
    if (SCORES && srow)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) put_scores(srow, t0 + nt * 8 + 2 * c, lim, s[nt][0], s[nt][1]);
    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
    const float mnew = fmaxf(m, mx);
    if (__any_sync(0xFFFFFFFFu, mnew > m)) {
      const float corr = m == -INFINITY ? 0.f : exp2f(m - mnew);
      l *= corr;
#pragma unroll
      for (int j = 0; j < HD / 8; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[j][i] *= corr;
      m = mnew;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float p0 = s[nt][0] == -INFINITY ? 0.f : exp2f(s[nt][0] - m);
      const float p1 = s[nt][1] == -INFINITY ? 0.f : exp2f(s[nt][1] - m);
      l += p0 + p1;
      const Split p = split2(p0, p1);
      const int slot = nt * 8 + 2 * c;
#pragma unroll
      for (int u = 0; u < HD / 32; ++u) {
        const float4 x = lds128(vs + slot * SH::ROW_BYTES + swz<T, HD>(slot, n + 8 * u) * 16);
        const float4 y = lds128(vs + (slot + 1) * SH::ROW_BYTES + swz<T, HD>(slot + 1, n + 8 * u) * 16);
        const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const Split b = split2(xs[t], ys[t]);
          float z[4] = {0.f, 0.f, 0.f, 0.f};
          mma_k8(z, p.h, p.m, b.l);
          mma_k8(z, p.l, 0u, b.h);
          mma_k8(z, p.h, p.m, b.m);
          mma_k8(z, p.h, p.m, b.h);
          acc[4 * u + t][0] += z[0] + z[2];
          acc[4 * u + t][1] += z[1] + z[3];
        }
      }
    }
  }

  __device__ __forceinline__ void store(float* rec, int rows, int lane) {
    l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
    l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
    const int r = lane >> 2, c = lane & 3;
    if (r >= rows) return;
#pragma unroll
    for (int u = 0; u < HD / 32; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        *reinterpret_cast<float4*>(rec + r * HD + 4 * (2 * c + i + 8 * u)) =
            make_float4(acc[4 * u][i], acc[4 * u + 1][i], acc[4 * u + 2][i], acc[4 * u + 3][i]);
    if (c == 0) {
      rec[rows * HD + 2 * r] = m;
      rec[rows * HD + 2 * r + 1] = l;
    }
  }
};

// ------------------------------------------------------------ fp32, up to 4 rows: FMAs
template <int HD, int NR>
struct FmaMath {
  using T = float;
  using SH = Shape<T, HD>;
  static constexpr int SS = SH::SS, NV = HD / 32;  // 16-byte vectors per lane
  float4 acc[NR][NV];
  float m[NR], l[NR];

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) acc[r][v] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }

  // qs: [NR][HD] queries, lims: [NR] slots per row, both in shared memory
  template <bool SCORES>
  __device__ __forceinline__ void stage(const float* ks, const float* vs, const float* qs, const int* lims, int lane,
                                        int t0, uint32_t live, float qscale, float* srows, int64_t sstride) {
    const int lp = lane & 7;
#pragma unroll
    for (int it = 0; it < SS / 4; ++it) {
      const int slot = it * 4 + (lane >> 3);
      float4 k[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) k[v] = *reinterpret_cast<const float4*>(ks + slot * HD + swz<T, HD>(slot, v * 8 + lp) * 4);
      float s[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        float x = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const float4 q = *reinterpret_cast<const float4*>(qs + r * HD + (v * 8 + lp) * 4);
          x = fmaf(q.x, k[v].x, x);
          x = fmaf(q.y, k[v].y, x);
          x = fmaf(q.z, k[v].z, x);
          x = fmaf(q.w, k[v].w, x);
        }
        x = group_sum<8>(x) * qscale;
        const bool see = ((live >> slot) & 1u) && t0 + slot < lims[r];
        s[r] = see ? x : -INFINITY;
        if (SCORES && lp == 0 && t0 + slot < lims[r]) srows[r * sstride + t0 + slot] = s[r];
      }
      float4 w[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) w[v] = *reinterpret_cast<const float4*>(vs + slot * HD + swz<T, HD>(slot, v * 8 + lp) * 4);
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        if (s[r] == -INFINITY) continue;
        if (s[r] > m[r]) {
          const float corr = exp2f(m[r] - s[r]);  // 0 while m is still -inf
          l[r] *= corr;
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            acc[r][v].x *= corr;
            acc[r][v].y *= corr;
            acc[r][v].z *= corr;
            acc[r][v].w *= corr;
          }
          m[r] = s[r];
        }
        const float p = exp2f(s[r] - m[r]);
        l[r] += p;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          acc[r][v].x = fmaf(p, w[v].x, acc[r][v].x);
          acc[r][v].y = fmaf(p, w[v].y, acc[r][v].y);
          acc[r][v].z = fmaf(p, w[v].z, acc[r][v].z);
          acc[r][v].w = fmaf(p, w[v].w, acc[r][v].w);
        }
      }
    }
  }

  // joins the four slot groups of the warp
  __device__ __forceinline__ void store(float* rec, int lane) {
    auto across = [](float x) {
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
      return x + __shfl_xor_sync(0xFFFFFFFFu, x, 16);
    };
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float M = fmaxf(m[r], __shfl_xor_sync(0xFFFFFFFFu, m[r], 8));
      M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, 16));
      const float w = m[r] == -INFINITY ? 0.f : exp2f(m[r] - M);
      const float L = across(l[r] * w);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float4 a = acc[r][v];
        a = make_float4(across(a.x * w), across(a.y * w), across(a.z * w), across(a.w * w));
        if (lane < 8) *reinterpret_cast<float4*>(rec + r * HD + (v * 8 + lane) * 4) = a;
      }
      if (lane == 0) {
        rec[NR * HD + 2 * r] = M;
        rec[NR * HD + 2 * r + 1] = L;
      }
    }
  }
};

// The math of NR rows per unit.
template <typename T, int HD, int NR>
struct MathOf {
  using type = FmaMath<HD, NR>;
};
template <int HD, int NR>
struct MathOf<__nv_bfloat16, HD, NR> {
  using type = MmaMath<HD>;
};
template <int HD>
struct MathOf<float, HD, kRangeRows> {
  using type = SplitMath<HD>;
};

// NR: rows per unit (bf16: 8 in any case, of which p.rows are used)
template <typename T, int HD, int NR, bool SCORES>
__global__ void __launch_bounds__(kThreads, kRangeCtasPerSm) range_attn_kernel(const RangeParams p) {
  using SH = Shape<T, HD>;
  constexpr int SS = SH::SS, ROWV = SH::ROWV, VEC = SH::VEC;
  constexpr unsigned FULL = 0xFFFFFFFFu;
  constexpr bool FMA = sizeof(T) == 4 && NR < kRangeRows;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint32_t live_s[kRangeWarps][kStages];
  __shared__ int lims[kRangeRows];
  __shared__ float wts[kRangeRows][kRangeMaxCluster + kRangeMaxRecords];  // weights of the records joined
  __shared__ float row_m[kRangeRows], row_inv[kRangeRows];                // joined max and 1 / sum

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int C = p.pieces;
  const int unit = (int)(blockIdx.x / (unsigned)C), piece = (int)(blockIdx.x - (unsigned)unit * C);
  const int grp = unit / p.Hkv, h = unit - grp * p.Hkv;  // sequence or row group
  const int rows = p.rows, max_slots = p.max_pages * p.P;
  unsigned char* ring = smem_raw + warp * kStages * SH::STAGE_BYTES;
  float* crec = reinterpret_cast<float*>(smem_raw + kRangeWarps * kStages * SH::STAGE_BYTES);

  // Dependents start only after this grid's own wait, so that everything before
  // it is visible to them whatever they wait for.  A suffix runs behind the prefix
  // kernel of the same call and relies on that: it reads the cache at once and
  // waits only for the prefix's records, at the end.
  const bool late = p.records > 0;
  if (!late) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }

  // ---- this unit's rows and slots.  Row i is query head h G + g of sequence b.
  const bool shared_prefix = p.mode == kRangePrefix;
  auto row_of = [&](int i, int& b, int& g) -> bool {
    const int x = shared_prefix ? grp * kRangeRows + i : i;
    b = shared_prefix ? x / p.G : grp;
    g = shared_prefix ? x - b * p.G : i;
    return i < rows && b < p.B;
  };
  auto length = [&](int b, bool& bad) -> int {  // 0 for a bad length
    const int n = __ldg(p.seq_lens + b);
    bad = n < 0 || n > max_slots - p.len_add;
    return bad ? 0 : n + p.len_add;
  };
  bool bad;
  Range R;
  if (shared_prefix) {
    int top = 0;
    for (int i = 0; i < kRangeRows; i += p.G) {
      int b, g;
      if (row_of(i, b, g)) top = max(top, min(length(b, bad), p.begin));
    }
    R = make_range<SS>(top, 0, 0);
  } else {
    const int S = length(grp, bad);
    if (bad && h == 0 && piece == 0 && tid == 0) report(p.status, WM_ERR_BOUNDS);
    R = p.mode == kRangeWindow ? make_range<SS>(S, p.sinks, S - p.window)
                               : make_range<SS>(S, 0, p.mode == kRangeSuffix ? p.begin : 0);
  }
  const int32_t* ptab = p.page_table + (shared_prefix ? 0 : (int64_t)(grp / p.rows_per_seq) * p.max_pages);

  const int npieces = C * kRangeWarps, mine = piece * kRangeWarps + warp;
  const int j0 = (int)((int64_t)mine * R.n / npieces);
  const int nmine = (int)((int64_t)(mine + 1) * R.n / npieces) - j0;

  auto first_slot = [&](int j) -> int { return (j < R.n0 ? j : R.f + (j - R.n0)) * SS; };
  // lane l < SS: cache row of slot l of stage j (-1: not seen, or no such page)
  auto row_at = [&](int j) -> int {
    int row = -1;
    if (j < j0 + nmine && lane < SS) {
      const int t = first_slot(j) + lane;
      if (t < R.S && (t < R.a || t >= R.w0)) {
        const int pg = __ldg(ptab + (t >> p.log2P));
        if (pg >= 0 && pg < p.num_pages) row = (pg * p.Hkv + h) * p.P + (t & (p.P - 1));
        else report(p.status, WM_ERR_BOUNDS);
      }
    }
    return row;
  };
  const T* kb = reinterpret_cast<const T*>(p.k_pool);
  const T* vb = reinterpret_cast<const T*>(p.v_pool);
  auto issue = [&](int i, int row) {  // the warp's i-th stage into ring slot i % kStages
    const uint32_t kd = smem_u32(ring + (i % kStages) * SH::STAGE_BYTES);
    const uint32_t mask = __ballot_sync(FULL, row >= 0);
    if (lane == 0) live_s[warp][i % kStages] = mask;
#pragma unroll
    for (int x = 0; x < SH::CHUNKS / 32; ++x) {
      const int q = x * 32 + lane, slot = q / ROWV, c = q - slot * ROWV;
      const int r = __shfl_sync(FULL, row, slot);
      const int64_t off = r >= 0 ? (int64_t)r * HD + c * VEC : 0;
      const uint32_t d = kd + slot * SH::ROW_BYTES + swz<T, HD>(slot, c) * 16;
      cp_async16_zfill(d, kb + off, r >= 0);
      cp_async16_zfill(d + SH::HALF_BYTES, vb + off, r >= 0);
    }
  };

  // one commit group per stage, empty ones included, so that group i is stage i
  int row_next = row_at(j0);
#pragma unroll
  for (int i = 0; i < kStages; ++i) {
    const int row = row_next;
    row_next = row_at(j0 + i + 1);
    if (i < nmine) issue(i, row);
    cp_async_commit();
  }

  // ---- queries and per-row limits
  const T* qbase = reinterpret_cast<const T*>(p.q);
  typename MathOf<T, HD, NR>::type mm;
  float* qs = crec + range_rec(kRangeRows, HD);  // FMA: queries [NR][HD]
  if constexpr (FMA) {
    for (int e = tid; e < NR * HD; e += kThreads) {
      int b, g;
      const bool in = row_of(e / HD, b, g);
      qs[e] = in ? __ldcg(reinterpret_cast<const float*>(p.q) + ((int64_t)b * p.Hq + h * p.G + g) * HD + e % HD) : 0.f;
    }
    if (tid < NR) {
      int b, g;
      lims[tid] = row_of(tid, b, g) ? length(b, bad) : 0;
    }
    __syncthreads();
    mm.init();
  } else {
    int b, g;
    const bool in = row_of(lane >> 2, b, g);
    mm.init(in ? qbase + ((int64_t)b * p.Hq + h * p.G + g) * HD : nullptr, lane, in ? length(b, bad) : 0);
  }

  // scores: in global memory, or this CTA's slots of them in shared memory
  const bool own_mass = SCORES && p.mass != nullptr;
  const int jA = (int)((int64_t)piece * kRangeWarps * R.n / npieces);
  const int jB = (int)((int64_t)(piece + 1) * kRangeWarps * R.n / npieces);  // (kRangeScores: R is [0, S))
  const int64_t sstride = own_mass ? p.mass_slots : p.score_stride;
  float* smass = qs + (FMA ? NR * HD : 0);
  float* srows = nullptr;
  if (SCORES) srows = own_mass ? smass - jA * SS : p.scores + (int64_t)unit * p.G * p.score_stride;
  for (int i = 0; i < nmine; ++i) {
    cp_async_wait<kStages - 1>();
    __syncwarp();
    unsigned char* st = ring + (i % kStages) * SH::STAGE_BYTES;
    const uint32_t live = live_s[warp][i % kStages];
    const int t0 = first_slot(j0 + i);
    if constexpr (FMA) {
      mm.template stage<SCORES>(reinterpret_cast<const float*>(st), reinterpret_cast<const float*>(st + SH::HALF_BYTES),
                                qs, lims, lane, t0, live, p.qscale, srows, sstride);
    } else {
      const uint32_t ks = smem_u32(st);
      float* srow = SCORES && (lane >> 2) < rows ? srows + (lane >> 2) * sstride : nullptr;
      mm.template stage<SCORES>(ks, ks + SH::HALF_BYTES, lane, t0, live, p.qscale, srow);
    }
    __syncwarp();  // every lane is done with this ring slot
    const int row = row_next;
    row_next = row_at(j0 + i + kStages + 1);
    if (i + kStages < nmine) issue(i + kStages, row);
    cp_async_commit();
  }
  cp_async_wait<0>();
  __syncwarp();

  // ---- join the CTA's warps (each warp's state in its idle ring)
  float* wrec = reinterpret_cast<float*>(ring);
  if constexpr (FMA) mm.store(wrec, lane);
  else mm.store(wrec, rows, lane);
  __syncthreads();
  const int E = rows * HD;
  auto warp_rec = [&](int w) -> const float* {
    return reinterpret_cast<const float*>(smem_raw + w * kStages * SH::STAGE_BYTES);
  };
  T* outp = reinterpret_cast<T*>(p.out) + ((int64_t)grp * p.Hq + h * p.G) * HD;  // kRangeWindow
  float* gpart = p.part + (int64_t)blockIdx.x * range_rec(rows, HD);
  const bool final_out = p.mode == kRangeWindow || p.mode == kRangeSuffix || own_mass;
  const bool direct = final_out && C == 1 && p.records == 0 && !own_mass;
  for (int e = tid; e < E; e += kThreads) {
    const int r = e / HD;
    float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < kRangeWarps; ++w) M = fmaxf(M, warp_rec(w)[E + 2 * r]);
#pragma unroll
    for (int w = 0; w < kRangeWarps; ++w) {
      const float mw = warp_rec(w)[E + 2 * r];
      const float wt = mw == -INFINITY ? 0.f : exp2f(mw - M);
      L = fmaf(wt, warp_rec(w)[E + 2 * r + 1], L);
      O = fmaf(wt, warp_rec(w)[e], O);
    }
    if (direct) {
      outp[e] = Elem<T>::from_f(O * (L > 0.f ? 1.f / L : 0.f));
    } else {
      float* rec = final_out ? crec : gpart;
      rec[e] = O;
      if (e == r * HD) {
        rec[E + 2 * r] = M;
        rec[E + 2 * r + 1] = L;
      }
    }
  }
  if (direct || !final_out) return;

  // ---- join the cluster's CTAs through distributed shared memory, and the
  // records of the shared prefix: CTA `piece` finishes its share of the outputs.
  // The last barrier keeps each CTA's shared memory until every reader is done.
  cg::cluster_group cluster = cg::this_cluster();
  if (C > 1) cluster.sync();
  else __syncthreads();
  const int np = p.records;
  const int e0 = piece * E / C, e1 = (piece + 1) * E / C;
  if (np == 0 && !own_mass) {
    for (int e = e0 + tid; e < e1; e += kThreads) {
      const int r = e / HD;
      float mq[kRangeMaxCluster], lq[kRangeMaxCluster], oq[kRangeMaxCluster];
#pragma unroll
      for (int c = 0; c < kRangeMaxCluster; ++c) {
        const float* cr = cluster.map_shared_rank(crec, c < C ? c : 0);
        mq[c] = c < C ? cr[E + 2 * r] : -INFINITY;
        lq[c] = c < C ? cr[E + 2 * r + 1] : 0.f;
        oq[c] = c < C ? cr[e] : 0.f;
      }
      float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
      for (int c = 0; c < kRangeMaxCluster; ++c) M = fmaxf(M, mq[c]);
#pragma unroll
      for (int c = 0; c < kRangeMaxCluster; ++c) {
        const float wt = mq[c] == -INFINITY ? 0.f : exp2f(mq[c] - M);
        L = fmaf(wt, lq[c], L);
        O = fmaf(wt, oq[c], O);
      }
      outp[e] = Elem<T>::from_f(O * (L > 0.f ? 1.f / L : 0.f));
    }
    cluster.sync();
    return;
  }
  if (late) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
  // record i of the prefix for row r: outputs, and (max, sum) at offset `pml`
  auto prefix_rec = [&](int r, int i, int& pml) -> const float* {
    const int x = grp * p.G + r;  // the row among the batch's rows of this kv head
    if (p.tile_records) {
      pml = HD;
      return p.prefix + (((int64_t)h * p.B * p.G + x) * np + i) * tile_rec(HD);
    }
    const int g8 = x / kRangeRows, xr = x - g8 * kRangeRows;
    pml = kRangeRows * HD + 2 * xr - xr * HD;
    return p.prefix + (((int64_t)g8 * p.Hkv + h) * np + i) * range_rec(kRangeRows, HD) + xr * HD;
  };
  for (int r = warp; r < rows; r += kRangeWarps) {
    auto ml = [&](int i) -> float2 {
      if (i < C) {
        const float* cr = C > 1 ? cluster.map_shared_rank(crec, i) : crec;
        return make_float2(cr[E + 2 * r], cr[E + 2 * r + 1]);
      }
      int pml;
      const float* rec = prefix_rec(r, i - C, pml);
      return make_float2(__ldcg(rec + pml), __ldcg(rec + pml + 1));
    };
    float M = -INFINITY, L = 0.f;
    for (int i = lane; i < C + np; i += 32) M = fmaxf(M, ml(i).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(FULL, M, o));
    for (int i = lane; i < C + np; i += 32) {
      const float2 x = ml(i);
      // a record whose every score is NaN has no maximum either, but its sum is NaN
      const float w = x.x == -INFINITY ? (x.y == x.y ? 0.f : 1.f) : exp2f(x.x - M);
      wts[r][i] = w;
      if (w != 0.f) L = fmaf(w, x.y, L);
    }
    L = warp_sum(L);
    if (lane == 0) {
      row_m[r] = M;
      row_inv[r] = L > 0.f ? 1.f / L : 0.f;
    }
  }
  __syncthreads();
  // four outputs per thread; a record without a visible slot may hold no
  // outputs: weight 0, not read
  const int64_t rstride = p.tile_records ? tile_rec(HD) : range_rec(kRangeRows, HD);
  for (int q = piece * (E / 4) / C + tid; q < (piece + 1) * (E / 4) / C; q += kThreads) {
    const int r = q / (HD / 4), x = (q - r * (HD / 4)) * 4;
    float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float w, const float4& v) {
      O.x = fmaf(w, v.x, O.x);
      O.y = fmaf(w, v.y, O.y);
      O.z = fmaf(w, v.z, O.z);
      O.w = fmaf(w, v.w, O.w);
    };
    for (int c = 0; c < C; ++c) {
      const float* cr = C > 1 ? cluster.map_shared_rank(crec, c) : crec;
      add(wts[r][c], *reinterpret_cast<const float4*>(cr + r * HD + x));
    }
    int pml;
    const float* rec = np > 0 ? prefix_rec(r, 0, pml) + x : nullptr;
    constexpr int NB = 10;  // records in flight
    for (int i0 = 0; i0 < np; i0 += NB) {
      float4 v[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i0 + i < np && wts[r][C + i0 + i] != 0.f)
          v[i] = __ldcg(reinterpret_cast<const float4*>(rec + (i0 + i) * rstride));
      }
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (i0 + i < np) add(wts[r][C + i0 + i], v[i]);
    }
    const float inv = row_inv[r];
    T* to = outp + r * HD + x;
    to[0] = Elem<T>::from_f(O.x * inv);
    to[1] = Elem<T>::from_f(O.y * inv);
    to[2] = Elem<T>::from_f(O.z * inv);
    to[3] = Elem<T>::from_f(O.w * inv);
  }
  if (own_mass) {
    // mass[t] += sum_r 2^(s_r[t] - m_r) / l_r over this CTA's slots
    float* mass = p.mass + (int64_t)unit * max_slots;
    for (int t = jA * SS + tid; t < min(jB * SS, R.S); t += kThreads) {
      float w = 0.f;
      for (int r = 0; r < rows; ++r) {
        const float x = srows[r * sstride + t];
        if (x != -INFINITY) w = fmaf(exp2f(x - row_m[r]), row_inv[r], w);
      }
      mass[t] += w;
    }
  }
  if (C > 1) cluster.sync();
}

template <typename T, int HD, int NR>
constexpr size_t range_smem() {
  return (size_t)kRangeWarps * kStages * Shape<T, HD>::STAGE_BYTES +
         (range_rec(kRangeRows, HD) + (sizeof(T) == 4 && NR < kRangeRows ? NR * HD : 0)) * sizeof(float);
}

template <typename T, int HD, int NR, bool SCORES>
inline cudaError_t launch_t(const RangeParams& p, int units, cudaStream_t stream) {
  static size_t smem_set[kSmemOptDevices] = {};
  auto kern = range_attn_kernel<T, HD, NR, SCORES>;
  const size_t smem = range_smem<T, HD, NR>() + (p.mass ? (size_t)p.G * p.mass_slots * sizeof(float) : 0);
  if (cudaError_t e = opt_in_smem(kern, smem, smem_set); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)units * (unsigned)p.pieces);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.pieces;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.mode == kRangeWindow || p.mode == kRangeSuffix || p.mass ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

template <typename T, int HD, int NR>
inline cudaError_t launch_n(const RangeParams& p, int units, cudaStream_t s) {
  return p.mode == kRangeScores ? launch_t<T, HD, NR, true>(p, units, s) : launch_t<T, HD, NR, false>(p, units, s);
}

template <typename T, int HD>
inline cudaError_t launch_d(const RangeParams& p, int units, cudaStream_t s) {
  if constexpr (sizeof(T) == 4) {
    if (p.rows == 1) return launch_n<T, HD, 1>(p, units, s);
    if (p.rows == 2) return launch_n<T, HD, 2>(p, units, s);
    if (p.rows == 4) return launch_n<T, HD, 4>(p, units, s);
  }
  return launch_n<T, HD, kRangeRows>(p, units, s);
}

}  // namespace range_detail

// Per-dtype dispatch (one translation unit each, compiled in parallel).
cudaError_t launch_range_bf16(const RangeParams& p, int d, int units, cudaStream_t s);
cudaError_t launch_range_f32(const RangeParams& p, int d, int units, cudaStream_t s);

}  // namespace wm
