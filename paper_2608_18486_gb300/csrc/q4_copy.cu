// Rows of a cache to 4 bits and back (layout and rounding in q4.h).
//
// Both are bound by HBM: 2 d elements and 2 (d/2 + d/16) bytes per (slot, kv head,
// channel), each read or written once.  A warp takes 16 slots of one (channel,
// sequence, kv head), K and V together, so that it has 8 KB of bf16 rows (d = 128)
// in flight; a lane takes whole groups of 16 elements, so no value crosses lanes.
// Measured: 8 prompts of 511 to 2047 slots, 12 channels of 12 heads of 64, written 78 us and
// read back 76 (6.3 TB/s); 8 contexts of 4097 to 8192 slots, 2 channels of 32 heads of 128,
// read back 308 us (6.7 TB/s).  CTAs of 128 threads: 256, 181 against 172 (the two calls on
// prompts, one head per item); several heads per item 153.
//
// Quantising: y = x / s has to fall on the right side of a rounding border.
//  * bf16: x and (border) * s are both multiples of 2^-8 of their size, so either they
//    are equal or y is 2^-9 of itself off the border.  1 / s rounded to fp32 is s's
//    reciprocal or up to 2^-24 more (8 mantissas), so x * (1 / s) of an equal x is the
//    border or one step above: cut to 16 bits it is the border, and no other y is cut
//    across one.
//  * fp32: x * (1 / s) and one Newton step give the correctly rounded quotient or its
//    neighbour, which may be the border without x being equal; there y is moved to the
//    side that the exact remainder x - y s shows (its last bit set), as in rounding to odd.
#include <type_traits>

#include "common.cuh"
#include "internal.h"
#include "q4.h"

namespace wm {
namespace {

constexpr int kThreads = 128;
constexpr int kCtasPerSm = 128;   // CTAs of a launch per SM at most
constexpr int kItemsPerSm = 128;  // items per SM from which they get more heads
constexpr int kMaxHeads = 4;

__device__ __forceinline__ float scale_value(uint32_t byte) {
  float f;
  asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"((uint16_t)(byte << 7)));
  return f;
}

// The scale nearest to a / 6 (ties to even), a >= 0 and finite.
__device__ __forceinline__ uint32_t scale_byte(float a) {
  const float y = a * 0.16666660f;  // at most a / 6: the byte below it, or one less
  uint32_t byte = y < 6.103515625e-5f ? (uint32_t)(y * 131072.f) : (__float_as_uint(y) >> 20) - (112u << 3);
  byte = min(byte, (uint32_t)kQ4MaxScale);
  // 6 (s0 + s1) / 2, exact in fp32: 5 significant bits times 3
  const float mid = 3.f * (scale_value(byte) + scale_value(byte + 1));
  if (a > mid || (a == mid && (byte & 1u))) ++byte;
  return min(byte, (uint32_t)kQ4MaxScale);
}

// Codes of four pairs (a the lower element), elements already over the scale.
__device__ __forceinline__ uint32_t pack8(const float* y) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return r;
}

// 16 elements (as they lie in memory) to codes and a scale byte.
__device__ __forceinline__ uint2 quantise(const uint4 (&v)[4], uint32_t& byte) {  // fp32
  float x[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) Elem<float>::unpack(v[i], x + 4 * i);
  uint32_t top = 0;  // (bit patterns of magnitudes order like the values, NaN last)
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  if (top >= 0x7F800000u) {
    byte = 0xFFu;
    return make_uint2(0u, 0u);
  }
  byte = scale_byte(__uint_as_float(top));
  if (byte == 0) return make_uint2(0u, 0u);
  const float s = scale_value(byte), r = 1.f / s;
  float y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float a = fabsf(x[i]);
    float q = a * r;
    q = fmaf(fmaf(-q, s, a), r, q);
    const float rest = fmaf(-q, s, a);
    const uint32_t u = __float_as_uint(q);
    if (rest != 0.f && (u & 1u) == 0 && u != 0) q = __uint_as_float(rest > 0.f ? u + 1 : u - 1);
    y[i] = __uint_as_float(__float_as_uint(q) | (__float_as_uint(x[i]) & 0x80000000u));
  }
  return make_uint2(pack8(y), pack8(y + 8));
}
__device__ __forceinline__ uint2 quantise(const uint4 (&v)[2], uint32_t& byte) {  // bf16
  const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
  uint32_t m[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) m[i] = w[i] & 0x7FFF7FFFu;
  const uint32_t pair = __vmaxu2(__vimax3_u16x2(__vimax3_u16x2(m[0], m[1], m[2]), m[3], m[4]), __vimax3_u16x2(m[5], m[6], m[7]));
  const uint32_t top = max(pair << 16, pair & 0xFFFF0000u);
  if (top >= 0x7F800000u) {
    byte = 0xFFu;
    return make_uint2(0u, 0u);
  }
  byte = scale_byte(__uint_as_float(top));
  if (byte == 0) return make_uint2(0u, 0u);
  const float r = 1.f / scale_value(byte);
  float y[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 q = __fmul2_rn(make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u)), make_float2(r, r));
    y[2 * i] = __uint_as_float(__float_as_uint(q.x) & 0xFFFFFF00u);
    y[2 * i + 1] = __uint_as_float(__float_as_uint(q.y) & 0xFFFFFF00u);
  }
  return make_uint2(pack8(y), pack8(y + 8));
}

// Values (f16 pairs) of the 4 bytes of w times s.
__device__ __forceinline__ void values8(uint32_t w, uint32_t s2, float* f) {
  uint32_t r[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm("{\n\t.reg .b32 p;\n\t.reg .b16 lo, hi;\n\t"
        "mul.rn.f16x2 p, %2, %3;\n\t"
        "mov.b32 {lo, hi}, p;\n\t"
        "cvt.f32.f16 %0, lo;\n\t"
        "cvt.f32.f16 %1, hi;\n\t}"
        : "=f"(f[2 * i]), "=f"(f[2 * i + 1])
        : "r"(r[i]), "r"(s2));
}

// 32 bytes, in one access where they lie on a 32-byte boundary: a lane's group of bf16
// elements is a whole sector then (two accesses of 16 bytes each touch half of it;
// 8 contexts of 8192 slots, 2 channels of 32 heads of 128, read back: 384 against 308 us).
__device__ __forceinline__ void load32(const void* p, bool wide, uint4& a, uint4& b) {
  if (wide) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
                 : "l"(p)
                 : "memory");
  } else {
    a = __ldcs(reinterpret_cast<const uint4*>(p));
    b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
  }
}
__device__ __forceinline__ void store32(void* p, bool wide, const uint4& a, const uint4& b) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z),
                 "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = a;
    reinterpret_cast<uint4*>(p)[1] = b;
  }
}

// 16 consecutive elements as they lie in memory.
template <typename T>
struct Row16 {
  static constexpr int NV = 16 * (int)sizeof(T) / 16;
  uint4 v[NV];
  __device__ __forceinline__ void load(const T* p, bool wide) {
#pragma unroll
    for (int i = 0; i < NV; i += 2) load32(reinterpret_cast<const uint4*>(p) + i, wide, v[i], v[i + 1]);
  }
};
// Values as fp16 pairs, in which they are exact as well.
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ void put16_half(void* p, bool wide, const float (&f)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = half_pair(f[2 * i], f[2 * i + 1]);
  store32(p, wide, make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7]));
}
__device__ __forceinline__ uint4 bits4(const float* f) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ void put16(float* p, bool wide, const float (&f)[16]) {
  store32(p, wide, bits4(f), bits4(f + 4));
  store32(p + 8, wide, bits4(f + 8), bits4(f + 12));
}
__device__ __forceinline__ void put16(__nv_bfloat16* p, bool wide, const float (&f)[16]) {
  uint32_t w[8];  // (exact: the values have at most 6 significant bits)
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = __byte_perm(__float_as_uint(f[2 * i]), __float_as_uint(f[2 * i + 1]), 0x7632);
  store32(p, wide, make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7]));
}

// What a warp takes at once: 16 slots from t0 on, [f, l) of them, of `heads` kv heads
// from h on, channel c, sequence b.
struct Item {
  int c, b, h, t0, f, l;
};
__device__ __forceinline__ bool item_at(const Q4CopyParams& p, int it, int lane, Item& x) {
  const int blocks = (p.Hkv + p.heads - 1) / p.heads;
  x.h = it % blocks * p.heads;
  it /= blocks;
  const int step = it % p.steps;
  it /= p.steps;
  x.b = it % p.B;
  x.c = it / p.B;
  const int slots = p.max_pages * p.P;
  x.f = p.first ? __ldg(p.first + x.b) : 0;
  bool bad;
  if (p.last) {
    x.l = __ldg(p.last + x.b);
    bad = x.f < 0 || x.l < x.f || x.l > slots;
  } else {  // slot 0 is the dummy's
    x.l = x.f + 1;
    bad = x.f < 1 || x.f >= slots;
  }
  if (bad) x.l = x.f = 0;
  const bool longer = x.l - x.f > p.span;
  if (longer) x.l = x.f + p.span;
  if ((bad || longer) && x.c == 0 && x.h == 0 && step == 0 && lane == 0) report(p.status, WM_ERR_BOUNDS);
  x.t0 = (x.f / kQ4Step + step) * kQ4Step;
  return x.t0 < x.l;
}

// Physical pages of slot t of an item; false (and reported): one out of range.
__device__ __forceinline__ bool pages_of(const Q4CopyParams& p, const Item& x, int t, int& row_page, int& q4_page) {
  const int64_t entry = (int64_t)x.b * p.max_pages + (t >> p.log2P);
  q4_page = __ldg(p.q4_table + entry);
  row_page = p.rows_at == kQ4Paged ? __ldg(p.row_table + entry) : 0;
  if (q4_page >= 0 && q4_page < p.q4_pages && row_page >= 0 && row_page < p.row_pages) return true;
  report(p.status, WM_ERR_BOUNDS);
  return false;
}

// Addresses of 16 consecutive slots in pages of at least 16 (of slot t alone: r its
// place in its tile).
template <int HD>
struct Place {
  int64_t row;    // element offset of the first row
  uint8_t* tile;  // 4-bit tile
  int r;
  __device__ __forceinline__ bool at(const Q4CopyParams& p, const Item& x, int t) {
    int pr, pq;
    if (!pages_of(p, x, t, pr, pq)) return false;
    const int in = t & (p.P - 1);
    if (p.rows_at == kQ4Staged) {
      row = (((int64_t)x.c * p.B + x.b) * p.Hkv + x.h) * HD;
    } else {
      const int64_t page = p.rows_at == kQ4Dense ? (int64_t)x.b * p.max_pages + (t >> p.log2P) : (int64_t)x.c * p.row_pages + pr;
      row = ((page * p.Hkv + x.h) * p.P + in) * HD;
    }
    tile = p.pool + (((int64_t)x.c * p.q4_pages + pq) * p.Hkv + x.h) * p.page_bytes +
           (int64_t)(in >> p.log2tile) * p.tile_bytes;
    r = in & (p.tile - 1);
    return true;
  }
  // K (X = 0) or V codes and scale of group g of the slot
  __device__ __forceinline__ uint2* codes(const Q4CopyParams& p, int X, int g) const {
    return reinterpret_cast<uint2*>(tile + (X * p.tile + r) * (HD / 2)) + g;
  }
  __device__ __forceinline__ uint8_t* scale(const Q4CopyParams& p, int X, int g) const {
    return tile + p.tile * HD + (X * p.tile + r) * (HD / kQ4Group) + g;
  }
};

// The groups of an item: group q = 32 i + lane of a head's 16 rows.  BIG (pages of at
// least 16 slots, rows in pages): rows, codes and scales of a head are contiguous.
template <int HD, bool BIG>
struct Groups {
  static constexpr int GR = HD / kQ4Group, NI = HD / 32;  // groups per row; per lane and pool
  static constexpr uint32_t ALL = (1u << NI) - 1;
  Place<HD> place[BIG ? 1 : NI];
  uint32_t on;  // bit i: the lane's group i is copied
  int heads;
  // The warp's first item from `it` on that has slots to copy; it: where it is.
  __device__ __forceinline__ bool next(const Q4CopyParams& p, int& it, int items, int nwarps, int lane) {
    for (; it < items; it += nwarps) {
      Item x;
      if (!item_at(p, it, lane, x)) continue;
      heads = min(p.heads, p.Hkv - x.h);
      if (BIG) {
        if (!place[0].at(p, x, x.t0)) continue;
        place[0].row += lane * kQ4Group;
        place[0].tile += lane * 8;
      }
      on = 0;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int t = x.t0 + (i * 32 + lane) / GR;
        if (t >= x.f && t < x.l && (BIG || place[i].at(p, x, t))) on |= 1u << i;
      }
      return true;
    }
    return false;
  }
  __device__ __forceinline__ void next_head(const Q4CopyParams& p) {
#pragma unroll
    for (int i = 0; i < (BIG ? 1 : NI); ++i) {
      place[i].row += p.rows_at == kQ4Staged ? HD : p.P * HD;
      place[i].tile += p.page_bytes;
    }
  }
  __device__ __forceinline__ int64_t row(int i, int lane) const {
    return BIG ? place[0].row + i * 32 * kQ4Group : place[i].row + (i * 32 + lane) % GR * kQ4Group;
  }
  __device__ __forceinline__ uint2* codes(const Q4CopyParams& p, int X, int i, int lane) const {
    if (BIG) return reinterpret_cast<uint2*>(place[0].tile + X * kQ4Step * (HD / 2) + i * 256);
    return place[i].codes(p, X, (i * 32 + lane) % GR);
  }
  __device__ __forceinline__ uint8_t* scale(const Q4CopyParams& p, int X, int i, int lane) const {
    if (BIG) return place[0].tile - lane * 7 + kQ4Step * HD + X * kQ4Step * GR + i * 32;
    return place[i].scale(p, X, (i * 32 + lane) % GR);
  }
};

// CTAs per SM by registers: a lane holds a head's rows, K and V (fp32: one of them).  us of 8
// prompts of 511 to 2047 slots, pages of 16 / 8: fp32, 4 channels of 16 heads of 128, 3 CTAs
// 170 / 188, 4 with 106 / 298 bytes of spills 172 / 202; bf16, 12 channels of 12 heads of 64, 6 CTAs
// with 16 / 98 bytes of spills 78 / 90, 5 without them 81 / 87; 4 channels of 32 heads of 128,
// 3 CTAs 154 / 171 (68 bytes in pages of 8), 2 154 / 211.
constexpr int write_ctas(int hd) { return hd == 64 ? 6 : hd == 96 ? 4 : 3; }

template <typename T, int HD, bool BIG>
__global__ void __launch_bounds__(kThreads, write_ctas(HD)) q4_write_kernel(const Q4CopyParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // (Dependents start when this grid ends: attention that starts beside it would crowd on
  // the SMs that have most room, 304 units of 2048 slots behind a write 40 us instead of 29.)
  using G = Groups<HD, BIG>;
  const int lane = threadIdx.x & 31, nwarps = (int)gridDim.x * (kThreads / 32);
  G at;
  auto head = [&](auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    constexpr int XS = sizeof(T) == 4 ? 1 : 2;  // pools at once
#pragma unroll 1
    for (int X0 = 0; X0 < 2; X0 += XS) {
      Row16<T> v[XS][G::NI];
#pragma unroll
      for (int X = 0; X < XS; ++X)
#pragma unroll
        for (int i = 0; i < G::NI; ++i)
          if (WHOLE || ((at.on >> i) & 1u))
            v[X][i].load(reinterpret_cast<const T*>(X0 + X ? p.v_rows : p.k_rows) + at.row(i, lane), p.wide);
#pragma unroll
      for (int X = 0; X < XS; ++X)
#pragma unroll
        for (int i = 0; i < G::NI; ++i) {
          if (!WHOLE && !((at.on >> i) & 1u)) continue;
          uint32_t byte;
          *at.codes(p, X0 + X, i, lane) = quantise(v[X][i].v, byte);
          *at.scale(p, X0 + X, i, lane) = (uint8_t)byte;
        }
    }
  };
  for (int it = (int)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); at.next(p, it, p.items, nwarps, lane); it += nwarps) {
    const bool whole = __all_sync(0xFFFFFFFFu, at.on == G::ALL);
    for (int h = 0; h < at.heads; ++h) {
      if (whole) head(std::true_type{});
      else head(std::false_type{});
      at.next_head(p);
    }
  }
}

// VHALF: V rows as fp16 instead of bf16.
template <typename T, int HD, bool BIG, bool VHALF>
__global__ void __launch_bounds__(kThreads) q4_read_kernel(const Q4CopyParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  using G = Groups<HD, BIG>;
  const int lane = threadIdx.x & 31, nwarps = (int)gridDim.x * (kThreads / 32);
  G at;
  auto head = [&](auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    uint2 w[2][G::NI];
    uint32_t s[2][G::NI];
#pragma unroll
    for (int X = 0; X < 2; ++X)
#pragma unroll
      for (int i = 0; i < G::NI; ++i)
        if (WHOLE || ((at.on >> i) & 1u)) {
          w[X][i] = __ldcs(at.codes(p, X, i, lane));
          s[X][i] = __ldcs(at.scale(p, X, i, lane));
        }
#pragma unroll
    for (int X = 0; X < 2; ++X)
#pragma unroll
      for (int i = 0; i < G::NI; ++i) {
        if (!WHOLE && !((at.on >> i) & 1u)) continue;
        float f[16];
        const uint32_t s2 = s[X][i] * 0x00800080u;
        values8(w[X][i].x, s2, f);
        values8(w[X][i].y, s2, f + 8);
        T* const to = reinterpret_cast<T*>(X ? p.v_rows : p.k_rows) + at.row(i, lane);
        if (VHALF && X == 1) put16_half(to, p.wide, f);
        else put16(to, p.wide, f);
      }
  };
  for (int it = (int)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); at.next(p, it, p.items, nwarps, lane); it += nwarps) {
    const bool whole = __all_sync(0xFFFFFFFFu, at.on == G::ALL);
    for (int h = 0; h < at.heads; ++h) {
      if (whole) head(std::true_type{});
      else head(std::false_type{});
      at.next_head(p);
    }
  }
}

template <typename Kern>
cudaError_t launch(Kern kern, Q4CopyParams p, int sms, cudaStream_t s) {
  p.wide = (((uintptr_t)p.k_rows | (uintptr_t)p.v_rows) & 31) == 0 ? 1 : 0;
  // heads per item: the item's place costs as much as a head's groups, while there are
  // items for every warp
  const int64_t all = (int64_t)p.k * p.B * p.steps * p.Hkv, per = all / ((int64_t)sms * kItemsPerSm);
  p.heads = (int)(per < 1 ? 1 : per < kMaxHeads ? per : kMaxHeads);
  p.items = p.k * p.B * p.steps * ((p.Hkv + p.heads - 1) / p.heads);
  const int64_t ctas = (p.items + kThreads / 32 - 1) / (kThreads / 32), most = (int64_t)sms * kCtasPerSm;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ctas < most ? ctas : most));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

// 16 slots of a head lie together (rows staged one per sequence do not).
bool whole_tiles(const Q4CopyParams& p) { return p.P >= kQ4Step && p.rows_at != kQ4Staged; }

template <typename T, int HD>
cudaError_t launch_write(const Q4CopyParams& p, int sms, cudaStream_t s) {
  return whole_tiles(p) ? launch(q4_write_kernel<T, HD, true>, p, sms, s) : launch(q4_write_kernel<T, HD, false>, p, sms, s);
}

template <typename T, int HD>
cudaError_t launch_read(const Q4CopyParams& p, int sms, cudaStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (p.rows_at == kQ4Dense)
      return whole_tiles(p) ? launch(q4_read_kernel<T, HD, true, true>, p, sms, s)
                            : launch(q4_read_kernel<T, HD, false, true>, p, sms, s);
  }
  return whole_tiles(p) ? launch(q4_read_kernel<T, HD, true, false>, p, sms, s)
                        : launch(q4_read_kernel<T, HD, false, false>, p, sms, s);
}

}  // namespace

cudaError_t launch_q4_write(const Q4CopyParams& p, int dtype, int d, int sms, cudaStream_t s) {
  if (dtype == WM_DT_F32)
    return d == 64 ? launch_write<float, 64>(p, sms, s) : d == 96 ? launch_write<float, 96>(p, sms, s)
                                                                  : launch_write<float, 128>(p, sms, s);
  return d == 64 ? launch_write<__nv_bfloat16, 64>(p, sms, s) : d == 96 ? launch_write<__nv_bfloat16, 96>(p, sms, s)
                                                                        : launch_write<__nv_bfloat16, 128>(p, sms, s);
}

cudaError_t launch_q4_read(const Q4CopyParams& p, int dtype, int d, int sms, cudaStream_t s) {
  if (dtype == WM_DT_F32)
    return d == 64 ? launch_read<float, 64>(p, sms, s) : d == 96 ? launch_read<float, 96>(p, sms, s)
                                                                 : launch_read<float, 128>(p, sms, s);
  return d == 64 ? launch_read<__nv_bfloat16, 64>(p, sms, s) : d == 96 ? launch_read<__nv_bfloat16, 96>(p, sms, s)
                                                                       : launch_read<__nv_bfloat16, 128>(p, sms, s);
}

}  // namespace wm
