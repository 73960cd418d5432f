// Rows of a cache to 4 bits and back (layout and rounding in q4.h).
//
// Both are bound by HBM: 2 d elements and 2 (d/2 + d/16) bytes per (slot, kv head,
// channel), each read or written once.  A warp takes 16 slots of one (channel,
// sequence, kv head), K and V together, so that it has 8 KB of bf16 rows (d = 128)
// in flight; a lane takes whole groups of 16 elements, so no value crosses lanes.
//
// Quantising: y = x / s has to fall on the right side of a rounding border.  q = x * (1 / s)
// and one Newton step give the correctly rounded quotient or its neighbour.  A bf16 x
// and (border) * s are both multiples of 2^-8 of their size, so either they are equal,
// and y is the border itself, or y is well off it.  An fp32 x can lie within half a step
// of y from the border; there y is moved to the side that the exact remainder x - y s
// shows (its last bit set), as in rounding to odd.
#include "common.cuh"
#include "internal.h"
#include "q4.h"

namespace wm {
namespace {

constexpr int kThreads = 256;

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

// 16 elements to codes and a scale byte.
template <bool F32>
__device__ __forceinline__ uint2 quantise(const float (&x)[16], uint32_t& byte) {
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
    float v = a * r;
    v = fmaf(fmaf(-v, s, a), r, v);
    if (F32) {
      const float rest = fmaf(-v, s, a);
      const uint32_t u = __float_as_uint(v);
      if (rest != 0.f && (u & 1u) == 0 && u != 0) v = __uint_as_float(rest > 0.f ? u + 1 : u - 1);
    }
    y[i] = __uint_as_float(__float_as_uint(v) | (__float_as_uint(x[i]) & 0x80000000u));
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

// 16 consecutive elements as they lie in memory.
template <typename T>
struct Row16 {
  static constexpr int NV = 16 * (int)sizeof(T) / 16;
  uint4 v[NV];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void get(float (&f)[16]) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) Elem<T>::unpack(v[i], f + i * Elem<T>::kVec);
  }
};
__device__ __forceinline__ void put16(float* p, const float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    reinterpret_cast<float4*>(p)[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
}
__device__ __forceinline__ void put16(__nv_bfloat16* p, const float (&f)[16]) {
  uint32_t w[8];  // (exact: the values have at most 6 significant bits)
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = __byte_perm(__float_as_uint(f[2 * i]), __float_as_uint(f[2 * i + 1]), 0x7632);
  reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
  reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// A warp's 16 slots: channel c, sequence b, kv head h, from slot t0; [f, l) of them.
struct Item {
  int c, b, h, t0, f, l;
};
__device__ __forceinline__ bool item_at(const Q4CopyParams& p, int it, int lane, Item& x) {
  x.h = it % p.Hkv;
  it /= p.Hkv;
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

// Addresses of slot t of an item; false (and reported): a page id out of range.
template <int HD>
struct Place {
  int64_t row;      // element offset of the row
  uint8_t* tile;    // 4-bit tile
  int r;            // the slot's place in it
  __device__ __forceinline__ bool at(const Q4CopyParams& p, const Item& x, int t) {
    const int lp = t >> p.log2P, in = t & (p.P - 1);
    const int64_t entry = (int64_t)x.b * p.max_pages + lp;
    const int pq = __ldg(p.q4_table + entry);
    int pr = x.b;
    if (p.rows_at == kQ4Paged) pr = __ldg(p.row_table + entry);
    if (pq < 0 || pq >= p.q4_pages || pr < 0 || pr >= p.row_pages) {
      report(p.status, WM_ERR_BOUNDS);
      return false;
    }
    if (p.rows_at == kQ4Staged) {
      row = (((int64_t)x.c * p.B + x.b) * p.Hkv + x.h) * HD;
    } else {
      const int64_t page = p.rows_at == kQ4Dense ? entry : (int64_t)x.c * p.row_pages + pr;
      row = ((page * p.Hkv + x.h) * p.P + in) * HD;
    }
    tile = p.pool + (((int64_t)x.c * p.q4_pages + pq) * p.Hkv + x.h) * p.page_bytes +
           (int64_t)(in >> p.log2tile) * p.tile_bytes;
    r = in & (p.tile - 1);
    return true;
  }
  // K (X = 0) or V codes and scale of group g
  __device__ __forceinline__ uint2* codes(const Q4CopyParams& p, int X, int g) const {
    return reinterpret_cast<uint2*>(tile + (X * p.tile + r) * (HD / 2)) + g;
  }
  __device__ __forceinline__ uint8_t* scale(const Q4CopyParams& p, int X, int g) const {
    return tile + p.tile * HD + (X * p.tile + r) * (HD / kQ4Group) + g;
  }
};

template <typename T, int HD>
__global__ void __launch_bounds__(kThreads) q4_write_kernel(const Q4CopyParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int GR = HD / kQ4Group, NI = HD / 32;  // groups per row; per lane and pool
  const int lane = threadIdx.x & 31, nwarps = (int)gridDim.x * (kThreads / 32);
  const int items = p.k * p.B * p.steps * p.Hkv;
  for (int it = (int)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); it < items; it += nwarps) {
    Item x;
    if (!item_at(p, it, lane, x)) continue;
    Place<HD> at[NI];
    bool on[NI];
    Row16<T> v[2][NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int t = x.t0 + (i * 32 + lane) / GR;
      on[i] = t >= x.f && t < x.l && at[i].at(p, x, t);
    }
#pragma unroll
    for (int X = 0; X < 2; ++X)
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (on[i])
          v[X][i].load(reinterpret_cast<const T*>(X ? p.v_rows : p.k_rows) + at[i].row + (i * 32 + lane) % GR * kQ4Group);
#pragma unroll
    for (int X = 0; X < 2; ++X)
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        if (!on[i]) continue;
        const int g = (i * 32 + lane) % GR;
        float f[16];
        v[X][i].get(f);
        uint32_t byte;
        *at[i].codes(p, X, g) = quantise<sizeof(T) == 4>(f, byte);
        *at[i].scale(p, X, g) = (uint8_t)byte;
      }
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kThreads) q4_read_kernel(const Q4CopyParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int GR = HD / kQ4Group, NI = HD / 32;
  const int lane = threadIdx.x & 31, nwarps = (int)gridDim.x * (kThreads / 32);
  const int items = p.k * p.B * p.steps * p.Hkv;
  for (int it = (int)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); it < items; it += nwarps) {
    Item x;
    if (!item_at(p, it, lane, x)) continue;
    Place<HD> at[NI];
    bool on[NI];
    uint2 w[2][NI];
    uint32_t s[2][NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int t = x.t0 + (i * 32 + lane) / GR;
      on[i] = t >= x.f && t < x.l && at[i].at(p, x, t);
    }
#pragma unroll
    for (int X = 0; X < 2; ++X)
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (on[i]) {
          const int g = (i * 32 + lane) % GR;
          w[X][i] = __ldcs(at[i].codes(p, X, g));
          s[X][i] = __ldcs(at[i].scale(p, X, g));
        }
#pragma unroll
    for (int X = 0; X < 2; ++X)
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        if (!on[i]) continue;
        float f[16];
        const uint32_t s2 = s[X][i] * 0x00800080u;
        values8(w[X][i].x, s2, f);
        values8(w[X][i].y, s2, f + 8);
        put16(reinterpret_cast<T*>(X ? p.v_rows : p.k_rows) + at[i].row + (i * 32 + lane) % GR * kQ4Group, f);
      }
  }
}

template <typename Kern>
cudaError_t launch(Kern kern, const Q4CopyParams& p, int sms, cudaStream_t s) {
  const int64_t items = (int64_t)p.k * p.B * p.steps * p.Hkv, ctas = (items + kThreads / 32 - 1) / (kThreads / 32);
  const int64_t most = (int64_t)sms * 16;
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

}  // namespace

cudaError_t launch_q4_write(const Q4CopyParams& p, int dtype, int d, int sms, cudaStream_t s) {
  if (dtype == WM_DT_F32) {
    if (d == 64) return launch(q4_write_kernel<float, 64>, p, sms, s);
    if (d == 96) return launch(q4_write_kernel<float, 96>, p, sms, s);
    return launch(q4_write_kernel<float, 128>, p, sms, s);
  }
  if (d == 64) return launch(q4_write_kernel<__nv_bfloat16, 64>, p, sms, s);
  if (d == 96) return launch(q4_write_kernel<__nv_bfloat16, 96>, p, sms, s);
  return launch(q4_write_kernel<__nv_bfloat16, 128>, p, sms, s);
}

cudaError_t launch_q4_read(const Q4CopyParams& p, int dtype, int d, int sms, cudaStream_t s) {
  if (dtype == WM_DT_F32) {
    if (d == 64) return launch(q4_read_kernel<float, 64>, p, sms, s);
    if (d == 96) return launch(q4_read_kernel<float, 96>, p, sms, s);
    return launch(q4_read_kernel<float, 128>, p, sms, s);
  }
  if (d == 64) return launch(q4_read_kernel<__nv_bfloat16, 64>, p, sms, s);
  if (d == 96) return launch(q4_read_kernel<__nv_bfloat16, 96>, p, sms, s);
  return launch(q4_read_kernel<__nv_bfloat16, 128>, p, sms, s);
}

}  // namespace wm
