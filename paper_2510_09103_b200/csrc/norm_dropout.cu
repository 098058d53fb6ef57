// Dropout, and RMS normalisation with the residual's addition and the branch's dropout, forward and backward.
//
//   s = residual + drop(x)      rstd = 1 / sqrt(mean(s^2) + eps)      y = s rstd w      q = e4m3(y 448 / amax|y|)
//   xh = s rstd    ds = rstd (dy w - xh mean(dy w xh)) + dsum    dx = drop(ds)    dw = sum over rows of dy xh
//
// Every element is read and written once (the norm's gradient reads rows above 8192 columns twice); a row is held in registers
// between its reduction and its output (up to 32768 columns), in chunks of eight elements: one 16-byte access in bf16, one
// counter of the generator.  Dropout is bound by HBM, the norm and its gradient by issue slots and by the reduction between a
// row's loads and its stores; odd widths by the two blocks of the generator that a chunk takes.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "device_math.cuh"
#include "op_checks.h"
#include "philox.cuh"

namespace adapm {
namespace {

constexpr int64_t kMaxCols = 32768;

// ---- eight elements of a row -------------------------------------------------------------------------
// VEC: the chunk starts on 16 bytes; a chunk cut by the end of the row goes element by element.  (Plain loads: an output may
// lie on an input, and what an earlier launch wrote must not be asked for before this one may start.)
// A chunk is held as it was read until it is used: in bf16 that is half the registers.
template <typename T> struct Elem;
template <> struct Elem<float> {
  struct raw8 { float4 a, b; };
  static __device__ __forceinline__ float get(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
  static __device__ __forceinline__ raw8 load(const float* p) { return raw8{*reinterpret_cast<const float4*>(p), *(reinterpret_cast<const float4*>(p) + 1)}; }
  static __device__ __forceinline__ raw8 zero() { return raw8{make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)}; }
  static __device__ __forceinline__ void set(raw8& r, int e, float x) { (e < 4 ? (&r.a.x)[e] : (&r.b.x)[e - 4]) = x; }
  static __device__ __forceinline__ void unpack(const raw8& r, float* x) {
    x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w; x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
  }
  static __device__ __forceinline__ void put8(float* p, const float* x) { store8f(p, x); }
};
template <> struct Elem<uint16_t> {
  using raw8 = uint4;
  static __device__ __forceinline__ float get(const uint16_t* p) { return bf16_bits_to_float(*p); }
  static __device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }
  static __device__ __forceinline__ raw8 load(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }
  static __device__ __forceinline__ raw8 zero() { return make_uint4(0, 0, 0, 0); }
  static __device__ __forceinline__ void set(raw8& r, int e, float x) {      // (x is a bf16 number)
    uint32_t& w = (&r.x)[e >> 1];
    w |= e & 1 ? __float_as_uint(x) & 0xffff0000u : __float_as_uint(x) >> 16;
  }
  static __device__ __forceinline__ void unpack(const raw8& r, float* x) { GradBF16::unpack(r, x); }
  static __device__ __forceinline__ void put8(uint16_t* p, const float* x) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
};

// How the rows of a call's matrices lie.
//   SCALAR   anyhow: element by element
//   VEC      every row starts on 16 bytes: chunk g is columns 8 g to 8 g + 7, one access but for the end of the row
//   SHIFTED  the rows are one pitch apart that is no multiple of eight elements (odd widths), from aligned bases and alike in all
//            matrices: the chunks of a row are the windows of eight elements between multiples of eight elements from the
//            base, so that chunk g is columns 8 g - m to 8 g - m + 7 with m = row * pitch mod 8, again one access but for the two
//            ends.  (A chunk then takes bits of two groups of the generator.)
// With dropout, element by element -> windows, us: 16373 x 1601 in bf16 norm 121 -> 62, its gradient 152 -> 118, dropout 70 -> 48;
// 3200 x 8191 136 -> 62, 238 -> 116, 70 -> 45; 8186 x 1601 in fp32 76 -> 39, 103 -> 62, 48 -> 29.  (Reading the cut chunks whole as well and
// clearing what is not the row's was slower, by up to a quarter.)
enum : int { SCALAR = 0, VEC = 1, SHIFTED = 2 };

// The chunk's first column (below zero for a cut first chunk) and the part [lo, hi) of its eight elements that exist.
struct Span { int c0, lo, hi; };
template <int FORM>
__device__ __forceinline__ Span span_of(int g, int m, int cols) {
  if (FORM != SHIFTED) return Span{8 * g, 0, min(8, cols - 8 * g)};
  const int c0 = 8 * g - m;
  return Span{c0, max(0, -c0), min(8, cols - c0)};
}

// `row`: the row's first element.  Elements that do not exist are zero.
template <int FORM, typename T>
__device__ __forceinline__ typename Elem<T>::raw8 fetch8(const T* row, const Span& s) {
  const T* const p = row + s.c0;
  if (FORM != SCALAR && (FORM == VEC || s.lo == 0) && s.hi >= 8) return Elem<T>::load(p);
  typename Elem<T>::raw8 r = Elem<T>::zero();
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < s.hi && (FORM != SHIFTED || e >= s.lo)) Elem<T>::set(r, e, Elem<T>::get(p + e));
  return r;
}
template <int FORM>
__device__ __forceinline__ void load_weight8(const void* w, int f32, const Span& s, float* x) {      // (w is aligned, the windows of a row are not)
  if (FORM == SHIFTED) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = 0.f;
      if (e >= s.lo && e < s.hi) x[e] = f32 ? static_cast<const float*>(w)[s.c0 + e] : bf16_bits_to_float(static_cast<const uint16_t*>(w)[s.c0 + e]);
    }
    return;
  }
  if (f32) Elem<float>::unpack(fetch8<FORM>(static_cast<const float*>(w), s), x);
  else Elem<uint16_t>::unpack(fetch8<FORM>(static_cast<const uint16_t*>(w), s), x);
}
template <int FORM, typename T>
__device__ __forceinline__ void store8(T* row, const Span& s, const float* x) {
  T* const p = row + s.c0;
  if (FORM != SCALAR && (FORM == VEC || s.lo == 0) && s.hi >= 8) {
    Elem<T>::put8(p, x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < s.hi && (FORM != SHIFTED || e >= s.lo)) Elem<T>::put(p + e, x[e]);
  }
}

// The generator's bits of a chunk: element e has the e-th 16 of them.  `first`: number of the row's first group.
template <int FORM>
__device__ __forceinline__ Philox4 bits_of(const DropRule& d, const DropKey& k, uint64_t first, int g, int m) {
  const Philox4 b = drop_bits(d, k, first + (uint64_t)g);
  if (FORM != SHIFTED || m == 0) return b;
  // the last m elements of the group before, then the first 8 - m of this one: eight halfwords from halfword 8 - m on
  const Philox4 a = drop_bits(d, k, first + (uint64_t)g - 1);
  const int from = 8 - m, w = from >> 1;
  uint32_t v[8] = {a.w[0], a.w[1], a.w[2], a.w[3], b.w[0], b.w[1], b.w[2], b.w[3]};
#pragma unroll
  for (int i = 0; i < 7; ++i) v[i] = w & 1 ? v[i + 1] : v[i];
#pragma unroll
  for (int i = 0; i < 6; ++i) v[i] = w & 2 ? v[i + 2] : v[i];
  Philox4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = __funnelshift_r(v[i], v[i + 1], from & 1 ? 16 : 0);
  return r;
}

// ---- dropout -------------------------------------------------------------------------------------------

constexpr int kDropUnits = 2;      // groups of eight per thread

struct DropArgs {
  const void* x;
  const void* residual;
  void* y;
  int64_t x_ld, r_ld, y_ld, cols, groups, slots, total;     // groups of eight columns per row, chunks per row and in all
  DropRule drop;
};

// Bound by HBM: 65536 x 1600 in bf16 with a residual 95 us = 6.6 TB/s, the copy rate, with two thirds of the issue slots taken
// (a group of eight costs 20 32-bit products with 64-bit results and about 100 other instructions).  175 us in its first form,
// which looped over the groups with 64 registers, found every row by a 64-bit division and made the bits after the loads.
// DENSE: the rows lie one behind the other and hold whole groups, so that group i is at element 8 i.
template <typename T, int FORM, bool DENSE>
__global__ void __launch_bounds__(256) dropout_kernel(const DropArgs a) {
  wait_for_previous_kernel();
  const DropKey key = drop_key(a.drop);
  const T* const x = static_cast<const T*>(a.x);
  const T* const res = static_cast<const T*>(a.residual);
  T* const y = static_cast<T*>(a.y);
  typename Elem<T>::raw8 xs[kDropUnits], rs[kDropUnits];
  Philox4 bits[kDropUnits];
  int64_t row[kDropUnits];
  Span span[kDropUnits];
  const int64_t i0 = (int64_t)blockIdx.x * (256 * kDropUnits) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kDropUnits; ++u) {
    const int64_t i = i0 + u * 256;
    span[u] = Span{0, 0, 0};
    row[u] = 0;
    if (i >= a.total) continue;
    if (DENSE) {
      xs[u] = Elem<T>::load(x + 8 * i);
      if (res) rs[u] = Elem<T>::load(res + 8 * i);
      bits[u] = drop_bits(a.drop, key, (uint64_t)i);
      continue;
    }
    row[u] = a.total <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)a.slots) : i / a.slots;
    const int64_t g = i - row[u] * a.slots;
    const int m = FORM == SHIFTED ? (int)((row[u] * a.x_ld) & 7) : 0;
    // (wider than 2^31: columns are counted from the chunk)
    const int64_t c0 = 8 * g - m;
    span[u] = Span{0, FORM == SHIFTED ? (int)max((int64_t)0, -c0) : 0, (int)max((int64_t)0, min((int64_t)8, a.cols - c0))};
    xs[u] = fetch8<FORM>(x + row[u] * a.x_ld + c0, span[u]);
    if (res) rs[u] = fetch8<FORM>(res + row[u] * a.r_ld + c0, span[u]);
    bits[u] = bits_of<FORM>(a.drop, key, (uint64_t)(row[u] * a.groups + g), 0, m);
    row[u] = row[u] * a.y_ld + c0;                       // where the output goes
  }
#pragma unroll
  for (int u = 0; u < kDropUnits; ++u) {
    const int64_t i = i0 + u * 256;
    if (i >= a.total) continue;
    float v[8];
    Elem<T>::unpack(xs[u], v);
    if (a.drop.mode) drop8(a.drop, bits[u], v);
    if (res) {
      float r[8];
      Elem<T>::unpack(rs[u], r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
    if (DENSE) Elem<T>::put8(y + 8 * i, v);
    else store8<FORM>(y + row[u], span[u], v);
  }
}

// ---- sums and maxima over the threads of a row ---------------------------------------------------------
// WARP: a row belongs to one warp; else to the whole CTA.  `red` is one of two arrays that alternate, so that one barrier per
// reduction is enough.
template <bool WARP>
__device__ __forceinline__ float row_sum(float x, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (WARP) return x;
  const int warps = blockDim.x >> 5;
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = (int)(threadIdx.x & 31) < warps ? red[threadIdx.x & 31] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
template <bool WARP>
__device__ __forceinline__ float row_max(float x, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  if (WARP) return x;
  const int warps = blockDim.x >> 5;
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = (int)(threadIdx.x & 31) < warps ? red[threadIdx.x & 31] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}

// ---- RMS norm, forward -----------------------------------------------------------------------------------

struct NormArgs {
  const void* x;
  const void* residual;
  const void* weight;
  void* sum;
  void* y;
  uint8_t* y8;
  float* scales;
  float* rstd;
  int64_t x_ld, r_ld, s_ld, y_ld, y8_ld, rows;
  int32_t cols, groups, slots, q8_group, n_scales, weight_f32;      // groups of eight columns, chunks of a row
  float eps;
  DropRule drop;
};

__device__ __forceinline__ uint32_t pack_e4m3x4(const float* x) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1]), "f"(x[0]));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3]), "f"(x[2]));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// The scale of values whose greatest magnitude is m, and what they are multiplied by: m / 448 and 448 / m, one where m is 0.  The
// quotient by the hardware's reciprocal (an ulp off) where that has a normal result, else by the division, and at most the
// greatest float (zeros stay zeros).
__device__ __forceinline__ float scale_of(float m) { return m > 0.f ? m * (1.f / 448.f) : 1.f; }
__device__ __forceinline__ float inverse_scale_of(float m) {
  if (m >= 1e-30f && m <= 1e30f) return __fdividef(448.f, m);
  return m > 0.f ? fminf(448.f / m, 3.402823466e38f) : 1.f;
}
__device__ __forceinline__ void times(float* x, float f) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float2 t = mul2(make_float2(x[e], x[e + 1]), make_float2(f, f));
    x[e] = t.x; x[e + 1] = t.y;
  }
}

// s stays in 32 bits for the statistic and the output and is rounded only where it is stored.
// 16384 x 1600 in bf16: 36 us without dropout (5.8 TB/s), 42.5 with it; 8192 x 4096 to 8 bits with a scale per 128 columns 45 us (5.2
// TB/s).  DRAM is busy for half of that time and the issue slots for 70 to 75 %: what is left is the row's reduction between its
// loads and its stores.
template <typename T, int NC, bool WARP, int FORM, bool DROP>
__global__ void __launch_bounds__(WARP ? 128 : NC == 4 ? 1024 : 512) rmsnorm_forward_kernel(const NormArgs a) {
  __shared__ float red[2][32];
  wait_for_previous_kernel();
  const int team = WARP ? 32 : (int)blockDim.x, me = WARP ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
  const int64_t row = WARP ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  if (row >= a.rows) return;                       // (a whole warp, or never)
  const T* const x = static_cast<const T*>(a.x) + row * a.x_ld;
  const T* const res = a.residual ? static_cast<const T*>(a.residual) + row * a.r_ld : nullptr;
  T* const sum = a.sum ? static_cast<T*>(a.sum) + row * a.s_ld : nullptr;
  T* const y = a.y ? static_cast<T*>(a.y) + row * a.y_ld : nullptr;
  const int m = FORM == SHIFTED ? (int)((row * a.x_ld) & 7) : 0;
  auto span = [&](int i) { return span_of<FORM>(me + i * team, m, a.cols); };
  typename Elem<T>::raw8 xs[NC], rs[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    xs[i] = rs[i] = Elem<T>::zero();
    if (me + i * team < a.slots) {
      xs[i] = fetch8<FORM>(x, span(i));
      if (res) rs[i] = fetch8<FORM>(res, span(i));
    }
  }
  float s[NC][8];
  float2 sq = make_float2(0.f, 0.f);
  // (with four chunks there are no registers for their bits too)
  constexpr bool kAhead = DROP && NC < 4;
  constexpr int kBits = kAhead ? NC : 1;
  Philox4 bits[kBits];
  const DropKey key = DROP ? drop_key(a.drop) : DropKey{0, 0};
  if (kAhead) {
#pragma unroll
    for (int i = 0; i < NC; ++i) bits[i % kBits] = bits_of<FORM>(a.drop, key, (uint64_t)row * a.groups, me + i * team, m);
  }
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    Elem<T>::unpack(xs[i], s[i]);
    if (me + i * team < a.slots) {
      if (DROP) drop8(a.drop, kAhead ? bits[i % kBits] : bits_of<FORM>(a.drop, key, (uint64_t)row * a.groups, me + i * team, m), s[i]);
      if (res) {
        float r[8];
        Elem<T>::unpack(rs[i], r);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float2 t = add2(make_float2(s[i][e], s[i][e + 1]), make_float2(r[e], r[e + 1]));
          s[i][e] = t.x; s[i][e + 1] = t.y;
        }
      }
      if (sum) store8<FORM>(sum, span(i), s[i]);
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float2 t = make_float2(s[i][e], s[i][e + 1]);
        sq = fma2(t, t, sq);
      }
    }
  }
  const float rstd = 1.f / sqrtf(row_sum<WARP>(sq.x + sq.y, red[0]) / (float)a.cols + a.eps);
  if (a.rstd && me == 0) a.rstd[row] = rstd;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int g = me + i * team;
    if (g < a.slots) {
      float w[8];
      load_weight8<FORM>(a.weight, a.weight_f32, span(i), w);
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float2 t = mul2(mul2(make_float2(s[i][e], s[i][e + 1]), make_float2(rstd, rstd)), make_float2(w[e], w[e + 1]));
        s[i][e] = t.x; s[i][e + 1] = t.y;
      }
      if (y) store8<FORM>(y, span(i), s[i]);
    }
    if (!a.y8) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(s[i][e]));
    if (FORM != SHIFTED && a.q8_group) {           // a group of 128 columns: sixteen neighbouring lanes
      float m = top;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      top = 0.f;
      if (g < a.groups) {
        if ((g & 15) == 0) a.scales[row * a.n_scales + (g >> 4)] = scale_of(m);
        times(s[i], inverse_scale_of(m));
      }
    }
  }
  if (!a.y8) return;
  if (!a.q8_group) {
    const float m = row_max<WARP>(top, red[1]), inv = inverse_scale_of(m);
    if (me == 0) a.scales[row] = scale_of(m);
#pragma unroll
    for (int i = 0; i < NC; ++i) times(s[i], inv);
  }
  uint8_t* const q = a.y8 + row * a.y8_ld;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    if (me + i * team >= a.slots) continue;
    const Span t = span(i);
    const uint2 v = make_uint2(pack_e4m3x4(s[i]), pack_e4m3x4(s[i] + 4));
    if (FORM != SCALAR && t.lo == 0 && t.hi >= 8) {
      *reinterpret_cast<uint2*>(q + t.c0) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e >= t.lo && e < t.hi) q[t.c0 + e] = (uint8_t)((e < 4 ? v.x : v.y) >> (8 * (e & 3)));
    }
  }
}

// ---- RMS norm, backward ------------------------------------------------------------------------------------

struct NormGradArgs {
  const void* dy;
  const void* dsum;
  const void* sum;
  const float* rstd;
  const void* weight;
  void* dres;
  void* dx;
  float* partial;                // [CTAs][cols], or null: no gradient of the weight
  int64_t dy_ld, s_ld, r_ld, x_ld, rows;
  int32_t cols, groups, slots, weight_f32;
  DropRule drop;
};

// A CTA takes row after row; a thread has the same columns in each, whose share of dw it keeps.  The next row's elements are
// on their way while a row is worked on.  16384 x 1600 in bf16 with dropout 62.5 us (4.2 TB/s), of which the sum of the CTAs'
// shares takes 6; 79 us without the look-ahead.  Not kept: rows copied ahead into shared memory (cp.async, three rows deep: 70),
// three CTAs of 256 threads per SM with the registers of two (86, spills), five of 128 with 96 registers (75).  NC = 4 (rows above
// 8192 columns): dw alone fills the registers, so a row is read a second time, out of L2.
template <typename T, int NC, int FORM, bool DROP>
__global__ void __launch_bounds__(NC == 1 ? 256 : NC == 2 ? 512 : 1024) rmsnorm_backward_kernel(const NormGradArgs a) {
  using E = Elem<T>;
  constexpr bool kTwice = NC == 4;
  constexpr int kHeld = kTwice ? 1 : NC;
  __shared__ float red[2][32];
  wait_for_previous_kernel();
  const int team = (int)blockDim.x, me = (int)threadIdx.x;
  const DropKey key = DROP ? drop_key(a.drop) : DropKey{0, 0};
  typename E::raw8 dys[kHeld], ss[kHeld], more[kHeld];
  float w[kHeld][8];
  float2 dw[NC][4];
  const int m = FORM == SHIFTED ? (int)(((int64_t)blockIdx.x * a.dy_ld) & 7) : 0;      // (of all its rows: see grad_form)
  auto span = [&](int i) {
    const Span t = span_of<FORM>(me + i * team, m, a.cols);
    return me + i * team < a.slots ? t : Span{t.c0, 0, 0};
  };
  auto fetch = [&](int i, int64_t row, bool with_more) {
    const Span t = span(i);
    dys[i % kHeld] = fetch8<FORM>(static_cast<const T*>(a.dy) + row * a.dy_ld, t);
    ss[i % kHeld] = fetch8<FORM>(static_cast<const T*>(a.sum) + row * a.s_ld, t);
    if (kTwice) load_weight8<FORM>(a.weight, a.weight_f32, t, w[0]);
    if (with_more) more[i % kHeld] = a.dsum ? fetch8<FORM>(static_cast<const T*>(a.dsum) + row * a.s_ld, t) : E::zero();
  };
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    if (!kTwice) {
      load_weight8<FORM>(a.weight, a.weight_f32, span(i), w[i % kHeld]);
      fetch(i, blockIdx.x, true);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) dw[i][e] = make_float2(0.f, 0.f);
  }
  float rstd_next = a.rstd[blockIdx.x];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const int64_t next = row + gridDim.x;
    const float rstd = rstd_next;
    const float2 rstd2 = make_float2(rstd, rstd);
    // with g = rstd dy w: mean(dy w xh) = sum(g s) / cols, ds = g - s (rstd^2 sum(g s) / cols) + dsum
    float2 g8[kHeld][4], s8[kHeld][4], extra[kHeld][4], c2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if (kTwice) fetch(i, row, false);
      const int h = i % kHeld;
      float dy[8], sv[8], ev[8];
      E::unpack(dys[h], dy);
      E::unpack(ss[h], sv);
      if (!kTwice) E::unpack(more[h], ev);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 d = mul2(make_float2(dy[2 * e], dy[2 * e + 1]), rstd2);
        s8[h][e] = make_float2(sv[2 * e], sv[2 * e + 1]);
        if (!kTwice) extra[h][e] = make_float2(ev[2 * e], ev[2 * e + 1]);
        dw[i][e] = fma2(d, s8[h][e], dw[i][e]);
        g8[h][e] = mul2(d, make_float2(w[h][2 * e], w[h][2 * e + 1]));
        c2 = fma2(g8[h][e], s8[h][e], c2);
      }
    }
    if (next < a.rows) {
      rstd_next = a.rstd[next];
      if (!kTwice) {
#pragma unroll
        for (int i = 0; i < NC; ++i) fetch(i, next, true);
      }
    }
    const float c = row_sum<false>(c2.x + c2.y, red[turn]) * (rstd * rstd) / (float)a.cols;
    const float2 minus = make_float2(-c, -c);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int h = i % kHeld;
      if (me + i * team >= a.slots) continue;
      if (kTwice) {
        fetch(i, row, true);
        float dy[8], sv[8], ev[8];
        E::unpack(dys[h], dy);
        E::unpack(ss[h], sv);
        E::unpack(more[h], ev);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s8[h][e] = make_float2(sv[2 * e], sv[2 * e + 1]);
          extra[h][e] = make_float2(ev[2 * e], ev[2 * e + 1]);
          g8[h][e] = mul2(mul2(make_float2(dy[2 * e], dy[2 * e + 1]), rstd2), make_float2(w[h][2 * e], w[h][2 * e + 1]));
        }
      }
      float ds[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 d = fma2(s8[h][e], minus, g8[h][e]);
        ds[2 * e] = d.x + extra[h][e].x;
        ds[2 * e + 1] = d.y + extra[h][e].y;
      }
      if (a.dres) store8<FORM>(static_cast<T*>(a.dres) + row * a.r_ld, span(i), ds);
      if (a.dx) {
        if (DROP) drop8(a.drop, bits_of<FORM>(a.drop, key, (uint64_t)row * a.groups, me + i * team, m), ds);
        store8<FORM>(static_cast<T*>(a.dx) + row * a.x_ld, span(i), ds);
      }
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    float out[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) { out[2 * e] = dw[i][e].x; out[2 * e + 1] = dw[i][e].y; }
    const Span t = span(i);
    float* const p = a.partial + (int64_t)blockIdx.x * a.cols + t.c0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= t.lo && e < t.hi) p[e] = out[e];
  }
}

// dw = the sum of the CTAs' shares, in a fixed order: 32 columns per CTA, 32 warps that share the rows.
template <typename G>
__global__ void __launch_bounds__(1024) column_sum_kernel(const float* partial, int n_partial, int cols, G* out, int accumulate) {
  __shared__ float sums[32][33];
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = (int)blockIdx.x * 32 + lane;
  float x = 0.f;
  if (col < cols) {
#pragma unroll 8
    for (int p = warp; p < n_partial; p += 32) x += partial[(int64_t)p * cols + col];
  }
  sums[warp][lane] = x;
  __syncthreads();
  x = sums[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  const int c = (int)blockIdx.x * 32 + warp;
  if (lane == 0 && c < cols) {
    if (accumulate) x += Elem<G>::get(out + c);
    Elem<G>::put(out + c, x);
  }
}

// ---- host ------------------------------------------------------------------------------------------------

int drop_rule(float p, uint64_t seed, uint64_t offset, const uint64_t* step, DropRule& d) {
  if (!(p >= 0.f && p <= 1.f)) return ADAPM_ERANGE;
  const uint32_t least = (uint32_t)std::lrint((double)p * 65536.0);
  d.cut = least << 16;
  d.mode = least == 0 ? 0u : least < 65536u ? 1u : 2u;
  d.factor = d.mode == 2 ? 0.f : (float)(65536.0 / (65536.0 - least));
  d.seed_lo = (uint32_t)seed; d.seed_hi = (uint32_t)(seed >> 32);
  d.offset = offset; d.step = step;
  return ADAPM_OK;
}

int check_desc(const adapm_rmsnorm& d, DropRule& drop) {
  if (d.rows < 0 || d.cols <= 0) return ADAPM_EINVAL;
  if (d.rows > INT32_MAX || d.cols > kMaxCols) return ADAPM_ERANGE;
  if (!known_type(d.dtype) || !known_type(d.weight_dtype)) return ADAPM_EINVAL;
  if (d.q8_group != 0 && d.q8_group != 128) return ADAPM_EINVAL;
  if (!(d.eps >= 0.f) || !std::isfinite(d.eps)) return ADAPM_ERANGE;
  return drop_rule(d.drop_p, d.seed, d.offset, d.step, drop);
}

struct Pitched { const void* p; int64_t ld; int64_t bytes; };

// Pitches hold a row, pointers are multiples of their element; `form`: how the rows lie (elements of 8 bits: their eights on 8 bytes).
int check_rows(std::initializer_list<Pitched> all, int64_t rows, int64_t cols, int& form) {
  bool aligned = true, bases = true, alike = true;
  int64_t eighth = -1;
  for (const Pitched& t : all) {
    if (!t.p) continue;
    if (t.ld < cols) return ADAPM_EINVAL;
    if (rows > 1 && t.ld > INT64_MAX / 8 / rows) return ADAPM_ERANGE;
    if ((uintptr_t)t.p % (uintptr_t)t.bytes) return ADAPM_EALIGN;
    const int64_t unit = t.bytes == 1 ? 8 : 16;
    bases = bases && (uintptr_t)t.p % (uintptr_t)unit == 0;
    aligned = aligned && (rows <= 1 || t.ld * t.bytes % unit == 0);
    alike = alike && (eighth < 0 || t.ld % 8 == eighth);
    eighth = t.ld % 8;
  }
  form = !bases ? SCALAR : aligned ? VEC : alike ? SHIFTED : SCALAR;
  return ADAPM_OK;
}
// Chunks that a row may have.
int64_t slots_of(int64_t cols, int form) { return (cols + 7) / 8 + (form == SHIFTED && cols % 8 != 1 ? 1 : 0); }

int sm_count(int device, int* sms) {
  ADAPM_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
  return ADAPM_OK;
}

// Threads of a CTA that has `groups` chunks of a row, nc at most per thread.
unsigned threads_for(int64_t groups, int nc) { return (unsigned)(((groups + nc - 1) / nc + 31) / 32 * 32); }

template <typename T, int NC, bool WARP, int FORM, bool DROP>
cudaError_t forward_launch(const NormArgs& a, cudaStream_t s) {
  return launch_chained(true, rmsnorm_forward_kernel<T, NC, WARP, FORM, DROP>, (unsigned)(WARP ? (a.rows + 3) / 4 : a.rows),
                        WARP ? 128u : threads_for(a.slots, NC), 0, s, a);
}

// A warp per row up to 512 columns, else a CTA, with two chunks of eight per thread, where there are rows for all SMs; one chunk
// per thread where there are few (a row then takes less time).  Two reads and two writes of 67 MB each, bf16: 65536 x 512 42 us
// (a CTA per row: 69), 32768 x 1024 43 (warp 44, one chunk 45), 16384 x 2048 42 (one chunk 46), 8192 x 4096 43 (one chunk 48):
// 0.95 of the copy rate.  CTAs that take row after row with the next row's elements on their way: 45 to 48.
template <typename T, int FORM, bool DROP>
cudaError_t forward_form(const NormArgs& a, int sms, cudaStream_t s) {
  const bool many = a.rows >= 8 * (int64_t)sms;
  if (FORM == VEC && many && a.slots <= 32) return forward_launch<T, 1, true, FORM, DROP>(a, s);
  if (FORM == VEC && many && a.slots <= 64) return forward_launch<T, 2, true, FORM, DROP>(a, s);
  if (a.slots <= 512 && (FORM == SCALAR || !many || a.slots <= 64)) return forward_launch<T, 1, false, FORM, DROP>(a, s);
  if (FORM != SCALAR && a.slots <= 1024) return forward_launch<T, 2, false, FORM, DROP>(a, s);
  return forward_launch<T, 4, false, FORM, DROP>(a, s);
}

struct GradForm { int nc; unsigned threads; int ctas; };
// Two chunks of eight per thread where there are rows for all SMs (16384 rows of 1600 in bf16 with dropout 63 us, one chunk per
// thread 69), one where there are few (a row then takes less time), four above 8192 columns.  As many CTAs as the registers of
// an SM hold at once: with four of 128 threads 63 us, three 80, five 84 (the fifth waits for one of the four to end).  Where the
// rows' windows are shifted, a multiple of eight, so that all rows of a CTA (one grid apart) are shifted alike.
GradForm grad_form(int64_t rows, int64_t groups, int form, int sms) {
  GradForm f;
  f.nc = groups > 1024 ? 4 : groups > 256 || rows >= 4 * (int64_t)sms ? 2 : 1;
  f.threads = threads_for(groups, f.nc);
  const int per = std::max(1, (f.nc == 4 ? 1024 : 512) / (int)f.threads);
  f.ctas = (int)std::min<int64_t>(rows, (int64_t)sms * per);
  if (form == SHIFTED && f.ctas < rows) f.ctas = (int)std::min<int64_t>(rows, std::max(8, f.ctas / 8 * 8));
  return f;
}

template <typename T, int FORM, bool DROP>
cudaError_t backward_form(const NormGradArgs& a, const GradForm& f, cudaStream_t s) {
  if (f.nc == 1) return launch_chained(true, rmsnorm_backward_kernel<T, 1, FORM, DROP>, (unsigned)f.ctas, f.threads, 0, s, a);
  if (f.nc == 2) return launch_chained(true, rmsnorm_backward_kernel<T, 2, FORM, DROP>, (unsigned)f.ctas, f.threads, 0, s, a);
  return launch_chained(true, rmsnorm_backward_kernel<T, 4, FORM, DROP>, (unsigned)f.ctas, f.threads, 0, s, a);
}

}  // namespace
}  // namespace adapm

using namespace adapm;

extern "C" int adapm_dropout(const void* x, const void* residual, void* y, int32_t dtype, int64_t rows, int64_t cols, int64_t x_ld,
                             int64_t residual_ld, int64_t y_ld, float p, uint64_t seed, uint64_t offset, const uint64_t* step,
                             adapm_stream stream) {
  if (rows < 0 || cols < 0 || !known_type(dtype)) return ADAPM_EINVAL;
  DropArgs a;
  int rc = drop_rule(p, seed, offset, step, a.drop);
  if (rc != ADAPM_OK || rows == 0 || cols == 0) return rc;
  if (!x || !y) return ADAPM_EINVAL;
  if (cols > INT64_MAX / 64 / rows) return ADAPM_ERANGE;
  const int64_t eb = type_bytes(dtype);
  int form;
  rc = check_rows({{x, x_ld, eb}, {residual, residual_ld, eb}, {y, y_ld, eb}}, rows, cols, form);
  if (rc != ADAPM_OK) return rc;
  if ((uintptr_t)step % 8) return ADAPM_EALIGN;
  const Place out = matrix_at(y, rows, y_ld, cols, eb);
  if (!apart_or_same(out, matrix_at(x, rows, x_ld, cols, eb)) || !apart_or_same(out, matrix_at(residual, rows, residual_ld, cols, eb)) ||
      share(out, vector_at(step, 1, 8))) {
    set_error_text("adapm_dropout: the output lies over an input, but not element on element");
    return ADAPM_EINVAL;
  }
  int device;
  rc = check_on_this_device({x, residual, y, step}, &device);
  if (rc != ADAPM_OK) return rc;
  a.x = x; a.residual = residual; a.y = y;
  a.x_ld = x_ld; a.r_ld = residual_ld; a.y_ld = y_ld; a.cols = cols;
  a.groups = (cols + 7) / 8; a.slots = slots_of(cols, form); a.total = rows * a.slots;
  cudaStream_t s = (cudaStream_t)stream;
  if (a.total > (int64_t)INT32_MAX * (256 * kDropUnits)) return ADAPM_ERANGE;
  const unsigned grid = (unsigned)((a.total + 256 * kDropUnits - 1) / (256 * kDropUnits));
  const bool dense = form == VEC && cols % 8 == 0 && x_ld == cols && y_ld == cols && (!residual || residual_ld == cols);
#define ADAPM_DROP(T)                                                                                                \
  (dense ? launch_chained(true, dropout_kernel<T, VEC, true>, grid, 256, 0, s, a)                                    \
   : form == VEC ? launch_chained(true, dropout_kernel<T, VEC, false>, grid, 256, 0, s, a)                           \
   : form == SHIFTED ? launch_chained(true, dropout_kernel<T, SHIFTED, false>, grid, 256, 0, s, a)                   \
                     : launch_chained(true, dropout_kernel<T, SCALAR, false>, grid, 256, 0, s, a))
  ADAPM_CUDA(dtype == ADAPM_TYPE_F32 ? ADAPM_DROP(float) : ADAPM_DROP(uint16_t));
#undef ADAPM_DROP
  return ADAPM_OK;
}

extern "C" int adapm_rmsnorm_forward(const adapm_rmsnorm* d, const void* x, const void* residual, const void* weight, void* sum, void* y,
                                     void* y8, float* y8_scales, float* rstd, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  NormArgs a;
  int rc = check_desc(*d, a.drop);
  if (rc != ADAPM_OK || d->rows == 0) return rc;
  if (!x || !weight || (!y && !y8 && !sum) || (y8 && !y8_scales)) return ADAPM_EINVAL;
  const int64_t eb = type_bytes(d->dtype);
  int form;
  rc = check_rows({{x, d->x_ld, eb}, {residual, d->residual_ld, eb}, {sum, d->sum_ld, eb}, {y, d->y_ld, eb}, {y8, d->y8_ld, 1}}, d->rows,
                  d->cols, form);
  if (rc != ADAPM_OK) return rc;
  if ((uintptr_t)weight % 16 || slots_of(d->cols, form) > kMaxCols / 8 || (form == SHIFTED && y8 && d->q8_group)) form = SCALAR;
  if ((uintptr_t)weight % (uintptr_t)type_bytes(d->weight_dtype) || (uintptr_t)y8_scales % 4 || (uintptr_t)rstd % 4 || (uintptr_t)d->step % 8) return ADAPM_EALIGN;
  const Place px = matrix_at(x, d->rows, d->x_ld, d->cols, eb), pr = matrix_at(residual, d->rows, d->residual_ld, d->cols, eb),
              ps = matrix_at(sum, d->rows, d->sum_ld, d->cols, eb), py = matrix_at(y, d->rows, d->y_ld, d->cols, eb),
              pq = matrix_at(y8, d->rows, d->y8_ld, d->cols, 1), pw = vector_at(weight, d->cols, type_bytes(d->weight_dtype)),
              pscales = vector_at(y8 ? y8_scales : nullptr, d->rows * (d->q8_group ? (d->cols + 127) / 128 : 1), 4), prstd = vector_at(rstd, d->rows, 4),
              pstep = vector_at(d->step, 1, 8);
  bool apart = !share(ps, py) && !share(pscales, prstd);
  for (const Place& out : {ps, py}) apart = apart && apart_or_same(out, px) && apart_or_same(out, pr) && !share(out, pw) && !share(out, pstep);
  for (const Place& t : {px, pr, ps, py, pw, pstep}) apart = apart && !share(pq, t) && !share(pscales, t) && !share(prstd, t);
  apart = apart && !share(pq, pscales) && !share(pq, prstd);
  if (!apart) {
    set_error_text("adapm_rmsnorm_forward: an output lies over an input, but not element on element, or over another output");
    return ADAPM_EINVAL;
  }
  int device, sms;
  rc = check_on_this_device({x, residual, weight, sum, y, y8, y8_scales, rstd, d->step}, &device);
  if (rc == ADAPM_OK) rc = sm_count(device, &sms);
  if (rc != ADAPM_OK) return rc;
  a.x = x; a.residual = residual; a.weight = weight; a.sum = sum; a.y = y; a.y8 = (uint8_t*)y8; a.scales = y8_scales; a.rstd = rstd;
  a.x_ld = d->x_ld; a.r_ld = d->residual_ld; a.s_ld = d->sum_ld; a.y_ld = d->y_ld; a.y8_ld = d->y8_ld; a.rows = d->rows;
  a.cols = (int32_t)d->cols; a.groups = (int32_t)((d->cols + 7) / 8); a.slots = (int32_t)slots_of(d->cols, form); a.q8_group = d->q8_group;
  a.n_scales = d->q8_group ? (int32_t)((d->cols + 127) / 128) : 1;
  a.eps = d->eps;
  a.weight_f32 = d->weight_dtype == ADAPM_TYPE_F32;
  const bool f32 = d->dtype == ADAPM_TYPE_F32;
  cudaStream_t s = (cudaStream_t)stream;
#define ADAPM_NORM_OF(T, DROP)                                                                                         \
  (form == VEC ? forward_form<T, VEC, DROP>(a, sms, s) : form == SHIFTED ? forward_form<T, SHIFTED, DROP>(a, sms, s) : forward_form<T, SCALAR, DROP>(a, sms, s))
#define ADAPM_NORM(DROP) (f32 ? ADAPM_NORM_OF(float, DROP) : ADAPM_NORM_OF(uint16_t, DROP))
  ADAPM_CUDA(a.drop.mode ? ADAPM_NORM(true) : ADAPM_NORM(false));
#undef ADAPM_NORM
#undef ADAPM_NORM_OF
  return ADAPM_OK;
}

extern "C" size_t adapm_rmsnorm_backward_scratch_bytes(const adapm_rmsnorm* d) {
  DropRule drop;
  if (!d || check_desc(*d, drop) != ADAPM_OK) return 0;
  // the largest grid of any row length, on a device of up to 256 SMs
  // The number of SMs is not known here.  256 at most are used, and there are never more CTAs than this many or than rows.
  const int64_t groups = (d->cols + 7) / 8;
  auto per = [](int64_t slots) { return slots > 1024 ? (int64_t)(1024 / threads_for(slots, 4)) : std::max<int64_t>(1, 512 / threads_for(slots, 2)); };
  const int64_t ctas = std::min<int64_t>(std::max<int64_t>(d->rows, 1), 256 * std::max(per(groups), per(std::min<int64_t>(groups + 1, kMaxCols / 8))));
  return (size_t)round_up(ctas * d->cols * 4, 256);
}

extern "C" int adapm_rmsnorm_backward(const adapm_rmsnorm* d, const void* dy, const void* dsum, const void* sum, const float* rstd,
                                      const void* weight, void* dresidual, void* dx, void* dweight, int32_t dweight_dtype,
                                      int32_t accumulate, void* scratch, size_t scratch_bytes, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  NormGradArgs a;
  int rc = check_desc(*d, a.drop);
  if (rc != ADAPM_OK) return rc;
  if (!dresidual && !dx && !dweight) return ADAPM_EINVAL;
  if (dweight && !known_type(dweight_dtype)) return ADAPM_EINVAL;
  const int64_t gb = type_bytes(dweight_dtype);
  if (dweight && (uintptr_t)dweight % (uintptr_t)gb) return ADAPM_EALIGN;
  cudaStream_t s = (cudaStream_t)stream;
  int device, sms;
  if (d->rows == 0) {                          // no row: the gradient of the weight is zero
    if (!dweight || accumulate) return ADAPM_OK;
    rc = check_on_this_device({dweight}, &device);
    if (rc != ADAPM_OK) return rc;
    ADAPM_CUDA(cudaMemsetAsync(dweight, 0, (size_t)(d->cols * gb), s));
    return ADAPM_OK;
  }
  if (!dy || !sum || !rstd || !weight) return ADAPM_EINVAL;
  const int64_t eb = type_bytes(d->dtype);
  int form;
  rc = check_rows({{dy, d->y_ld, eb}, {dsum, d->sum_ld, eb}, {sum, d->sum_ld, eb}, {dresidual, d->residual_ld, eb}, {dx, d->x_ld, eb}},
                  d->rows, d->cols, form);
  if (rc != ADAPM_OK) return rc;
  if ((uintptr_t)weight % 16 || slots_of(d->cols, form) > kMaxCols / 8) form = SCALAR;
  // In short rows the two cut chunks, which go element by element, fall to one warp and are most of its work; above 96 chunks they
  // fall to two.  bf16 with dropout, by elements and by windows, us: 49554 x 529 174 and 227, 39420 x 665 157 and 194, 34447 x 761
  // 143 and 172, 33825 x 775 143 and 128, 29224 x 897 137 and 114, 25575 x 1025 163 and 146 (without dropout 761 columns 114 and
  // 141, 775 114 and 98).  In fp32 windows are faster there too: 24777 x 529 108 and 90.
  if (form == SHIFTED && d->dtype == ADAPM_TYPE_BF16 && d->cols < 768) form = SCALAR;
  if ((uintptr_t)weight % (uintptr_t)type_bytes(d->weight_dtype) || (uintptr_t)rstd % 4 || (uintptr_t)d->step % 8) return ADAPM_EALIGN;
  const Place pdy = matrix_at(dy, d->rows, d->y_ld, d->cols, eb), pds = matrix_at(dsum, d->rows, d->sum_ld, d->cols, eb),
              ps = matrix_at(sum, d->rows, d->sum_ld, d->cols, eb), pdr = matrix_at(dresidual, d->rows, d->residual_ld, d->cols, eb),
              pdx = matrix_at(dx, d->rows, d->x_ld, d->cols, eb), pw = vector_at(weight, d->cols, type_bytes(d->weight_dtype)),
              pdw = vector_at(dweight, d->cols, gb), prstd = vector_at(rstd, d->rows, 4), pstep = vector_at(d->step, 1, 8);
  bool apart = !share(pdr, pdx);
  for (const Place& out : {pdr, pdx}) {
    for (const Place& in : {pdy, pds, ps}) apart = apart && apart_or_same(out, in);
    for (const Place& t : {pw, pdw, prstd, pstep}) apart = apart && !share(out, t);
  }
  for (const Place& in : {pdy, pds, ps, pw, prstd, pstep}) apart = apart && !share(pdw, in);
  if (!apart) {
    set_error_text("adapm_rmsnorm_backward: an output lies over an input, but not element on element, or over another output");
    return ADAPM_EINVAL;
  }
  if (dweight) {
    if (!scratch) return ADAPM_EINVAL;
    if ((uintptr_t)scratch % 256) return ADAPM_EALIGN;
    const size_t needed = adapm_rmsnorm_backward_scratch_bytes(d);
    if (scratch_bytes < needed) return ADAPM_ENOWORKSPACE;
    for (const Place& t : {pdy, pds, ps, pdr, pdx, pw, pdw, prstd, pstep}) apart = apart && !share(vector_at(scratch, (int64_t)needed, 1), t);
    if (!apart) {
      set_error_text("adapm_rmsnorm_backward: the scratch overlaps another buffer");
      return ADAPM_EINVAL;
    }
  }
  rc = check_on_this_device({dy, dsum, sum, rstd, weight, dresidual, dx, dweight, dweight ? scratch : nullptr, d->step}, &device);
  if (rc == ADAPM_OK) rc = sm_count(device, &sms);
  if (rc != ADAPM_OK) return rc;
  a.dy = dy; a.dsum = dsum; a.sum = sum; a.rstd = rstd; a.weight = weight; a.dres = dresidual; a.dx = dx;
  a.partial = dweight ? (float*)scratch : nullptr;
  a.dy_ld = d->y_ld; a.s_ld = d->sum_ld; a.r_ld = d->residual_ld; a.x_ld = d->x_ld; a.rows = d->rows;
  a.cols = (int32_t)d->cols; a.groups = (int32_t)((d->cols + 7) / 8); a.slots = (int32_t)slots_of(d->cols, form);
  const GradForm f = grad_form(d->rows, a.slots, form, std::min(sms, 256));
  a.weight_f32 = d->weight_dtype == ADAPM_TYPE_F32;
  const bool f32 = d->dtype == ADAPM_TYPE_F32;
#define ADAPM_NORM_OF(T, DROP)                                                                                         \
  (form == VEC ? backward_form<T, VEC, DROP>(a, f, s) : form == SHIFTED ? backward_form<T, SHIFTED, DROP>(a, f, s) : backward_form<T, SCALAR, DROP>(a, f, s))
#define ADAPM_NORM(DROP) (f32 ? ADAPM_NORM_OF(float, DROP) : ADAPM_NORM_OF(uint16_t, DROP))
  ADAPM_CUDA(a.drop.mode ? ADAPM_NORM(true) : ADAPM_NORM(false));
#undef ADAPM_NORM
#undef ADAPM_NORM_OF
  if (!dweight) return ADAPM_OK;
  const unsigned grid = (unsigned)((d->cols + 31) / 32);
  ADAPM_CUDA(dweight_dtype == ADAPM_TYPE_F32
                 ? launch_chained(true, column_sum_kernel<float>, grid, 1024, 0, s, (const float*)scratch, f.ctas, a.cols, (float*)dweight, (int)(accumulate != 0))
                 : launch_chained(true, column_sum_kernel<uint16_t>, grid, 1024, 0, s, (const float*)scratch, f.ctas, a.cols, (uint16_t*)dweight, (int)(accumulate != 0)));
  return ADAPM_OK;
}
