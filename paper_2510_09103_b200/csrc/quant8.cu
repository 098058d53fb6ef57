// Matrices to 8 bits and back: the codes of a linear layer's operands, and activations kept for the backward pass.
//
//   m = max |x| over a row, or over 128 columns of it     top = 127 (int8), 448 (e4m3)
//   s = max(fl(m / top), 2^-126), or the least power of two that is m / top or more; 1 where m = 0; NaN where an x is not finite
//   code = round(x / s), ties to even (codes of a group with a NaN scale are zero)          x' = code s
//
// Every element is read once and written once (rows with one scale above 65536 columns in bf16, 32768 in fp32, are read twice).  A row, or a group
// of 128 columns, is held in registers between its maximum and its codes.  Bound by HBM: 14336 x 4096 with a scale per row 27 us = 6.5 TB/s, 8192 x
// 14336 with one per 128 columns 57 to 61 (6.2 to 5.8; 72 % of the issue slots), back 54 (6.6); rows that start anywhere at 0.5 to 0.75 of that.
#include <algorithm>

#include "codes.cuh"
#include "device_math.cuh"
#include "op_checks.h"
#include "philox.cuh"
#include "tc_common.cuh"

namespace adapm {
namespace {

// The greater magnitude, NaN if either is.
__device__ __forceinline__ float top_of(float m, float x) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(x)));
  return m;
}

// ---- eight elements, as they were read -------------------------------------------------------------------
template <typename T> struct Eight;
template <> struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
  }
  __device__ __forceinline__ void load(const float* p) { load8f(p, v); }
  static __device__ __forceinline__ void load_two(Eight& a, Eight& b, const float* p) { tc::ldcg_f32x8(p, a.v); tc::ldcg_f32x8(p + 8, b.v); }
  __device__ __forceinline__ void set(int e, float x) { v[e] = x; }
  __device__ __forceinline__ uint32_t top_bits() const {          // of the greatest magnitude; NaN if there is one
    float m = fabsf(v[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) m = top_of(m, v[e]);
    return __float_as_uint(m);
  }
  __device__ __forceinline__ void unpack(float* x) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v[e];
  }
};
template <> struct Eight<uint16_t> {
  uint32_t w[4];
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0; }
  __device__ __forceinline__ void load(const uint16_t* p) {
    const uint4 t = *reinterpret_cast<const uint4*>(p);
    w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
  }
  static __device__ __forceinline__ void load_two(Eight& a, Eight& b, const uint16_t* p) {
    asm volatile("ld.global.cg.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=r"(a.w[0]), "=r"(a.w[1]), "=r"(a.w[2]), "=r"(a.w[3]), "=r"(b.w[0]), "=r"(b.w[1]), "=r"(b.w[2]), "=r"(b.w[3]) : "l"(p));
  }
  __device__ __forceinline__ void set(int e, uint16_t x) { w[e >> 1] |= (uint32_t)x << (16 * (e & 1)); }
  __device__ __forceinline__ uint32_t top_bits() const {
    uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
    for (int e = 1; e < 4; ++e) asm("{\n.reg .b32 t;\nabs.bf16x2 t, %1;\nmax.NaN.bf16x2 %0, %0, t;\n}" : "+r"(m) : "r"(w[e]));
    return max(m << 16, m & 0xffff0000u);
  }
  __device__ __forceinline__ void unpack(float* x) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
  }
};

// A thread's sixteen elements among the `team` threads that share 16 x team columns from `base` on, as two eights; those past the row's end
// are zero.  VEC (rows of x start on 16 bytes, rows of codes on 8): sixteen neighbours.  Else every team-th element, so that neighbouring
// threads still read and write neighbouring elements.  (Neighbours there too, by the widest accesses that each address allows: 16384 x 1601
// 35 -> 36 us, back 41 -> 53.)
template <bool VEC, typename T>
__device__ __forceinline__ void fetch16(Eight<T>* x, const T* row, int64_t base, int me, int team, int64_t cols, bool wide) {
  const int64_t c = base + (VEC ? 16 * me : me);
  if (VEC && c + 16 <= cols) {
    if (wide) {
      Eight<T>::load_two(x[0], x[1], row + c);
    } else {
      x[0].load(row + c);
      x[1].load(row + c + 8);
    }
    return;
  }
  const T* const p = row + c;
  const int step = VEC ? 1 : team, left = (int)min((int64_t)INT32_MAX, cols - c);
  x[0].clear();
  x[1].clear();
  if (VEC && left <= 0) return;                      // (the other lanes wait for what these ask: 16384 x 1600 back 22 -> 10.5 us, 28312 x 4128 72 -> 53)
  if (!VEC && base + 16 * team <= cols) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e >> 3].set(e & 7, p[e * step]);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e * step < left) x[e >> 3].set(e & 7, p[e * step]);
  }
}
// Four words of codes to the same places.
template <bool VEC>
__device__ __forceinline__ void put_codes(uint8_t* row, int64_t base, int me, int team, int64_t cols, bool codes16, const uint32_t* q) {
  const int64_t c = base + (VEC ? 16 * me : me);
  uint8_t* const p = row + c;
  if (VEC && c + 16 <= cols) {
    if (codes16) {
      *reinterpret_cast<uint4*>(p) = make_uint4(q[0], q[1], q[2], q[3]);
    } else {
      *reinterpret_cast<uint2*>(p) = make_uint2(q[0], q[1]);
      *reinterpret_cast<uint2*>(p + 8) = make_uint2(q[2], q[3]);
    }
    return;
  }
  const int step = VEC ? 1 : team, left = (int)min((int64_t)INT32_MAX, cols - c);
  if (VEC && left <= 0) return;
  if (!VEC && base + 16 * team <= cols) {
#pragma unroll
    for (int e = 0; e < 16; ++e) p[e * step] = (uint8_t)(q[e >> 2] >> (8 * (e & 3)));
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e * step < left) p[e * step] = (uint8_t)(q[e >> 2] >> (8 * (e & 3)));
  }
}

// ---- scales and codes ----------------------------------------------------------------------------------------
enum : int { INT8_MAX_SCALE = 0, INT8_POW2 = 1, E4M3_POW2 = 2 };

struct Scale { float s, inv; };

// From the bits of the greatest magnitude.
__device__ __forceinline__ Scale scale_of(uint32_t m, int mode) {
  if (m >= 0x7f800000u) return Scale{__uint_as_float(0x7fffffffu), 0.f};
  if (m == 0) return Scale{1.f, 1.f};
  if (mode == INT8_MAX_SCALE) {
    const float s = fmaxf(__fdiv_rn(__uint_as_float(m), 127.f), 1.17549435e-38f);
    return Scale{s, __frcp_rn(s)};
  }
  // 127 = 1.984375 x 2^6, 448 = 1.75 x 2^8: m's exponent less that one's, and one more where m's fraction is above
  const uint32_t fraction = m & 0x7fffffu, limit = mode == INT8_POW2 ? 0x7e0000u : 0x600000u;
  const int e = max(1, (int)(m >> 23) - (mode == INT8_POW2 ? 6 : 8) + (fraction > limit ? 1 : 0));
  return Scale{__uint_as_float((uint32_t)e << 23), __uint_as_float((uint32_t)(254 - e) << 23)};
}

// The codes of four elements.  F32: they may have more than the 8 bits of bf16.
template <bool F32, int MODE>
__device__ __forceinline__ uint32_t encode4(const float* x, const Scale& k) {
  if (MODE == E4M3_POW2) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1] * k.inv), "f"(x[0] * k.inv));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3] * k.inv), "f"(x[2] * k.inv));
    return (uint32_t)lo | ((uint32_t)hi << 16);
  }
  // x / s + 1.5 2^23, rounded once: a whole number, whose low byte is the code
  constexpr float kMagic = 12582912.f;
  float t[4];
#pragma unroll
  for (int e = 0; e < 4; e += 2) {
    const float2 q = fma2(make_float2(x[e], x[e + 1]), make_float2(k.inv, k.inv), make_float2(kMagic, kMagic));
    t[e] = q.x; t[e + 1] = q.y;
  }
  if (MODE == INT8_MAX_SCALE) {
    // 1 / s is rounded, so that a quotient next to half a step may have gone the wrong way.  What is left, d = x - code s, has no
    // rounding (it is a multiple of half the last place of s, and below s), and code + d / s is rounded once more.  With s = f 2^e, 1 <= f < 2, a quotient
    // that is not half a step is at least 2^-24 / f away from it, and d (1 / s) is off by f 2^-26 at most, which is less.  A quotient
    // that is half a step wants 2 x / s to be a whole number: of bf16 elements, where s is the nearest number to an
    // 8-bit number over 127, only for powers of two, whose reciprocal is not rounded; of fp32 elements it has to be looked for.
    // (What is left is doubled for that, which rounds nothing; half of s has no fp32 number where s is below 2^-125 and odd in its last place.)
    float left[4], worst = 0.f;
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      const float2 r = add2(make_float2(t[e], t[e + 1]), make_float2(-kMagic, -kMagic));
      const float2 d = fma2(r, make_float2(-k.s, -k.s), make_float2(x[e], x[e + 1]));
      if (F32) {
        const float2 twice = add2(d, d);
        left[e] = twice.x; left[e + 1] = twice.y;
        worst = fmaxf(worst, fmaxf(fabsf(twice.x), fabsf(twice.y)));
      } else {
        const float2 q = fma2(d, make_float2(k.inv, k.inv), make_float2(t[e], t[e + 1]));
        t[e] = q.x; t[e + 1] = q.y;
      }
    }
    if (F32 && worst >= k.s) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float d = fabsf(left[e]);
        if (d > k.s || (d == k.s && (__float_as_uint(t[e]) & 1u))) t[e] += copysignf(1.f, left[e]);
      }
    }
  }
  return __byte_perm(__byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040), __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040), 0x5410);
}

template <bool F32, int MODE>
__device__ __forceinline__ void encode16(const float* x, const Scale& k, uint32_t* q) {
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = encode4<F32, MODE>(x + 4 * i, k);
}
// (the form is chosen once for sixteen elements; once for four: 8192 x 14336 in groups 62 us, 57 now)
template <typename T>
__device__ __forceinline__ void encode16(const Eight<T>* x, const Scale& k, int mode, uint32_t* q) {
  constexpr bool kF32 = sizeof(T) == 4;
  float v[16];
  x[0].unpack(v);
  x[1].unpack(v + 8);
  if (mode == INT8_POW2) encode16<kF32, INT8_POW2>(v, k, q);
  else if (mode == INT8_MAX_SCALE) encode16<kF32, INT8_MAX_SCALE>(v, k, q);
  else encode16<kF32, E4M3_POW2>(v, k, q);
  if (!(k.s <= 3.402823466e38f)) q[0] = q[1] = q[2] = q[3] = 0;
}

struct QuantArgs {
  const void* x;
  uint8_t* codes;
  float* scales;
  int64_t x_ld, codes_ld, rows, cols, groups, total;      // groups of 128 columns per row, and of kRows rows in all
  int32_t mode, codes16, wide;   // rows of codes start on 16 bytes, rows of x on 32
};

// ---- a scale per 128 columns -----------------------------------------------------------------------------------
// Rows per thread: several in bf16 and back (8192 x 14336 58.4 -> 56.3 us, back 54.8 -> 53.5), one of fp32 (8192 x 4096 35.7 -> 26.3).
constexpr int kRows = 4;
template <typename T>
constexpr int kRowsOf = sizeof(T) == 2 ? kRows : 1;

// Which rows and columns a thread of eight that share a group works on: ROWS rows below one another, so that one division finds
// them all.  (16 elements per thread rather than eight: half the shuffles and half the scales per element.)
struct Spot { int64_t row; int64_t col; int64_t group; };
template <int ROWS>
__device__ __forceinline__ bool spot_of(Spot& s, int64_t groups, int64_t total) {
  const int64_t i = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
  if (i >= total) return false;
  const int64_t band = total <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)groups) : i / groups;
  s.group = i - band * groups;
  s.row = band * ROWS;
  s.col = s.group * 128;
  return true;
}

// ... and 512 columns of which row a warp works on, where rows start anywhere.
__device__ __forceinline__ bool block_of(int64_t& row, int64_t& base, int64_t cols, int64_t rows) {
  const uint32_t blocks = (uint32_t)((cols + 511) / 512);
  const int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  row = i <= UINT32_MAX ? (int64_t)((uint32_t)i / blocks) : i / blocks;
  base = (i - row * blocks) * 512;
  return row < rows;
}

template <typename T>
__global__ void __launch_bounds__(256) quant8_groups_kernel(const QuantArgs a) {
  constexpr int ROWS = kRowsOf<T>;
  wait_for_previous_kernel();
  const int me = threadIdx.x & 7;
  Spot s = {0, 0, 0};
  const bool live = spot_of<ROWS>(s, a.groups, a.total);
  Eight<T> x[ROWS][2];
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    x[u][0].clear();
    x[u][1].clear();
    if (live && s.row + u < a.rows) fetch16<true>(x[u], static_cast<const T*>(a.x) + (s.row + u) * a.x_ld, s.col, me, 8, a.cols, a.wide);
  }
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    uint32_t m = max(x[u][0].top_bits(), x[u][1].top_bits());
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (!live || s.row + u >= a.rows) continue;
    const Scale k = scale_of(m, a.mode);
    uint32_t q[4];
    encode16(x[u], k, a.mode, q);
    put_codes<true>(a.codes + (s.row + u) * a.codes_ld, s.col, me, 8, a.cols, a.codes16, q);
    if (me == 0) a.scales[(s.row + u) * a.groups + s.group] = k.s;
  }
}

// Rows that start anywhere: a warp has 512 columns of a row, every thirty-second to a thread, so that four of a thread's sixteen belong to each of four groups.
// (Eight threads per group as above, every eighth column to a thread: 16384 x 1601 39.5 us.)
template <typename T>
__global__ void __launch_bounds__(256) quant8_odd_groups_kernel(const QuantArgs a) {
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31;
  int64_t row, base;
  if (!block_of(row, base, a.cols, a.rows)) return;       // (a whole warp)
  Eight<T> x[2];
  fetch16<false>(x, static_cast<const T*>(a.x) + row * a.x_ld, base, lane, 32, a.cols, false);
  uint8_t* const codes = a.codes + row * a.codes_ld;
  float v[16];
  x[0].unpack(v);
  x[1].unpack(v + 8);
  uint32_t q[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    float m = fabsf(v[4 * g]);
#pragma unroll
    for (int e = 1; e < 4; ++e) m = top_of(m, v[4 * g + e]);
    const Scale k = scale_of(__reduce_max_sync(0xffffffffu, __float_as_uint(m)), a.mode);
    const int64_t group = base / 128 + g;
    if (lane == 0 && group < a.groups) a.scales[row * a.groups + group] = k.s;
    constexpr bool kF32 = sizeof(T) == 4;
    q[g] = a.mode == INT8_POW2 ? encode4<kF32, INT8_POW2>(v + 4 * g, k) : a.mode == INT8_MAX_SCALE ? encode4<kF32, INT8_MAX_SCALE>(v + 4 * g, k) : encode4<kF32, E4M3_POW2>(v + 4 * g, k);
    if (!(k.s <= 3.402823466e38f)) q[g] = 0;
  }
  put_codes<false>(codes, base, lane, 32, a.cols, false, q);
}

// ---- a scale per row -------------------------------------------------------------------------------------------
template <bool WARP>
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t* red) {
  m = __reduce_max_sync(0xffffffffu, m);
  if (WARP) return m;
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
  __syncthreads();
  m = threadIdx.x % 32 < blockDim.x / 32 ? red[threadIdx.x & 31] : 0u;
  return __reduce_max_sync(0xffffffffu, m);
}

// NC: chunks of sixteen per thread; 0: as many as it takes, read once for the maximum and once for the codes.  WARP: a warp per row.
template <typename T, int NC, bool WARP, bool VEC>
__global__ void __launch_bounds__(WARP ? 128 : 1024) quant8_rows_kernel(const QuantArgs a) {
  __shared__ uint32_t red[32];
  wait_for_previous_kernel();
  const int team = WARP ? 32 : (int)blockDim.x, me = WARP ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
  const int64_t row = WARP ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  if (row >= a.rows) return;                       // (a whole warp, or never)
  const T* const x = static_cast<const T*>(a.x) + row * a.x_ld;
  uint8_t* const codes = a.codes + row * a.codes_ld;
  const int64_t step = 16 * (int64_t)team;
  constexpr int kHeld = NC ? NC : 1;
  Eight<T> r[kHeld][2];
  uint32_t m = 0;
  if (NC) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) fetch16<VEC>(r[i], x, i * step, me, team, a.cols, a.wide);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) m = max(m, max(r[i][0].top_bits(), r[i][1].top_bits()));
  } else {
    for (int64_t base = 0; base < a.cols; base += step) {
      fetch16<VEC>(r[0], x, base, me, team, a.cols, a.wide);
      m = max(m, max(r[0][0].top_bits(), r[0][1].top_bits()));
    }
  }
  m = row_max<WARP>(m, red);
  const Scale k = scale_of(m, a.mode);
  if (me == 0) a.scales[row] = k.s;
  uint32_t q[4];
  if (NC) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      encode16(r[i], k, a.mode, q);
      put_codes<VEC>(codes, i * step, me, team, a.cols, a.codes16, q);
    }
  } else {
    for (int64_t base = 0; base < a.cols; base += step) {
      fetch16<VEC>(r[0], x, base, me, team, a.cols, a.wide);
      encode16(r[0], k, a.mode, q);
      put_codes<VEC>(codes, base, me, team, a.cols, a.codes16, q);
    }
  }
}

// ---- back ------------------------------------------------------------------------------------------------------
struct DequantArgs {
  const uint8_t* codes;
  const float* scales;
  void* x;
  int64_t x_ld, codes_ld, rows, cols, groups, total;      // groups of 128 columns, whatever a scale stands for
  int32_t per_row, codes16, wide;                         // one scale per row; rows of codes start on 16 bytes, rows of x on 32
};

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }
__device__ __forceinline__ void put8(float* p, const float* x) { store8f(p, x); }
__device__ __forceinline__ void put8(uint16_t* p, const float* x) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
// 32 bytes at a time, from addresses that are multiples of that.
__device__ __forceinline__ void put16(float* p, const float* x) { tc::st_f32x8(p, x); tc::st_f32x8(p + 8, x + 8); }
__device__ __forceinline__ void put16(uint16_t* p, const float* x) {
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
  tc::st_b32x8(p, w);
}

template <typename T, bool E4M3>
__global__ void __launch_bounds__(256) dequant8_kernel(const DequantArgs a) {
  wait_for_previous_kernel();
  const int me = threadIdx.x & 7;
  Spot t;
  if (!spot_of<kRows>(t, a.groups, a.total)) return;
  uint4 q[kRows];
  float s[kRows];
  const int64_t c = t.col + 16 * me;
  if (c >= a.cols) return;         // (a lane without columns would hold up the others below)
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    q[u] = make_uint4(0, 0, 0, 0);
    s[u] = 0.f;
    const int64_t row = t.row + u;
    if (row >= a.rows) continue;
    const uint8_t* const p = a.codes + row * a.codes_ld;
    s[u] = a.scales[a.per_row ? row : row * a.groups + t.group];
    if (c + 16 <= a.cols && a.codes16) {
      q[u] = *reinterpret_cast<const uint4*>(p + c);
      continue;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = c + 8 * h;
      if (at + 8 <= a.cols) {
        const uint2 w = *reinterpret_cast<const uint2*>(p + at);
        (&q[u].x)[2 * h] = w.x; (&q[u].x)[2 * h + 1] = w.y;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at + e < a.cols) (&q[u].x)[2 * h + (e >> 2)] |= (uint32_t)p[at + e] << (8 * (e & 3));
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const int64_t row = t.row + u;
    if (row >= a.rows) continue;
    float v[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack4<E4M3>((&q[u].x)[i], v + 4 * i);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] *= s[u];
    T* const p = static_cast<T*>(a.x) + row * a.x_ld;
    if (c + 16 <= a.cols && a.wide) {
      put16(p + c, v);
      continue;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = c + 8 * h;
      if (at + 8 <= a.cols) {
        put8(p + at, v + 8 * h);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at + e < a.cols) put(p + at + e, v[8 * h + e]);
      }
    }
  }
}

// Rows that start anywhere, as in quant8_odd_groups_kernel.  (Every eighth column to a thread: 16384 x 1601 42 us.)
template <typename T, bool E4M3>
__global__ void __launch_bounds__(256) dequant8_odd_kernel(const DequantArgs a) {
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31;
  int64_t row, base;
  if (!block_of(row, base, a.cols, a.rows)) return;
  const uint8_t* const p = a.codes + row * a.codes_ld + base + lane;
  T* const to = static_cast<T*>(a.x) + row * a.x_ld + base + lane;
  const float* const scales = a.scales + (a.per_row ? row : row * a.groups + base / 128);
  const int left = (int)(a.cols - base < 512 ? a.cols - base : 512) - lane;
  float s[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) s[g] = base + 128 * g < a.cols ? scales[a.per_row ? 0 : g] : 0.f;
  uint32_t b[16] = {};
  auto decode = [&](int i, float* v) {
    unpack4<E4M3>(b[4 * i] | (b[4 * i + 1] << 8) | (b[4 * i + 2] << 16) | (b[4 * i + 3] << 24), v);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= s[i];
  };
  // (a block that is whole asks nothing of each element: 16384 x 1601 28 -> 18 us; two or four blocks per warp, their codes on the way at the same time: 20 and 23)
  if (left > 480) {
#pragma unroll
    for (int e = 0; e < 16; ++e) b[e] = p[32 * e];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[4];
      decode(i, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) put(to + 32 * (4 * i + e), v[e]);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) b[e] = 32 * e < left ? p[32 * e] : 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v[4];
    decode(i, v);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (32 * (4 * i + e) < left) put(to + 32 * (4 * i + e), v[e]);
  }
}

// ---- host ------------------------------------------------------------------------------------------------------

int check_desc(const adapm_codes8& d) {
  if (d.rows < 0 || d.cols <= 0) return ADAPM_EINVAL;
  if (!known_type(d.dtype) || (d.code != ADAPM_CODE_INT8 && d.code != ADAPM_CODE_E4M3) || (d.group != 0 && d.group != 128)) return ADAPM_EINVAL;
  if (d.rows > INT32_MAX || d.cols > (1 << 24)) return ADAPM_ERANGE;
  return ADAPM_OK;
}

// What both directions check of their buffers.
int check_buffers(const adapm_codes8& d, const void* x, const void* codes, const void* scales, bool to_codes, const char* overlap) {
  const int64_t eb = type_bytes(d.dtype), groups = d.group ? (d.cols + 127) / 128 : 1;
  if (!x || !codes || !scales || d.x_ld < d.cols || d.codes_ld < d.cols) return ADAPM_EINVAL;
  if (d.rows > 1 && std::max(d.x_ld, d.codes_ld) > INT64_MAX / 8 / d.rows) return ADAPM_ERANGE;
  if ((uintptr_t)x % (uintptr_t)eb || (uintptr_t)scales % 4) return ADAPM_EALIGN;
  const Place px = matrix_at(x, d.rows, d.x_ld, d.cols, eb), pc = matrix_at(codes, d.rows, d.codes_ld, d.cols, 1), ps = vector_at(scales, d.rows * groups, 4);
  if (share(px, pc) || share(px, ps) || (to_codes && share(pc, ps))) {
    set_error_text(overlap);
    return ADAPM_EINVAL;
  }
  int device;
  return check_on_this_device({x, codes, scales}, &device);
}

template <typename T, int NC, bool WARP, bool VEC>
cudaError_t launch_rows(const QuantArgs& a, cudaStream_t s) {
  const int64_t chunks = (a.cols + 15) / 16;
  const unsigned threads = WARP ? 128u : NC ? (unsigned)(((chunks + NC - 1) / NC + 31) / 32 * 32) : 1024u;
  return launch_chained(true, quant8_rows_kernel<T, NC, WARP, VEC>, (unsigned)(WARP ? (a.rows + 3) / 4 : a.rows), threads, 0, s, a);
}

template <typename T, bool VEC>
cudaError_t rows_form(const QuantArgs& a, int sms, cudaStream_t s) {
  const int64_t chunks = (a.cols + 15) / 16;
  const bool many = a.rows >= 8 * (int64_t)sms;
  if (many && chunks <= 32) return launch_rows<T, 1, true, VEC>(a, s);
  if (many && chunks <= 64) return launch_rows<T, 2, true, VEC>(a, s);
  if (many && chunks <= 128) return launch_rows<T, 4, true, VEC>(a, s);
  if (chunks <= (many ? 128 : 1024)) return launch_rows<T, 1, false, VEC>(a, s);
  if (chunks <= (sizeof(T) == 2 && VEC ? 512 : 2048)) return launch_rows<T, 2, false, VEC>(a, s);
  if constexpr (sizeof(T) == 2 && VEC) {
    if (chunks <= 4096) return launch_rows<T, 4, false, VEC>(a, s);
  }
  return launch_rows<T, 0, false, VEC>(a, s);
}

// Whether eight elements of a row are one access, and its codes start on `unit` bytes.
bool rows_of_eights(const adapm_codes8& d, const void* x, const void* codes, int unit) {
  const int64_t eb = type_bytes(d.dtype);
  return (uintptr_t)x % 16 == 0 && (uintptr_t)codes % (uintptr_t)unit == 0 && (d.rows <= 1 || (d.x_ld * eb % 16 == 0 && d.codes_ld % unit == 0));
}

// CTAs of eight warps that have 512 columns of a row each.
int64_t odd_grid(const adapm_codes8& d) { return (d.rows * ((d.cols + 511) / 512) + 7) / 8; }
bool rows_of_32(const adapm_codes8& d, const void* x) { return (uintptr_t)x % 32 == 0 && (d.rows <= 1 || d.x_ld * type_bytes(d.dtype) % 32 == 0); }

}  // namespace

int launch_dequant8(const adapm_codes8& d, const void* codes, const float* scales, void* x, cudaStream_t s) {
  DequantArgs a;
  a.codes = static_cast<const uint8_t*>(codes); a.scales = scales; a.x = x;
  a.x_ld = d.x_ld; a.codes_ld = d.codes_ld; a.rows = d.rows; a.cols = d.cols; a.groups = (d.cols + 127) / 128;
  a.total = (d.rows + kRows - 1) / kRows * a.groups;
  a.per_row = d.group == 0;
  a.codes16 = rows_of_eights(d, x, codes, 16);
  a.wide = rows_of_32(d, x);
  const bool f32 = d.dtype == ADAPM_TYPE_F32, e4m3 = d.code == ADAPM_CODE_E4M3, vec = rows_of_eights(d, x, codes, 8);
  const int64_t grid = vec ? (a.total + 31) / 32 : odd_grid(d);
  if (grid > INT32_MAX) return ADAPM_ERANGE;
#define ADAPM_DEQUANT(KERNEL, T, E) launch_chained(true, KERNEL<T, E>, (unsigned)grid, 256, 0, s, a)
#define ADAPM_DEQUANT_OF(KERNEL, T) (e4m3 ? ADAPM_DEQUANT(KERNEL, T, true) : ADAPM_DEQUANT(KERNEL, T, false))
  ADAPM_CUDA(f32 ? (vec ? ADAPM_DEQUANT_OF(dequant8_kernel, float) : ADAPM_DEQUANT_OF(dequant8_odd_kernel, float))
                 : (vec ? ADAPM_DEQUANT_OF(dequant8_kernel, uint16_t) : ADAPM_DEQUANT_OF(dequant8_odd_kernel, uint16_t)));
#undef ADAPM_DEQUANT_OF
#undef ADAPM_DEQUANT
  return ADAPM_OK;
}

}  // namespace adapm

using namespace adapm;

extern "C" int adapm_quant8(const adapm_codes8* d, const void* x, void* codes, float* scales, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  int rc = check_desc(*d);
  if (rc != ADAPM_OK) return rc;
  if (d->code == ADAPM_CODE_E4M3 && !d->pow2) return ADAPM_EUNSUPPORTED;
  if (d->rows == 0) return ADAPM_OK;
  rc = check_buffers(*d, x, codes, scales, true, "adapm_quant8: the codes or the scales overlap another buffer");
  if (rc != ADAPM_OK) return rc;
  QuantArgs a;
  a.x = x; a.codes = static_cast<uint8_t*>(codes); a.scales = scales;
  a.x_ld = d->x_ld; a.codes_ld = d->codes_ld; a.rows = d->rows; a.cols = d->cols;
  a.groups = (d->cols + 127) / 128;
  const int64_t per = d->dtype == ADAPM_TYPE_F32 ? kRowsOf<float> : kRowsOf<uint16_t>;
  a.total = (d->rows + per - 1) / per * a.groups;
  a.codes16 = rows_of_eights(*d, x, codes, 16);
  a.wide = rows_of_32(*d, x);
  a.mode = d->code == ADAPM_CODE_E4M3 ? E4M3_POW2 : d->pow2 ? INT8_POW2 : INT8_MAX_SCALE;
  cudaStream_t s = (cudaStream_t)stream;
  const bool f32 = d->dtype == ADAPM_TYPE_F32, vec = rows_of_eights(*d, x, codes, 8);
  if (d->group) {
    const int64_t grid = vec ? (a.total + 31) / 32 : odd_grid(*d);
    if (grid > INT32_MAX) return ADAPM_ERANGE;
#define ADAPM_QUANT(KERNEL, T) launch_chained(true, KERNEL<T>, (unsigned)grid, 256, 0, s, a)
    ADAPM_CUDA(f32 ? (vec ? ADAPM_QUANT(quant8_groups_kernel, float) : ADAPM_QUANT(quant8_odd_groups_kernel, float))
                   : (vec ? ADAPM_QUANT(quant8_groups_kernel, uint16_t) : ADAPM_QUANT(quant8_odd_groups_kernel, uint16_t)));
#undef ADAPM_QUANT
    return ADAPM_OK;
  }
  int device, sms;
  ADAPM_CUDA(cudaGetDevice(&device));
  ADAPM_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
  ADAPM_CUDA(f32 ? (vec ? rows_form<float, true>(a, sms, s) : rows_form<float, false>(a, sms, s))
                 : (vec ? rows_form<uint16_t, true>(a, sms, s) : rows_form<uint16_t, false>(a, sms, s)));
  return ADAPM_OK;
}

extern "C" int adapm_dequant8(const adapm_codes8* d, const void* codes, const float* scales, void* x, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  int rc = check_desc(*d);
  if (rc != ADAPM_OK || d->rows == 0) return rc;
  rc = check_buffers(*d, x, codes, scales, false, "adapm_dequant8: the output overlaps another buffer");
  if (rc != ADAPM_OK) return rc;
  return launch_dequant8(*d, codes, scales, x, (cudaStream_t)stream);
}
