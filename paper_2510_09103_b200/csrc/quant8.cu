// Matrices to 8 bits and back: the codes of a linear layer's operands, and activations kept for the backward pass.
//
//   m = max |x| over a row, or over 128 columns of it     top = 127 (int8), 448 (e4m3)
//   s = max(fl(m / top), 2^-126), or the least power of two that is m / top or more; 1 where m = 0; NaN where an x is not finite
//   code = round(x / s), ties to even (codes of a group with a NaN scale are zero)          x' = code s
//
// Every element is read once and written once (rows above 32768 columns with one scale are read twice); bound by HBM.  A row, or a group
// of 128 columns, is held in registers between its maximum and its codes.
#include <algorithm>

#include "codes.cuh"
#include "device_math.cuh"
#include "op_checks.h"
#include "philox.cuh"

namespace adapm {
namespace {

// ---- eight elements, as they were read -------------------------------------------------------------------
template <typename T> struct Eight;
template <> struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
  }
  __device__ __forceinline__ void load(const float* p) { load8f(p, v); }
  __device__ __forceinline__ void set(int e, float x) { v[e] = x; }
  __device__ __forceinline__ uint32_t top_bits() const {          // of the magnitudes, which are ordered like their bits (NaN last)
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
    return m;
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
  __device__ __forceinline__ void set(int e, uint16_t x) { w[e >> 1] |= (uint32_t)x << (16 * (e & 1)); }
  __device__ __forceinline__ uint32_t top_bits() const {
    uint32_t m = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16) << 16;
  }
  __device__ __forceinline__ void unpack(float* x) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
  }
};

// A thread's eight elements among `team` threads from column `base` on.  VEC: eight neighbours, one access (rows start on 16
// bytes, their codes on 8).  Else every team-th element, so that neighbouring threads still read neighbouring elements.
template <bool VEC, typename T>
__device__ __forceinline__ void fetch(Eight<T>& r, const T* row, int64_t base, int me, int team, int64_t cols) {
  r.clear();
  if (VEC) {
    const int64_t c = base + 8 * me;
    if (c + 8 <= cols) {
      r.load(row + c);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < cols) r.set(e, row[c + e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t c = base + e * team + me;
      if (c < cols) r.set(e, row[c]);
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void put_codes(uint8_t* row, int64_t base, int me, int team, int64_t cols, uint2 q) {
  if (VEC && base + 8 * me + 8 <= cols) {
    *reinterpret_cast<uint2*>(row + base + 8 * me) = q;
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t c = VEC ? base + 8 * me + e : base + e * team + me;
    if (c < cols) row[c] = (uint8_t)((e < 4 ? q.x : q.y) >> (8 * (e & 3)));
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

__device__ __forceinline__ uint2 encode(const float* x, const Scale& k, int mode) {
  if (!(k.s <= 3.402823466e38f)) return make_uint2(0, 0);
  if (mode == E4M3_POW2) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint16_t lo, hi;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[4 * h + 1] * k.inv), "f"(x[4 * h] * k.inv));
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[4 * h + 3] * k.inv), "f"(x[4 * h + 2] * k.inv));
      w[h] = (uint32_t)lo | ((uint32_t)hi << 16);
    }
    return make_uint2(w[0], w[1]);
  }
  // x / s + 1.5 2^23, rounded once: a whole number, whose low byte is the code
  constexpr float kMagic = 12582912.f;
  float t[8];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float2 q = fma2(make_float2(x[e], x[e + 1]), make_float2(k.inv, k.inv), make_float2(kMagic, kMagic));
    t[e] = q.x; t[e + 1] = q.y;
  }
  if (mode == INT8_MAX_SCALE) {
    // 1 / s is rounded, so that a quotient next to half a step may have gone the wrong way: what is left, x - code s, has no
    // rounding (it is a multiple of the last place of s, below s) and is compared with half a step
    float left[8], worst = 0.f;
    const float half = 0.5f * k.s;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float2 r = add2(make_float2(t[e], t[e + 1]), make_float2(-kMagic, -kMagic));
      const float2 d = fma2(r, make_float2(-k.s, -k.s), make_float2(x[e], x[e + 1]));
      left[e] = d.x; left[e + 1] = d.y;
      worst = fmaxf(worst, fmaxf(fabsf(d.x), fabsf(d.y)));
    }
    if (worst >= half) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = fabsf(left[e]);
        if (d > half || (d == half && (__float_as_uint(t[e]) & 1u))) t[e] += copysignf(1.f, left[e]);
      }
    }
  }
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __byte_perm(__float_as_uint(t[4 * h]), __float_as_uint(t[4 * h + 1]), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(t[4 * h + 2]), __float_as_uint(t[4 * h + 3]), 0x0040);
    w[h] = __byte_perm(lo, hi, 0x5410);
  }
  return make_uint2(w[0], w[1]);
}

struct QuantArgs {
  const void* x;
  uint8_t* codes;
  float* scales;
  int64_t x_ld, codes_ld, rows, cols, groups, total;      // groups of 128 columns per row, and in all
  int32_t mode;
};

// ---- a scale per 128 columns -----------------------------------------------------------------------------------
constexpr int kUnits = 4;         // groups per thread

__device__ __forceinline__ int64_t row_of(int64_t unit, int64_t groups, int64_t total) {
  return total <= UINT32_MAX ? (int64_t)((uint32_t)unit / (uint32_t)groups) : unit / groups;
}

// Sixteen threads per group.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) quant8_groups_kernel(const QuantArgs a) {
  wait_for_previous_kernel();
  const int me = threadIdx.x & 15;
  const int64_t u0 = (int64_t)blockIdx.x * (16 * kUnits) + (threadIdx.x >> 4);
  Eight<T> x[kUnits];
  int64_t row[kUnits], col[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int64_t unit = u0 + 16 * u;
    x[u].clear();
    if (unit >= a.total) continue;
    row[u] = row_of(unit, a.groups, a.total);
    col[u] = (unit - row[u] * a.groups) * 128;
    fetch<VEC>(x[u], static_cast<const T*>(a.x) + row[u] * a.x_ld, col[u], me, 16, a.cols);
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int64_t unit = u0 + 16 * u;
    uint32_t m = x[u].top_bits();
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (unit >= a.total) continue;
    const Scale k = scale_of(m, a.mode);
    float v[8];
    x[u].unpack(v);
    put_codes<VEC>(a.codes + row[u] * a.codes_ld, col[u], me, 16, a.cols, encode(v, k, a.mode));
    if (me == 0) a.scales[unit] = k.s;
  }
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

// NC: chunks of eight per thread; 0: as many as it takes, read once for the maximum and once for the codes.  WARP: a warp per row.
template <typename T, int NC, bool WARP, bool VEC>
__global__ void __launch_bounds__(WARP ? 128 : 1024) quant8_rows_kernel(const QuantArgs a) {
  __shared__ uint32_t red[32];
  wait_for_previous_kernel();
  const int team = WARP ? 32 : (int)blockDim.x, me = WARP ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
  const int64_t row = WARP ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  if (row >= a.rows) return;                       // (a whole warp, or never)
  const T* const x = static_cast<const T*>(a.x) + row * a.x_ld;
  uint8_t* const codes = a.codes + row * a.codes_ld;
  const int64_t step = 8 * (int64_t)team;
  constexpr int kHeld = NC ? NC : 1;
  Eight<T> r[kHeld];
  uint32_t m = 0;
  if (NC) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) fetch<VEC>(r[i], x, i * step, me, team, a.cols);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) m = max(m, r[i].top_bits());
  } else {
    for (int64_t base = 0; base < a.cols; base += step) {
      fetch<VEC>(r[0], x, base, me, team, a.cols);
      m = max(m, r[0].top_bits());
    }
  }
  m = row_max<WARP>(m, red);
  const Scale k = scale_of(m, a.mode);
  if (me == 0) a.scales[row] = k.s;
  float v[8];
  if (NC) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      r[i].unpack(v);
      put_codes<VEC>(codes, i * step, me, team, a.cols, encode(v, k, a.mode));
    }
  } else {
    for (int64_t base = 0; base < a.cols; base += step) {
      fetch<VEC>(r[0], x, base, me, team, a.cols);
      r[0].unpack(v);
      put_codes<VEC>(codes, base, me, team, a.cols, encode(v, k, a.mode));
    }
  }
}

// ---- back ------------------------------------------------------------------------------------------------------
struct DequantArgs {
  const uint8_t* codes;
  const float* scales;
  void* x;
  int64_t x_ld, codes_ld, cols, groups, total;            // groups of 128 columns, whatever a scale stands for
  int32_t per_row;                                        // one scale per row
};

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }
__device__ __forceinline__ void put8(float* p, const float* x) { store8f(p, x); }
__device__ __forceinline__ void put8(uint16_t* p, const float* x) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

template <typename T, bool E4M3, bool VEC>
__global__ void __launch_bounds__(256) dequant8_kernel(const DequantArgs a) {
  wait_for_previous_kernel();
  const int me = threadIdx.x & 15;
  const int64_t u0 = (int64_t)blockIdx.x * (16 * kUnits) + (threadIdx.x >> 4);
  uint2 q[kUnits];
  float s[kUnits];
  int64_t row[kUnits], col[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int64_t unit = u0 + 16 * u;
    q[u] = make_uint2(0, 0);
    s[u] = 0.f;
    if (unit >= a.total) continue;
    row[u] = row_of(unit, a.groups, a.total);
    col[u] = (unit - row[u] * a.groups) * 128;
    const uint8_t* const p = a.codes + row[u] * a.codes_ld;
    s[u] = a.scales[a.per_row ? row[u] : unit];
    if (VEC && col[u] + 8 * me + 8 <= a.cols) {
      q[u] = *reinterpret_cast<const uint2*>(p + col[u] + 8 * me);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int64_t c = VEC ? col[u] + 8 * me + e : col[u] + 16 * e + me;
        if (c < a.cols) (e < 4 ? q[u].x : q[u].y) |= (uint32_t)p[c] << (8 * (e & 3));
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (u0 + 16 * u >= a.total) continue;
    float v[8];
    unpack4<E4M3>(q[u].x, v);
    unpack4<E4M3>(q[u].y, v + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= s[u];
    T* const p = static_cast<T*>(a.x) + row[u] * a.x_ld;
    if (VEC && col[u] + 8 * me + 8 <= a.cols) {
      put8(p + col[u] + 8 * me, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int64_t c = VEC ? col[u] + 8 * me + e : col[u] + 16 * e + me;
        if (c < a.cols) put(p + c, v[e]);
      }
    }
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
  const int64_t chunks = (a.cols + 7) / 8;
  const unsigned threads = WARP ? 128u : NC ? (unsigned)(((chunks + NC - 1) / NC + 31) / 32 * 32) : 1024u;
  return launch_chained(true, quant8_rows_kernel<T, NC, WARP, VEC>, (unsigned)(WARP ? (a.rows + 3) / 4 : a.rows), threads, 0, s, a);
}

template <typename T, bool VEC>
cudaError_t rows_form(const QuantArgs& a, int sms, cudaStream_t s) {
  const int64_t chunks = (a.cols + 7) / 8;
  const bool many = a.rows >= 8 * (int64_t)sms;
  if (many && chunks <= 32) return launch_rows<T, 1, true, VEC>(a, s);
  if (many && chunks <= 64) return launch_rows<T, 2, true, VEC>(a, s);
  if (chunks <= (many ? 128 : 1024)) return launch_rows<T, 1, false, VEC>(a, s);
  if (chunks <= 1024) return launch_rows<T, 2, false, VEC>(a, s);
  if (VEC && chunks <= 4096) return launch_rows<T, 4, false, VEC>(a, s);
  return launch_rows<T, 0, false, VEC>(a, s);
}

// Whether eight elements of a row are one access.
bool rows_of_eights(const adapm_codes8& d, const void* x, const void* codes) {
  const int64_t eb = type_bytes(d.dtype);
  return (uintptr_t)x % 16 == 0 && (uintptr_t)codes % 8 == 0 && (d.rows <= 1 || (d.x_ld * eb % 16 == 0 && d.codes_ld % 8 == 0));
}

}  // namespace

int launch_dequant8(const adapm_codes8& d, const void* codes, const float* scales, void* x, cudaStream_t s) {
  DequantArgs a;
  a.codes = static_cast<const uint8_t*>(codes); a.scales = scales; a.x = x;
  a.x_ld = d.x_ld; a.codes_ld = d.codes_ld; a.cols = d.cols; a.groups = (d.cols + 127) / 128; a.total = d.rows * a.groups;
  a.per_row = d.group == 0;
  const int64_t grid = (a.total + 16 * kUnits - 1) / (16 * kUnits);
  if (grid > INT32_MAX) return ADAPM_ERANGE;
  const bool f32 = d.dtype == ADAPM_TYPE_F32, e4m3 = d.code == ADAPM_CODE_E4M3, vec = rows_of_eights(d, x, codes);
#define ADAPM_DEQUANT(T, E, VEC) launch_chained(true, dequant8_kernel<T, E, VEC>, (unsigned)grid, 256, 0, s, a)
#define ADAPM_DEQUANT_OF(T) (e4m3 ? (vec ? ADAPM_DEQUANT(T, true, true) : ADAPM_DEQUANT(T, true, false)) : (vec ? ADAPM_DEQUANT(T, false, true) : ADAPM_DEQUANT(T, false, false)))
  ADAPM_CUDA(f32 ? ADAPM_DEQUANT_OF(float) : ADAPM_DEQUANT_OF(uint16_t));
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
  a.groups = (d->cols + 127) / 128; a.total = d->rows * a.groups;
  a.mode = d->code == ADAPM_CODE_E4M3 ? E4M3_POW2 : d->pow2 ? INT8_POW2 : INT8_MAX_SCALE;
  cudaStream_t s = (cudaStream_t)stream;
  const bool f32 = d->dtype == ADAPM_TYPE_F32, vec = rows_of_eights(*d, x, codes);
  if (d->group) {
    const int64_t grid = (a.total + 16 * kUnits - 1) / (16 * kUnits);
    if (grid > INT32_MAX) return ADAPM_ERANGE;
#define ADAPM_QUANT(T, VEC) launch_chained(true, quant8_groups_kernel<T, VEC>, (unsigned)grid, 256, 0, s, a)
    ADAPM_CUDA(f32 ? (vec ? ADAPM_QUANT(float, true) : ADAPM_QUANT(float, false)) : (vec ? ADAPM_QUANT(uint16_t, true) : ADAPM_QUANT(uint16_t, false)));
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
