// Dropout, and RMS normalisation with the residual's addition and the branch's dropout, forward and backward.
//
//   s = residual + drop(x)      rstd = 1 / sqrt(mean(s^2) + eps)      y = s rstd w      q = e4m3(y 448 / amax|y|)
//   xh = s rstd    ds = rstd (dy w - xh mean(dy w xh)) + dsum    dx = drop(ds)    dw = sum over rows of dy xh
//
// All three read and write every element once and are bound by HBM; a row is held in registers between its reduction and its
// output (up to 32768 columns), in chunks of eight elements: one 16-byte access in bf16, one counter of the generator.
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
template <typename T> struct Elem;
template <> struct Elem<float> {
  static __device__ __forceinline__ float get(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
  static __device__ __forceinline__ void get8(const float* p, float* x) { load8f(p, x); }
  static __device__ __forceinline__ void put8(float* p, const float* x) { store8f(p, x); }
};
template <> struct Elem<uint16_t> {
  static __device__ __forceinline__ float get(const uint16_t* p) { return bf16_bits_to_float(*p); }
  static __device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }
  static __device__ __forceinline__ void get8(const uint16_t* p, float* x) { GradBF16::unpack(*reinterpret_cast<const uint4*>(p), x); }
  static __device__ __forceinline__ void put8(uint16_t* p, const float* x) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
};

template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* p, int n, float* x) {
  if (VEC && n >= 8) {
    Elem<T>::get8(p, x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < n ? Elem<T>::get(p + e) : 0.f;
  }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, int n, const float* x) {
  if (VEC && n >= 8) {
    Elem<T>::put8(p, x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) Elem<T>::put(p + e, x[e]);
  }
}

// ---- dropout -------------------------------------------------------------------------------------------

struct DropArgs {
  const void* x;
  const void* residual;
  void* y;
  int64_t x_ld, r_ld, y_ld, rows, cols, groups, total;     // groups of eight columns per row, and in all
  DropRule drop;
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dropout_kernel(const DropArgs a) {
  wait_for_previous_kernel();
  const DropKey key = drop_key(a.drop);
  const T* const x = static_cast<const T*>(a.x);
  const T* const res = static_cast<const T*>(a.residual);
  T* const y = static_cast<T*>(a.y);
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < a.total; i0 += 2 * stride) {
    float v[2][8], r[2][8];
    int64_t row[2], col[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t i = i0 + u * stride;
      if (i >= a.total) continue;
      row[u] = a.total <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)a.groups) : i / a.groups;
      col[u] = (i - row[u] * a.groups) * 8;
      const int n = (int)min((int64_t)8, a.cols - col[u]);
      load8<VEC>(x + row[u] * a.x_ld + col[u], n, v[u]);
      if (res) load8<VEC>(res + row[u] * a.r_ld + col[u], n, r[u]);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t i = i0 + u * stride;
      if (i >= a.total) continue;
      if (a.drop.least) drop8(a.drop, key, (uint64_t)i, v[u]);
      if (res) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] += r[u][e];
      }
      store8<VEC>(y + row[u] * a.y_ld + col[u], (int)min((int64_t)8, a.cols - col[u]), v[u]);
    }
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
  int32_t cols, groups, q8_group, n_scales;
  float eps;
  DropRule drop;
};

__device__ __forceinline__ uint32_t pack_e4m3x4(const float* x) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1]), "f"(x[0]));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3]), "f"(x[2]));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// s stays in 32 bits for the statistic and the output and is rounded only where it is stored.
template <typename T, typename W, int NC, bool WARP, bool VEC>
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
  const W* const weight = static_cast<const W*>(a.weight);
  float s[NC][8], r[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int g = me + i * team;
    if (g < a.groups) {
      load8<VEC>(x + 8 * g, a.cols - 8 * g, s[i]);
      if (res) load8<VEC>(res + 8 * g, a.cols - 8 * g, r[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] = 0.f;
    }
  }
  float sq = 0.f;
  const DropKey key = drop_key(a.drop);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int g = me + i * team;
    if (g < a.groups) {
      if (a.drop.least) drop8(a.drop, key, (uint64_t)row * a.groups + g, s[i]);
      if (res) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] += r[i][e];
      }
      if (sum) store8<VEC>(sum + 8 * g, a.cols - 8 * g, s[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = fmaf(s[i][e], s[i][e], sq);
    }
  }
  const float rstd = 1.f / sqrtf(row_sum<WARP>(sq, red[0]) / (float)a.cols + a.eps);
  if (a.rstd && me == 0) a.rstd[row] = rstd;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int g = me + i * team;
    if (g < a.groups) {
      float w[8];
      load8<VEC>(weight + 8 * g, a.cols - 8 * g, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] = s[i][e] * rstd * w[e];
      if (y) store8<VEC>(y + 8 * g, a.cols - 8 * g, s[i]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(s[i][e]));
    if (a.y8 && a.q8_group) {                      // a group of 128 columns: sixteen neighbouring lanes
      float m = top;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      top = 0.f;
      if (g < a.groups) {
        const float inv = m > 0.f ? 448.f / m : 1.f;
        if ((g & 15) == 0) a.scales[row * a.n_scales + (g >> 4)] = m > 0.f ? m / 448.f : 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] *= inv;
      }
    }
  }
  if (!a.y8) return;
  if (!a.q8_group) {
    const float m = row_max<WARP>(top, red[1]);
    const float inv = m > 0.f ? 448.f / m : 1.f;
    if (me == 0) a.scales[row] = m > 0.f ? m / 448.f : 1.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] *= inv;
  }
  uint8_t* const q = a.y8 + row * a.y8_ld;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int g = me + i * team, n = a.cols - 8 * g;
    if (g >= a.groups) continue;
    const uint2 v = make_uint2(pack_e4m3x4(s[i]), pack_e4m3x4(s[i] + 4));
    if (VEC && n >= 8) {
      *reinterpret_cast<uint2*>(q + 8 * g) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) q[8 * g + e] = (uint8_t)((e < 4 ? v.x : v.y) >> (8 * (e & 3)));
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
  int32_t cols, groups;
  DropRule drop;
};

// A CTA takes rows blockIdx, blockIdx + grid, ...; a thread has the same columns in each, whose share of dw it keeps.  NC = 4
// (rows above 8192 columns): dw alone fills the registers, so the row is read a second time, out of L2.
template <typename T, typename W, int NC, bool VEC>
__global__ void __launch_bounds__(NC == 1 ? 256 : NC == 2 ? 512 : 1024) rmsnorm_backward_kernel(const NormGradArgs a) {
  constexpr bool kTwice = NC == 4;
  constexpr int kHeld = kTwice ? 1 : NC;
  __shared__ float red[2][32];
  wait_for_previous_kernel();
  const int team = (int)blockDim.x, me = (int)threadIdx.x;
  const W* const weight = static_cast<const W*>(a.weight);
  const DropKey key = drop_key(a.drop);
  float w[kHeld][8], dw[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int g = me + i * team;
    if (!kTwice) load8<VEC>(weight + 8 * g, g < a.groups ? a.cols - 8 * g : 0, w[i % kHeld]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = 0.f;
  }
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const T* const dy = static_cast<const T*>(a.dy) + row * a.dy_ld;
    const T* const s = static_cast<const T*>(a.sum) + row * a.s_ld;
    const T* const ds_in = a.dsum ? static_cast<const T*>(a.dsum) + row * a.s_ld : nullptr;
    const float rstd = a.rstd[row];
    float g8[kHeld][8], xh[kHeld][8], more[kHeld][8], c = 0.f;
    auto fetch = [&](int i, bool with_more) {
      const int g = me + i * team, n = g < a.groups ? a.cols - 8 * g : 0;
      load8<VEC>(dy + 8 * g, n, g8[i % kHeld]);
      load8<VEC>(s + 8 * g, n, xh[i % kHeld]);
      if (kTwice) load8<VEC>(weight + 8 * g, n, w[0]);
      if (with_more && ds_in) load8<VEC>(ds_in + 8 * g, n, more[i % kHeld]);
    };
    if (!kTwice) {
#pragma unroll
      for (int i = 0; i < NC; ++i) fetch(i, true);
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if (kTwice) fetch(i, false);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float &g = g8[i % kHeld][e], &x = xh[i % kHeld][e];
        x *= rstd;
        dw[i][e] = fmaf(g, x, dw[i][e]);
        g *= w[i % kHeld][e];
        c = fmaf(g, x, c);
      }
    }
    c = row_sum<false>(c, red[turn]) / (float)a.cols;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int g = me + i * team, n = a.cols - 8 * g, h = i % kHeld;
      if (g >= a.groups) continue;
      if (kTwice) {
        fetch(i, true);
#pragma unroll
        for (int e = 0; e < 8; ++e) { xh[h][e] *= rstd; g8[h][e] *= w[h][e]; }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g8[h][e] = rstd * fmaf(-xh[h][e], c, g8[h][e]);
        if (ds_in) g8[h][e] += more[h][e];
      }
      if (a.dres) store8<VEC>(static_cast<T*>(a.dres) + row * a.r_ld + 8 * g, n, g8[h]);
      if (a.dx) {
        if (a.drop.least) drop8(a.drop, key, (uint64_t)row * a.groups + g, g8[h]);
        store8<VEC>(static_cast<T*>(a.dx) + row * a.x_ld + 8 * g, n, g8[h]);
      }
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int g = me + i * team;
    if (g < a.groups) store8<false>(a.partial + (int64_t)blockIdx.x * a.cols + 8 * g, a.cols - 8 * g, dw[i]);
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
  d.least = (uint32_t)std::lrint((double)p * 65536.0);
  d.factor = d.least >= 65536u ? 0.f : (float)(65536.0 / (65536.0 - d.least));
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

// Pitches hold a row, pointers are multiples of their element; `vec`: every row starts on 16 bytes (8 elements of 8 bits on 8).
int check_rows(std::initializer_list<Pitched> all, int64_t rows, int64_t cols, bool& vec) {
  vec = true;
  for (const Pitched& t : all) {
    if (!t.p) continue;
    if (t.ld < cols) return ADAPM_EINVAL;
    if (rows > 1 && t.ld > INT64_MAX / 8 / rows) return ADAPM_ERANGE;
    if ((uintptr_t)t.p % (uintptr_t)t.bytes) return ADAPM_EALIGN;
    const int64_t unit = t.bytes == 1 ? 8 : 16;
    vec = vec && (uintptr_t)t.p % (uintptr_t)unit == 0 && (rows <= 1 || t.ld * t.bytes % unit == 0);
  }
  return ADAPM_OK;
}

int sm_count(int device, int* sms) {
  ADAPM_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
  return ADAPM_OK;
}

// Threads of a CTA that has `groups` chunks of a row, nc at most per thread.
unsigned threads_for(int64_t groups, int nc) { return (unsigned)(((groups + nc - 1) / nc + 31) / 32 * 32); }

template <typename T, typename W, bool VEC>
cudaError_t forward_form(const NormArgs& a, int sms, cudaStream_t s) {
#define ADAPM_WARP(NC) return launch_chained(true, rmsnorm_forward_kernel<T, W, NC, true, VEC>, (unsigned)((a.rows + 3) / 4), 128, 0, s, a)
#define ADAPM_CTA(NC) return launch_chained(true, rmsnorm_forward_kernel<T, W, NC, false, VEC>, (unsigned)a.rows, threads_for(a.groups, NC), 0, s, a)
  // a warp per row where that keeps all SMs busy, else as many threads per row as there are chunks
  if (a.groups <= 256 && a.rows >= 16 * (int64_t)sms) {
    if (a.groups <= 32) ADAPM_WARP(1);
    if (a.groups <= 64) ADAPM_WARP(2);
    if (a.groups <= 128) ADAPM_WARP(4);
    ADAPM_WARP(8);
  }
  if (a.groups <= 512) ADAPM_CTA(1);
  if (a.groups <= 1024) ADAPM_CTA(2);
  ADAPM_CTA(4);
#undef ADAPM_WARP
#undef ADAPM_CTA
}

struct GradForm { int nc; unsigned threads; int ctas; };
// One chunk per thread up to 256 threads, then two, then four; as many CTAs as fit.
GradForm grad_form(int64_t rows, int64_t groups, int sms) {
  GradForm f;
  f.nc = groups <= 256 ? 1 : groups <= 1024 ? 2 : 4;
  f.threads = threads_for(groups, f.nc);
  f.ctas = (int)std::min<int64_t>(rows, (int64_t)sms * std::max(1, 1024 / (int)f.threads));
  return f;
}

template <typename T, typename W, bool VEC>
cudaError_t backward_form(const NormGradArgs& a, const GradForm& f, cudaStream_t s) {
  if (f.nc == 1) return launch_chained(true, rmsnorm_backward_kernel<T, W, 1, VEC>, (unsigned)f.ctas, f.threads, 0, s, a);
  if (f.nc == 2) return launch_chained(true, rmsnorm_backward_kernel<T, W, 2, VEC>, (unsigned)f.ctas, f.threads, 0, s, a);
  return launch_chained(true, rmsnorm_backward_kernel<T, W, 4, VEC>, (unsigned)f.ctas, f.threads, 0, s, a);
}

#define ADAPM_FORMS(F, vec, t, w, ...)                                                                          \
  ((vec) ? ((t) == ADAPM_TYPE_F32 ? ((w) == ADAPM_TYPE_F32 ? F<float, float, true>(__VA_ARGS__) : F<float, uint16_t, true>(__VA_ARGS__))          \
                                  : ((w) == ADAPM_TYPE_F32 ? F<uint16_t, float, true>(__VA_ARGS__) : F<uint16_t, uint16_t, true>(__VA_ARGS__)))   \
         : ((t) == ADAPM_TYPE_F32 ? ((w) == ADAPM_TYPE_F32 ? F<float, float, false>(__VA_ARGS__) : F<float, uint16_t, false>(__VA_ARGS__))        \
                                  : ((w) == ADAPM_TYPE_F32 ? F<uint16_t, float, false>(__VA_ARGS__) : F<uint16_t, uint16_t, false>(__VA_ARGS__))))

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
  bool vec;
  rc = check_rows({{x, x_ld, eb}, {residual, residual_ld, eb}, {y, y_ld, eb}}, rows, cols, vec);
  if (rc != ADAPM_OK) return rc;
  if ((uintptr_t)step % 8) return ADAPM_EALIGN;
  int device, sms;
  rc = check_on_this_device({x, residual, y, step}, &device);
  if (rc == ADAPM_OK) rc = sm_count(device, &sms);
  if (rc != ADAPM_OK) return rc;
  a.x = x; a.residual = residual; a.y = y;
  a.x_ld = x_ld; a.r_ld = residual_ld; a.y_ld = y_ld; a.rows = rows; a.cols = cols;
  a.groups = (cols + 7) / 8; a.total = rows * a.groups;
  cudaStream_t s = (cudaStream_t)stream;
  const unsigned grid = (unsigned)std::min<int64_t>((a.total + 511) / 512, (int64_t)sms * 64);
  const bool f32 = dtype == ADAPM_TYPE_F32;
  ADAPM_CUDA(f32 ? (vec ? launch_chained(true, dropout_kernel<float, true>, grid, 256, 0, s, a) : launch_chained(true, dropout_kernel<float, false>, grid, 256, 0, s, a))
                 : (vec ? launch_chained(true, dropout_kernel<uint16_t, true>, grid, 256, 0, s, a) : launch_chained(true, dropout_kernel<uint16_t, false>, grid, 256, 0, s, a)));
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
  bool vec;
  rc = check_rows({{x, d->x_ld, eb}, {residual, d->residual_ld, eb}, {sum, d->sum_ld, eb}, {y, d->y_ld, eb}, {y8, d->y8_ld, 1}}, d->rows,
                  d->cols, vec);
  if (rc != ADAPM_OK) return rc;
  vec = vec && (uintptr_t)weight % 16 == 0;
  if ((uintptr_t)weight % (uintptr_t)type_bytes(d->weight_dtype) || (uintptr_t)y8_scales % 4 || (uintptr_t)rstd % 4 || (uintptr_t)d->step % 8) return ADAPM_EALIGN;
  if (overlap(sum, ((d->rows - 1) * d->sum_ld + d->cols) * eb, y, ((d->rows - 1) * d->y_ld + d->cols) * eb)) {
    set_error_text("adapm_rmsnorm_forward: the sum and the output overlap");
    return ADAPM_EINVAL;
  }
  int device, sms;
  rc = check_on_this_device({x, residual, weight, sum, y, y8, y8_scales, rstd, d->step}, &device);
  if (rc == ADAPM_OK) rc = sm_count(device, &sms);
  if (rc != ADAPM_OK) return rc;
  a.x = x; a.residual = residual; a.weight = weight; a.sum = sum; a.y = y; a.y8 = (uint8_t*)y8; a.scales = y8_scales; a.rstd = rstd;
  a.x_ld = d->x_ld; a.r_ld = d->residual_ld; a.s_ld = d->sum_ld; a.y_ld = d->y_ld; a.y8_ld = d->y8_ld; a.rows = d->rows;
  a.cols = (int32_t)d->cols; a.groups = (int32_t)((d->cols + 7) / 8); a.q8_group = d->q8_group;
  a.n_scales = d->q8_group ? (int32_t)((d->cols + 127) / 128) : 1;
  a.eps = d->eps;
  ADAPM_CUDA(ADAPM_FORMS(forward_form, vec, d->dtype, d->weight_dtype, a, sms, (cudaStream_t)stream));
  return ADAPM_OK;
}

extern "C" size_t adapm_rmsnorm_backward_scratch_bytes(const adapm_rmsnorm* d) {
  DropRule drop;
  if (!d || check_desc(*d, drop) != ADAPM_OK) return 0;
  // the largest grid of any row length, on a device of up to 256 SMs
  const GradForm f = grad_form(std::max<int64_t>(d->rows, 1), (d->cols + 7) / 8, 256);
  return (size_t)round_up((int64_t)f.ctas * d->cols * 4, 256);
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
  bool vec;
  rc = check_rows({{dy, d->y_ld, eb}, {dsum, d->sum_ld, eb}, {sum, d->sum_ld, eb}, {dresidual, d->residual_ld, eb}, {dx, d->x_ld, eb}},
                  d->rows, d->cols, vec);
  if (rc != ADAPM_OK) return rc;
  vec = vec && (uintptr_t)weight % 16 == 0;
  if ((uintptr_t)weight % (uintptr_t)type_bytes(d->weight_dtype) || (uintptr_t)rstd % 4 || (uintptr_t)d->step % 8) return ADAPM_EALIGN;
  if (overlap(dresidual, ((d->rows - 1) * d->residual_ld + d->cols) * eb, dx, ((d->rows - 1) * d->x_ld + d->cols) * eb)) {
    set_error_text("adapm_rmsnorm_backward: the two gradients overlap");
    return ADAPM_EINVAL;
  }
  if (dweight) {
    if (!scratch) return ADAPM_EINVAL;
    if ((uintptr_t)scratch % 256) return ADAPM_EALIGN;
    if (scratch_bytes < adapm_rmsnorm_backward_scratch_bytes(d)) return ADAPM_ENOWORKSPACE;
  }
  rc = check_on_this_device({dy, dsum, sum, rstd, weight, dresidual, dx, dweight, dweight ? scratch : nullptr, d->step}, &device);
  if (rc == ADAPM_OK) rc = sm_count(device, &sms);
  if (rc != ADAPM_OK) return rc;
  a.dy = dy; a.dsum = dsum; a.sum = sum; a.rstd = rstd; a.weight = weight; a.dres = dresidual; a.dx = dx;
  a.partial = dweight ? (float*)scratch : nullptr;
  a.dy_ld = d->y_ld; a.s_ld = d->sum_ld; a.r_ld = d->residual_ld; a.x_ld = d->x_ld; a.rows = d->rows;
  a.cols = (int32_t)d->cols; a.groups = (int32_t)((d->cols + 7) / 8);
  const GradForm f = grad_form(d->rows, a.groups, std::min(sms, 256));
  ADAPM_CUDA(ADAPM_FORMS(backward_form, vec, d->dtype, d->weight_dtype, a, f, s));
  if (!dweight) return ADAPM_OK;
  const unsigned grid = (unsigned)((d->cols + 31) / 32);
  ADAPM_CUDA(dweight_dtype == ADAPM_TYPE_F32
                 ? launch_chained(true, column_sum_kernel<float>, grid, 1024, 0, s, (const float*)scratch, f.ctas, a.cols, (float*)dweight, (int)(accumulate != 0))
                 : launch_chained(true, column_sum_kernel<uint16_t>, grid, 1024, 0, s, (const float*)scratch, f.ctas, a.cols, (uint16_t*)dweight, (int)(accumulate != 0)));
  return ADAPM_OK;
}
