// The counter-based generator of dropout: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", SC 2011).  A counter gives 128 bits, which serve eight elements with 16 bits each, so that the mask of any
// element can be made again from (seed, offset, row, column) and is never stored.
#pragma once

#include <stdint.h>

namespace adapm {

struct Philox4 { uint32_t w[4]; };

__host__ __device__ __forceinline__ Philox4 philox4x32_10(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Philox4{{c0, c1, c2, c3}};
}

// Dropout of one call: elements whose 16 bits are below `least` = rint(65536 p) become zero, the others are multiplied by `factor`.
// 16 bits: p is taken to the nearest multiple of 2^-16 (7.6e-6 at most), and the factor is the one that belongs to that
// multiple, so that the expectation is kept.
struct DropRule {
  uint32_t cut;                // least << 16
  uint32_t mode;               // 0: nothing is dropped, 1: by the generator, 2: everything (least = 65536)
  float factor;
  uint32_t seed_lo, seed_hi;
  uint64_t offset;
  const uint64_t* step;        // device, added to the offset; may be null
};

#ifdef __CUDACC__
// Two fp32 operations per instruction (the same roundings as one at a time).
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmul.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nadd.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n.reg .b64 x, y, z, w;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmov.b64 z, {%6, %7};\nfma.rn.f32x2 w, x, y, z;\nmov.b64 {%0, %1}, w;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

struct DropKey { uint32_t off_lo, off_hi; };
__device__ __forceinline__ DropKey drop_key(const DropRule& d) {
  const uint64_t off = d.offset + (d.step ? *d.step : 0);
  return DropKey{(uint32_t)off, (uint32_t)(off >> 32)};
}
// The 128 bits of group `q` = row * ceil(cols / 8) + column / 8.  They follow from the place alone: a kernel makes them while
// its elements are on their way.
__device__ __forceinline__ Philox4 drop_bits(const DropRule& d, const DropKey& k, uint64_t q) {
  return philox4x32_10((uint32_t)q, (uint32_t)(q >> 32), k.off_lo, k.off_hi, d.seed_lo, d.seed_hi);
}
// Its eight elements.  Dropped ones are zero whatever they held.  (The upper 16 bits are compared in place, below the cut's
// zeros; the lower ones after a shift.)
__device__ __forceinline__ void drop8(const DropRule& d, const Philox4& r, float* x) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = (r.w[e] << 16) >= d.cut ? x[2 * e] * d.factor : 0.f;
    x[2 * e + 1] = r.w[e] >= d.cut ? x[2 * e + 1] * d.factor : 0.f;
  }
  if (d.mode == 2) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
  }
}
#endif

}  // namespace adapm
