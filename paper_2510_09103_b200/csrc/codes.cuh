// Codes of 8 bits back to fp32, shared by the operators that read them.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "philox.cuh"

namespace adapm {

// The four codes of a word as numbers.  int8: the byte, shifted to 0 .. 255, becomes the low bits of a number from 2^23 on, whose
// excess is taken off exactly (one permutation and one addition per code; no conversion unit is asked).
template <bool E4M3>
__device__ __forceinline__ void unpack4(uint32_t w, float* x) {
  if (E4M3) {
    uint32_t lo, hi;
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&lo)), q = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    x[0] = p.x; x[1] = p.y; x[2] = q.x; x[3] = q.y;
  } else {
    const uint32_t u = w ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const float2 t = add2(make_float2(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440u + (uint32_t)i)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7441u + (uint32_t)i))),
                            make_float2(-8388736.f, -8388736.f));
      x[i] = t.x; x[i + 1] = t.y;
    }
  }
}

}  // namespace adapm
