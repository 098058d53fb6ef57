// Checks that the stand-alone operators (dropout, RMS norm, head loss) make of their arguments before anything is launched.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "adapm_internal.h"

namespace adapm {

void set_error_text(const char* text);   // ctx.cu

inline bool known_type(int32_t t) { return t == ADAPM_TYPE_F32 || t == ADAPM_TYPE_BF16; }
inline int64_t type_bytes(int32_t t) { return t == ADAPM_TYPE_F32 ? 4 : 2; }

// Every pointer that is not null has to be memory that the current device can address as its own: a host address or another
// device's memory would fault the kernel.  (About 0.1 us each.)
inline int check_on_this_device(std::initializer_list<const void*> ptrs, int* device) {
  ADAPM_CUDA(cudaGetDevice(device));
  for (const void* p : ptrs) {
    if (!p) continue;
    cudaPointerAttributes at;
    ADAPM_CUDA(cudaPointerGetAttributes(&at, p));
    if (at.type == cudaMemoryTypeManaged) continue;
    if (at.type != cudaMemoryTypeDevice || at.device != *device) {
      set_error_text("a buffer is not memory of the current device");
      return ADAPM_EINVAL;
    }
  }
  return ADAPM_OK;
}

// Whether [a, a + an) and [b, b + bn) share a byte (null ranges do not).
inline bool overlap(const void* a, int64_t an, const void* b, int64_t bn) {
  if (!a || !b) return false;
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + (uintptr_t)bn && y < x + (uintptr_t)an;
}

// Whether an output [rows, cols] may lie where an input does: apart, or element on element.
inline bool apart_or_same(const void* out, int64_t out_ld, const void* in, int64_t in_ld, int64_t rows, int64_t cols, int64_t bytes) {
  if (out == in && (out_ld == in_ld || rows <= 1)) return true;
  return !overlap(out, ((rows - 1) * out_ld + cols) * bytes, in, ((rows - 1) * in_ld + cols) * bytes);
}

}  // namespace adapm
