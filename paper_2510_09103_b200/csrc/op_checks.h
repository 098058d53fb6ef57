// Checks that the stand-alone operators (dropout, RMS norm, head loss) make of their arguments before anything is launched.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "adapm_internal.h"

namespace adapm {

void set_error_text(const char* text);   // ctx.cu
// quant8.cu: codes to numbers, its arguments checked before
int launch_dequant8(const adapm_codes8& d, const void* codes, const float* scales, void* x, cudaStream_t s);

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

// Where a matrix lies: `rows` rows of `bytes` bytes, `pitch` bytes apart.  A vector is one row.  (Null: nowhere.)
struct Place {
  const void* p;
  int64_t rows, pitch, bytes;
  uint64_t begin() const { return (uint64_t)(uintptr_t)p; }
  uint64_t end() const { return begin() + (uint64_t)((rows - 1) * pitch + bytes); }
};
inline Place matrix_at(const void* p, int64_t rows, int64_t ld, int64_t cols, int64_t bytes) {
  return Place{p, rows, (rows > 1 ? ld : cols) * bytes, cols * bytes};
}
inline Place vector_at(const void* p, int64_t n, int64_t bytes) { return Place{p, 1, n * bytes, n * bytes}; }

// Whether two matrices share a byte.  What lies between the rows of one belongs to neither, so that another one of the same pitch may
// lie there; two matrices of different pitches count as sharing where one begins before the other ends.
inline bool share(const Place& a, const Place& b) {
  if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.bytes <= 0 || b.bytes <= 0) return false;
  if (a.begin() >= b.end() || b.begin() >= a.end()) return false;
  if (a.rows == 1 || b.rows == 1) {
    const Place &one = a.rows == 1 ? a : b, &m = a.rows == 1 ? b : a;
    if (m.rows == 1) return true;
    // the first row of m that ends behind the beginning of the other
    const uint64_t pitch = (uint64_t)m.pitch, first_end = m.begin() + (uint64_t)m.bytes;
    const uint64_t k = one.begin() < first_end ? 0 : (one.begin() - first_end) / pitch + 1;
    return k < (uint64_t)m.rows && m.begin() + k * pitch < one.end();
  }
  if (a.pitch != b.pitch) return true;
  const uint64_t pitch = (uint64_t)a.pitch, ahead = a.begin() <= b.begin() ? (b.begin() - a.begin()) % pitch : (pitch - (a.begin() - b.begin()) % pitch) % pitch;
  return ahead < (uint64_t)a.bytes || ahead + (uint64_t)b.bytes > pitch;
}

// Whether an output may lie where an input does: apart, or element on element.
inline bool apart_or_same(const Place& out, const Place& in) {
  return (out.p == in.p && out.bytes == in.bytes && out.pitch == in.pitch) || !share(out, in);
}

}  // namespace adapm
