// Host-side argument checks shared by the library's entry points (internal).
#pragma once

#include <cuda_runtime.h>
#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "flashslice.h"

namespace fs {

inline bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A byte range [p, p + n) of a caller buffer.
struct Span {
  const void* p;
  size_t n;
};
// True when two ranges share a byte (a null range shares none).
inline bool overlap(Span a, Span b) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.n && b.n && a0 < b0 + b.n && b0 < a0 + a.n;
}
// The out-of-place calls read every input while they write: no output may share a byte with
// an input or with another output.
inline bool disjoint(std::initializer_list<Span> ins, std::initializer_list<Span> outs) {
  for (const Span& o : outs) {
    for (const Span& i : ins)
      if (overlap(o, i)) return false;
    for (const Span& o2 : outs)
      if (&o2 != &o && overlap(o, o2)) return false;
  }
  return true;
}

inline fs_status cuda_status(cudaError_t e) { return e == cudaSuccess ? FS_OK : FS_ERR_CUDA; }

}  // namespace fs

#define FS_CHECK_PTR(p)                                      \
  do {                                                       \
    if (!(p) || !fs::aligned(p)) return FS_ERR_INVALID;      \
  } while (0)
// An argument that may be NULL.
#define FS_CHECK_OPT(p)                                      \
  do {                                                       \
    if (!fs::aligned(p)) return FS_ERR_INVALID;              \
  } while (0)

#define FS_CUDA(call)                                        \
  do {                                                       \
    cudaError_t e_ = (call);                                 \
    if (e_ != cudaSuccess) return FS_ERR_CUDA;               \
  } while (0)
