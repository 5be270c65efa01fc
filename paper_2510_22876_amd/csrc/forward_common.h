// Device helpers of the forward-side kernels (append, attention, logits):
// conversions between fp32 and the 16-bit types, and a cache's entries by
// (sequence, index).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "span_copy.h"
#include "specdec_internal.h"

namespace specdec {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int kDtype> struct Element;   // 0 f32, 1 bf16, 2 f16 (specdec_dtype_t)
template <> struct Element<0> { typedef float type; };
template <> struct Element<1> { typedef __bf16 type; };
template <> struct Element<2> { typedef _Float16 type; };

// Loads or stores kN consecutive elements; the address needs the element's
// alignment only (the compiler emits wide accesses, which gfx950 does at any
// alignment).
template <typename T, int kN>
__device__ __forceinline__ void load_elements(const T* p, float (&x)[kN]) {
  T v[kN];
  __builtin_memcpy(v, p, sizeof(v));
#pragma unroll
  for (int i = 0; i < kN; ++i) x[i] = static_cast<float>(v[i]);
}
template <typename T, int kN>
__device__ __forceinline__ void store_elements(T* p, const float (&x)[kN]) {
  T v[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = static_cast<T>(x[i]);   // rounds to nearest even
  __builtin_memcpy(p, v, sizeof(v));
}

// Runs `launch(first workgroup, workgroups)` for a grid of `blocks` workgroups
// of `threads` work-items each, in as many launches as one launch's limit on
// work-items asks for.
template <typename F>
hipError_t launch_blocks(int64_t blocks, int threads, F&& launch) {
  int64_t most = max_launch_items() / threads;
  if (most < 1) most = 1;
  if (most > 0x7FFFFFFF) most = 0x7FFFFFFF;
  for (int64_t at = 0; at < blocks; at += most) {
    launch(at, static_cast<uint32_t>(blocks - at < most ? blocks - at : most));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Entries in front of sequence i's window, or -1 where the sequence's padding
// or length is out of range.
__device__ __forceinline__ int32_t entries_before(const CacheView& c, int32_t i, int32_t T) {
  if (c.table) {
    const int32_t n = load_invariant(c.lens + i);
    return n < 0 || n > c.width - T ? -1 : n;
  }
  const int32_t pad = load_invariant(c.lens + i), L = c.width - T;
  return pad < 0 || pad > L ? -1 : L - pad;
}

}  // namespace specdec
