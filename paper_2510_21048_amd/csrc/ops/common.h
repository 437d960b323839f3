// common.h -- what the training operators' kernels share: element types, rounding, reductions.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ops/xmem_ops.h"

namespace xops {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

template <class T> struct Vec;  // eight 16-bit elements: what a lane holds of an operand
template <> struct Vec<bf16> {
  typedef bf16 x8 __attribute__((ext_vector_type(8)));
};
template <> struct Vec<f16> {
  typedef f16 x8 __attribute__((ext_vector_type(8)));
};

constexpr int kWave = 64;
constexpr int kCus = 256;
constexpr int kXcds = 8;
// Threads of one launch: a grid of 2^32 and more is refused, or run without its upper bits.
constexpr int64_t kMostThreads = int64_t(1) << 31;

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline size_t up256(size_t b) { return (b + 255) & ~size_t(255); }
inline int launched() { return hipGetLastError() == hipSuccess ? XMEM_OK : XMEM_EHIP; }

// Sums over the wavefront, every lane getting the result.  The order is fixed.
__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

}  // namespace xops
