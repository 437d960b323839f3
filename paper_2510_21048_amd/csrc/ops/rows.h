// rows.h -- what kernels over the rows of a matrix share: 16-byte pieces of any alignment, sums over a row's threads.
#pragma once
#include "common.h"
#include "ops/xmem_step.h"

namespace xops {

// Elements of a piece of 16 bytes.
template <class T> constexpr int kPiece = 16 / sizeof(T);

// Piece i of a row of n elements as it lies; 0 behind the row's end, where nothing is read.
template <class T>
__device__ inline u32x4 piece_of(const T* x, int64_t i, int64_t n) {
  constexpr int E = kPiece<T>;
  u32x4 c;
  if ((i + 1) * E <= n) {
    __builtin_memcpy(&c, x + i * E, 16);
  } else {
    T e[E];
#pragma unroll
    for (int k = 0; k < E; ++k) e[k] = i * E + k < n ? x[i * E + k] : T(0.0f);
    __builtin_memcpy(&c, e, 16);
  }
  return c;
}

// Where piece i of a row of n >= E elements is read and written: at i * E, but not past n - E.  The first `over` of its elements (all,
// where it is not smaller than E) are then other threads' too, which have the same values for them; they do not count in sums.
template <int E>
struct Place {
  int at, over;
  __device__ Place(int i, int n) : at(i * E < n - E ? i * E : n - E), over(i * E - at) {}
  __device__ void counted(float (&v)[E]) const {
    if (over > 0)
#pragma unroll
      for (int k = 0; k < E; ++k) v[k] = k < over ? 0.0f : v[k];
  }
};
template <class T>
__device__ inline u32x4 piece_at(const T* x, int at) {
  u32x4 c;
  __builtin_memcpy(&c, reinterpret_cast<const char*>(x) + unsigned(at) * unsigned(sizeof(T)), 16);
  return c;
}
template <class T>
__device__ inline void put_piece_at(T* x, int at, const float (&v)[kPiece<T>]) {
  T e[kPiece<T>];
#pragma unroll
  for (int k = 0; k < kPiece<T>; ++k) e[k] = T(v[k]);
  __builtin_memcpy(reinterpret_cast<char*>(x) + unsigned(at) * unsigned(sizeof(T)), e, 16);
}
// 16 bytes to a place of any alignment, past the caches: where they would only push out what is read again.
__device__ inline void store_past(void* to, u32x4 c) {
  typedef unsigned any4 __attribute__((ext_vector_type(4), aligned(2)));
  __builtin_nontemporal_store(any4(c), static_cast<any4*>(to));
}
template <class T>
__device__ inline void put_piece_past(T* x, int at, const float (&v)[kPiece<T>]) {
  T e[kPiece<T>];
#pragma unroll
  for (int k = 0; k < kPiece<T>; ++k) e[k] = T(v[k]);
  u32x4 c;
  __builtin_memcpy(&c, e, 16);
  store_past(reinterpret_cast<char*>(x) + unsigned(at) * unsigned(sizeof(T)), c);
}
template <int E>
__device__ inline void vector_at(const float* w, int at, float without, float (&v)[E]) {
  if (w) {
    __builtin_memcpy(v, reinterpret_cast<const char*>(w) + unsigned(at) * 4u, sizeof(v));
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = without;
  }
}

template <class T>
__device__ inline void unpack(u32x4 c, float (&v)[kPiece<T>]) {
  T e[kPiece<T>];
  __builtin_memcpy(e, &c, 16);
#pragma unroll
  for (int k = 0; k < kPiece<T>; ++k) v[k] = float(e[k]);
}

template <class T>
__device__ inline void put_piece(T* x, int64_t i, int64_t n, const float (&v)[kPiece<T>]) {
  constexpr int E = kPiece<T>;
  T e[E];
#pragma unroll
  for (int k = 0; k < E; ++k) e[k] = T(v[k]);
  if ((i + 1) * E <= n) {
    __builtin_memcpy(x + i * E, e, 16);
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (i * E + k < n) x[i * E + k] = e[k];
  }
}

// E neighbouring elements of a vector of n from element i * E; `without` where there is no vector or no element.
template <int E>
__device__ inline void vector_of(const float* w, int64_t i, int64_t n, float without, float (&v)[E]) {
  if (w && (i + 1) * E <= n) {
    __builtin_memcpy(v, w + i * E, sizeof(v));
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = w && i * E + k < n ? w[i * E + k] : without;
  }
}

template <int E>
__device__ inline void put_vector(float* w, int64_t i, int64_t n, const float (&v)[E]) {
  if ((i + 1) * E <= n) {
    __builtin_memcpy(w + i * E, v, sizeof(v));
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (i * E + k < n) w[i * E + k] = v[k];
  }
}

// The sum over a wavefront's lanes, by data-parallel primitives: rows of 16 lanes, then across them; the same in every lane.
template <int CTRL, int ROWS>
__device__ inline float from_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ inline float wave_total(float v) {
  v += from_lane<0x111, 0xf>(v);  // row_shr by 1, 2, 4, 8
  v += from_lane<0x112, 0xf>(v);
  v += from_lane<0x114, 0xf>(v);
  v += from_lane<0x118, 0xf>(v);
  v += from_lane<0x142, 0xa>(v);  // the last lane of a row to the next one
  v += from_lane<0x143, 0xc>(v);  // lane 31 to the upper half
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// The sum over each W neighbouring lanes, in all of them.
template <int W>
__device__ inline float lanes_total(float v) {
  if constexpr (W == kWave) {
    return wave_total(v);
  } else {
    if constexpr (W > 1) v += from_lane<0xb1, 0xf>(v);   // the other of a pair
    if constexpr (W > 2) v += from_lane<0x4e, 0xf>(v);   // the other pair of four
    if constexpr (W > 4) v += from_lane<0x141, 0xf>(v);  // the other half of eight
    if constexpr (W > 8) v += from_lane<0x140, 0xf>(v);  // of sixteen
    if constexpr (W > 16) v += __shfl_xor(v, 16);
    return v;
  }
}

// Sums over the W threads of a row, one of R rows of a workgroup: in a wavefront by themselves, or in wavefronts whose sums meet in
// LDS.  Two places take turns: who writes one again has passed the other's barrier, before which every wavefront has read it.
template <int W, int R = 1>
struct RowSums {
  static constexpr int kParts = W > kWave ? W / kWave : 1;  // wavefronts of a row
  typedef float Meet[2][2][R * kParts];
  Meet& meet;
  int slot, turn = 0;
  __device__ explicit RowSums(Meet& m, int slot = 0) : meet(m), slot(slot) {}

  __device__ float gather(int which) const {
    const float* at = meet[turn][which] + slot * kParts;
    float v = at[0];
#pragma unroll
    for (int i = 1; i < kParts; ++i) v += at[i];
    return v;
  }
  __device__ void two(float& a, float& b) {
    if constexpr (W <= kWave) {
      a = lanes_total<W>(a);
      b = lanes_total<W>(b);
    } else {
      a = wave_total(a);
      b = wave_total(b);
      if ((threadIdx.x & 63) == 0) {
        meet[turn][0][threadIdx.x >> 6] = a;
        meet[turn][1][threadIdx.x >> 6] = b;
      }
      __syncthreads();
      a = gather(0);
      b = gather(1);
      turn ^= 1;
    }
  }
  __device__ float one(float a) {
    if constexpr (W <= kWave) {
      a = lanes_total<W>(a);
    } else {
      a = wave_total(a);
      if ((threadIdx.x & 63) == 0) meet[turn][0][threadIdx.x >> 6] = a;
      __syncthreads();
      a = gather(0);
      turn ^= 1;
    }
    return a;
  }
};

constexpr int64_t kCacheBytes = int64_t(256) << 20;  // of the cache behind the L2s
constexpr int64_t kMostRows = int64_t(1) << 31, kMostLd = int64_t(1) << 40;
inline bool ld_ok(int64_t ld, int64_t width) { return ld >= width && ld < kMostLd; }
inline bool type_ok(int dtype) { return dtype >= XMEM_BF16 && dtype <= XMEM_F32; }

// Whether `bytes` of workspace have one in common with a matrix: they may lie between two of its rows.  Sizes and distances as the calls
// take them pass 64 bits.
inline bool shares(const void* workspace, size_t bytes, const void* x, int64_t rows, int64_t ld, int64_t width, int element) {
  if (!x || rows <= 0 || width <= 0 || !bytes) return false;
  typedef __int128 Wide;
  const Wide ws = reinterpret_cast<uintptr_t>(workspace), at = reinterpret_cast<uintptr_t>(x), step = Wide(ld) * element, row = Wide(width) * element;
  if (ws + Wide(bytes) <= at || ws >= at + (rows - 1) * step + row) return false;
  if (ws < at) return true;
  const Wide behind = (ws - at) % step;  // the row's beginning that is at or before the workspace's
  return behind < row || behind + Wide(bytes) > step;
}

}  // namespace xops
