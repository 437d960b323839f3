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

// The same for rows of less than 2^28 elements that begin at a place the wavefront shares: one load whatever the row's end is,
// the last piece's from the row's last 16 bytes, moved down.
template <class T>
__device__ inline u32x4 near_piece(const T* x, int i, int n) {
  constexpr int E = kPiece<T>;
  u32x4 c;
  if (n < E) {
    T e[E];
#pragma unroll
    for (int k = 0; k < E; ++k) e[k] = i == 0 && k < n ? x[k] : T(0.0f);
    __builtin_memcpy(&c, e, 16);
    return c;
  }
  const int from = i * E < n - E ? i * E : n - E, over = i * E - from;
  __builtin_memcpy(&c, reinterpret_cast<const char*>(x) + unsigned(from) * unsigned(sizeof(T)), 16);
  if (over > 0) {
    unsigned __int128 all = 0;
    __builtin_memcpy(&all, &c, 16);
    all = over < E ? all >> (over * int(sizeof(T)) * 8) : 0;
    __builtin_memcpy(&c, &all, 16);
  }
  return c;
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

// Sums over the W threads of a row, one of R rows of a workgroup: a wavefront by itself, or wavefronts whose sums meet in LDS.  Two
// places take turns: who writes one again has passed the other's barrier, before which every wavefront has read it.
template <int W, int R = 1>
struct RowSums {
  typedef float Meet[2][2][R * W / kWave];
  Meet& meet;
  int slot, turn = 0;
  __device__ explicit RowSums(Meet& m, int slot = 0) : meet(m), slot(slot) {}

  __device__ float gather(int which) const {
    const float* at = meet[turn][which] + slot * (W / kWave);
    float v = at[0];
#pragma unroll
    for (int i = 1; i < W / kWave; ++i) v += at[i];
    return v;
  }
  __device__ void two(float& a, float& b) {
    a = wave_total(a);
    b = wave_total(b);
    if constexpr (W > kWave) {
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
    a = wave_total(a);
    if constexpr (W > kWave) {
      if ((threadIdx.x & 63) == 0) meet[turn][0][threadIdx.x >> 6] = a;
      __syncthreads();
      a = gather(0);
      turn ^= 1;
    }
    return a;
  }
};

constexpr int64_t kMostRows = int64_t(1) << 31, kMostLd = int64_t(1) << 40;
inline bool ld_ok(int64_t ld, int64_t width) { return ld >= width && ld < kMostLd; }
inline bool type_ok(int dtype) { return dtype >= XMEM_BF16 && dtype <= XMEM_F32; }

}  // namespace xops
