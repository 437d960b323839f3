// gemm.h -- the matrix product of the training operators: out(m, n) = sum over k of A(m, k) B(n, k), with
// 16-bit operands, 32-bit sums on the matrix cores, and an epilogue that sees each sum once.
//
// Either operand may lie with k contiguous (A[m * ld + k]) or with its rows contiguous (A[k * ld + m]), so
// the three products of a linear layer (x w^T, dz w, dz^T x) need no transposed copy.
#pragma once
#include "common.h"

namespace xops {

constexpr int kBK = 64;  // k of one tile: 128 bytes of an operand row

struct GemmArgs {
  const void* a;
  const void* b;
  int64_t lda, ldb;
  int64_t stride_a, stride_b;  // between the matrices of a batch (grid z), in elements
  int64_t m, n, k;
  int tiles_m, tiles_n;
};

// One operand tile in LDS: R rows of kBK.  Chunks of 16 bytes are kept at swizzled places, so that the 16 lanes
// that read one column of chunks meet 16 different bank groups.
//   k contiguous:    [row][8 chunks of k],   chunk c at c ^ ((row >> 1) & 7)
//   rows contiguous: [k][R / 8 chunks of rows], pairs of chunks (the 16 rows of one product) at p ^ h(k)
template <class T, int R, bool KC>
struct Tile {
  typedef typename Vec<T>::x8 x8;
  static constexpr int kBytes = R * kBK * 2;
  static constexpr int kChunks = R * kBK / 8;

  __device__ static int pair_hash(int k) { return ((k & 3) | ((k >> 1) & 4)) & (R / 16 - 1); }
  // the row (or rows) and k of the chunk kept at place i
  __device__ static void at(int i, int& row, int& k) {
    if constexpr (KC) {
      row = i >> 3;
      k = ((i & 7) ^ ((row >> 1) & 7)) * 8;
    } else {
      k = i / (R / 8);
      const int c = i % (R / 8);
      row = (((c >> 1) ^ pair_hash(k)) * 2 + (c & 1)) * 8;
    }
  }
  // the operand of a 16x16x32 product: rows r0..r0+15 (r0 a multiple of 16), step s of the tile's k.
  // Lane l holds row l % 16, k = 32 s + 8 (l / 16) + 0..7.
  __device__ static x8 frag(const char* t, int r0, int s, int lane) {
    if constexpr (KC) {
      const int row = r0 + (lane & 15), c = 4 * s + (lane >> 4);
      return *reinterpret_cast<const x8*>(t + row * (kBK * 2) + ((c ^ ((row >> 1) & 7)) << 4));
    } else {
      // a transposing read: lane 4 r + q of 16 reads four rows at k + r and gets four k of row 4 q + r's column
      typedef short s4 __attribute__((ext_vector_type(4)));
      typedef short s8 __attribute__((ext_vector_type(8)));
      typedef __attribute__((address_space(3))) s4* lds4;
      const int k = 32 * s + 8 * (lane >> 4) + ((lane >> 2) & 3);
      const char* p0 = t + k * (R * 2) + (((r0 >> 4) ^ pair_hash(k)) << 5) + ((lane & 3) << 3);
      const char* p1 = t + (k + 4) * (R * 2) + (((r0 >> 4) ^ pair_hash(k + 4)) << 5) + ((lane & 3) << 3);
      const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p0));
      const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p1));
      const s8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(x8, v);
    }
  }
};

__device__ inline f32x4 mfma(Vec<bf16>::x8 a, Vec<bf16>::x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma(Vec<f16>::x8 a, Vec<f16>::x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight elements from p, of which only those below `valid` exist (the others are 0).
template <class T>
__device__ inline u32x4 load8(const T* p, int64_t valid) {
  u32x4 v = {0, 0, 0, 0};
  if (valid >= 8) {
    __builtin_memcpy(&v, p, 16);
  } else if (valid > 0) {
    T e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = j < valid ? p[j] : T(0.0f);
    __builtin_memcpy(&v, e, 16);
  }
  return v;
}

// Loads one tile through registers, for operands of any alignment; rows and k past the matrix are 0.
template <class T, int R, bool KC, int THREADS>
__device__ inline void stage(char* lds, const T* p, int64_t ld, int64_t r0, int64_t rows, int64_t k0, int64_t ks) {
  typedef Tile<T, R, KC> Ti;
#pragma unroll
  for (int j = 0; j < Ti::kChunks / THREADS; ++j) {
    const int i = j * THREADS + threadIdx.x;
    int row, k;
    Ti::at(i, row, k);
    const int64_t gr = r0 + row, gk = k0 + k;
    u32x4 v = {0, 0, 0, 0};
    if (gr < rows && gk < ks) v = KC ? load8(p + gr * ld + gk, ks - gk) : load8(p + gk * ld + gr, rows - gr);
    *reinterpret_cast<u32x4*>(lds + i * 16) = v;
  }
}

// Workgroups are dealt to the XCDs in turn: give each XCD a run of neighbouring tiles, and walk the tiles in
// groups of 8 tile rows, so that what an XCD works on at one time shares operand rows in its L2.
__device__ inline void tile_of(int id, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int total = tiles_m * tiles_n, per = total / kXcds, rest = total % kXcds;
  const int x = id % kXcds, i = id / kXcds;
  id = x * per + (x < rest ? x : rest) + i;
  const int group = 8 * tiles_n, g = id / group, first = g * 8;
  const int high = tiles_m - first < 8 ? tiles_m - first : 8;
  tm = first + (id - g * group) % high;
  tn = (id - g * group) / high;
}

// THREADS = 64 WM WN; each wavefront sums BM / WM by BN / WN.  The n side is the first operand of the matrix
// instruction, so that a lane ends with four neighbouring n of one m and the epilogue reads and writes 8 bytes.
template <class T, int BM, int BN, int WM, int WN, bool AKC, bool BKC, class Epi>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm(GemmArgs g, Epi epi) {
  typedef Tile<T, BM, AKC> TA;
  typedef Tile<T, BN, BKC> TB;
  constexpr int FM = BM / WM / 16, FN = BN / WN / 16, THREADS = 64 * WM * WN;
  __shared__ __attribute__((aligned(1024))) char lds[TA::kBytes + TB::kBytes];
  int tm, tn;
  tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
  if (Epi::kSymmetric && tm < tn) return;
  const int z = blockIdx.z;
  const T* a = static_cast<const T*>(g.a) + z * g.stride_a;
  const T* b = static_cast<const T*>(g.b) + z * g.stride_b;
  const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = {0, 0, 0, 0};
  for (int64_t k0 = 0; k0 < g.k; k0 += kBK) {
    stage<T, BM, AKC, THREADS>(lds, a, g.lda, m0, g.m, k0, g.k);
    stage<T, BN, BKC, THREADS>(lds + TA::kBytes, b, g.ldb, n0, g.n, k0, g.k);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      typename Vec<T>::x8 fa[FM], fb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = TA::frag(lds, wm + 16 * i, s, lane);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = TB::frag(lds + TA::kBytes, wn + 16 * j, s, lane);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mfma(fb[j], fa[i], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      epi(m0 + wm + 16 * i + (lane & 15), n0 + wn + 16 * j + 4 * (lane >> 4), acc[i][j], z, g.m, g.n);
}

template <class T, bool AKC, bool BKC, class Epi>
int gemm(GemmArgs g, const Epi& epi, int64_t count, hipStream_t st) {
  if (g.m <= 0 || g.n <= 0 || count <= 0) return XMEM_OK;
  g.tiles_m = int((g.m + 127) / 128);
  g.tiles_n = int((g.n + 127) / 128);
  k_gemm<T, 128, 128, 2, 2, AKC, BKC, Epi><<<dim3(unsigned(g.tiles_m) * g.tiles_n, 1, unsigned(count)), 256, 0, st>>>(g, epi);
  return launched();
}

// Four neighbouring elements of one row: one 8-byte access where the row has them and the address allows it.
template <class T>
__device__ inline f32x4 get4(const T* p, int64_t valid, bool wide) {
  f32x4 v = {0, 0, 0, 0};
  if (wide && valid >= 4) {
    const typename Vec<T>::x4 e = *reinterpret_cast<const typename Vec<T>::x4*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = float(e[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < valid) v[j] = float(p[j]);
  }
  return v;
}
template <class T>
__device__ inline void put4(T* p, f32x4 v, int64_t valid, bool wide) {
  if (wide && valid >= 4) {
    typename Vec<T>::x4 e;
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = T(v[j]);
    *reinterpret_cast<typename Vec<T>::x4*>(p) = e;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < valid) p[j] = T(v[j]);
  }
}

}  // namespace xops
