// gemm.h -- the matrix product of the training operators: out(m, n) = sum over k of A(m, k) B(n, k), with
// 16-bit operands, 32-bit sums on the matrix cores, and an epilogue that sees each sum once.
//
// Either operand may lie with k contiguous (A[m * ld + k]) or with its rows contiguous (A[k * ld + m]), so
// the three products of a linear layer (x w^T, dz w, dz^T x) and of a Newton-Schulz step need no transposed copy.
//
// What bounds it.  A tile of 256 x 256 reads 64 KiB an operand pair for 64 k, which its matrix instructions use for 2,048 cycles;
// its LDS reads take 1,536 of them without a bank conflict.  On values of 0 (no power limit) 8192 x 8192 x 8192 runs at 1,480
// TFLOP/s, and at 1,770 where every k tile's loads come from the same place: the loads that miss the L2 (21%) hold it back.
// On random values the clock falls: 1,270 to 1,440 TFLOP/s for x w^T, 1,050 to 1,200 for dz w, 1,120 to 1,290 for dz^T x, where the
// library's products reach 1,370 to 1,580, 1,210 to 1,370 and 1,070 to 1,210.  Small ones are bound by their latency: a launch
// (2.1 us), the first loads, one reduction and the writes take 6.5 us for one k tile, each further group of four 0.8.
#pragma once
#include "common.h"

namespace xops {

constexpr int kBK = 64;  // k of one tile: 128 bytes of an operand row

struct GemmArgs {
  const void* a;
  const void* b;
  int64_t lda, ldb;
  int64_t stride_a, stride_b;  // between the matrices of a batch, in elements
  int64_t m, n, k;
  // the operand's rows have room behind their ends up to a multiple of 8, and it holds zeros
  bool pad_a = false, pad_b = false;
  int64_t count = 1;
  // set by the launch
  int tiles_m = 0, tiles_n = 0, tiles = 0, splits = 1, span = 0;  // span: k tiles of a split
  int first = 0;  // workgroup of the launch
  float* part = nullptr;
};

// A workgroup's tile and its wavefronts: WM by WN of them, each with BM / WM by BN / WN of the tile, WK times over: each
// such group takes every WK-th k tile, and their sums are added in LDS.  Two k tiles of a group are in LDS, one of them
// on its way.  STAGED: whether there is a form whose loads go through registers.
// More k tiles on their way (four of the 128 tile, eight of the 64) in place of more groups: 1024 x 1024 x 1024 10.6 us against 9.4.
template <int BM_, int BN_, int WM_, int WN_, int WK_, bool STAGED_>
struct Config {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WK = WK_, FM = BM / WM / 16, FN = BN / WN / 16;
  static constexpr int GROUP = 64 * WM * WN, THREADS = GROUP * WK;
  static constexpr bool STAGED = STAGED_;
  static_assert(FN % 2 == 0);
};
typedef Config<256, 256, 2, 4, 1, false> Large;  // 128 KiB of LDS, two wavefronts on a SIMD: a CU to itself
typedef Config<128, 128, 2, 2, 2, true> Medium;  // 128 KiB, two wavefronts on a SIMD
typedef Config<64, 64, 2, 2, 4, true> Small;     // 128 KiB, four wavefronts on a SIMD
typedef Config<64, 64, 2, 2, 2, true> Half;      // 64 KiB, two workgroups a CU: where there are more tiles than CUs

// One operand tile in LDS: R rows of kBK.  Chunks of 16 bytes are kept at swizzled places, so that the 16 lanes
// that read one column of chunks meet 16 different bank groups.
//   k contiguous:    [row][8 chunks of k],   chunk c at c ^ ((row >> 1) & 7)
//   rows contiguous: [k][R / 8 chunks of rows], pairs of chunks (the 16 rows of one product) at p ^ h(k)
template <class T, int R, bool KC>
struct Tile {
  typedef typename Vec<T>::x8 x8;
  static constexpr int kBytes = R * kBK * 2;
  static constexpr int kChunks = R * kBK / 8;

  __host__ __device__ static int pair_hash(int k) { return ((k & 3) | ((k >> 1) & 4)) & (R / 16 - 1); }
  // the row (or first of eight rows) and the k (or first of eight) of the chunk kept at place i
  __host__ __device__ static void at(int i, int& row, int& k) {
    if constexpr (KC) {
      row = i >> 3;
      k = ((i & 7) ^ ((row >> 1) & 7)) * 8;
    } else {
      k = i / (R / 8);
      const int c = i % (R / 8);
      row = (((c >> 1) ^ pair_hash(k)) * 2 + (c & 1)) * 8;
    }
  }
  // the operand of a 16x16x32 product: places r0..r0+15 (r0 a multiple of 16), step s of the tile's k.
  // Lane l holds place l % 16, k = 32 s + 8 (l / 16) + 0..7.
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

// Row lengths for which a tile's bytes fit 31 bits.
constexpr int64_t kMostDirectLd = int64_t(1) << 21;

// A buffer load past num_records gives zeros, whose LDS place is written all the same.
constexpr unsigned kNowhere = 0x80000000u;

// One operand's loads straight from memory into LDS, 16 bytes a lane, for 16-byte aligned operands whose ld is a
// multiple of 8, and whose contiguous side is one or padded to one.  The swizzle is in which chunk a lane fetches.
template <class T, class Ti, int R, bool KC, int THREADS>
struct Direct {
  static constexpr int kLoads = Ti::kChunks / THREADS;
  unsigned off[kLoads];
  int kk;  // KC: the k of this lane's chunks within the tile

  __device__ void init(int tid, int64_t ld, int64_t r0, int64_t rows) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      int row, k;
      Ti::at(j * THREADS + tid, row, k);
      off[j] = KC ? unsigned(row) * unsigned(ld * 2) + k * 2 : unsigned(k) * unsigned(ld * 2) + row * 2;
      if (!KC && r0 + row >= rows) off[j] = kNowhere;
      if (KC) kk = k;  // the same for every j: a pass of THREADS chunks is a multiple of 16 rows
    }
  }
  // tile t of the operand; past the last one it only clears LDS.  ld < 2^21, so that a tile's bytes fit 31 bits.
  __device__ void issue(char* lds, const T* p, int64_t ld, int64_t r0, int64_t rows, int t, int ks, int wave) const {
    const int k0 = t * kBK, left = ks - k0, step = int(ld);
    const T* base = KC ? p + r0 * ld + k0 : p + k0 * ld + r0;
    const int high = KC ? (rows - r0 < R ? int(rows - r0) : R) : (left < kBK ? left : kBK);
    const int wide = ((KC ? left : int(rows - r0)) + 7) & ~7;
    int bytes = ((high - 1) * step + wide) * 2;
    bytes = left > 0 ? bytes : 0;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, bytes, 0x00020000);
    const bool out = KC && kk >= left;
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(lds + (j * THREADS + wave * 64) * 16),
                                               16, out ? kNowhere : off[j], 0, 0, 0);
  }
};

// v >> 16 s bits as one number of 128 bits, s = 0..8: the elements past the end of a row, dropped.
__host__ __device__ inline u32x4 drop(u32x4 v, int s) {
  if (s & 1) {
    v[0] = (v[0] >> 16) | (v[1] << 16);
    v[1] = (v[1] >> 16) | (v[2] << 16);
    v[2] = (v[2] >> 16) | (v[3] << 16);
    v[3] >>= 16;
  }
  if (s & 2) v = u32x4{v[1], v[2], v[3], 0};
  if (s & 4) v = u32x4{v[2], v[3], 0, 0};
  if (s & 8) v = u32x4{0, 0, 0, 0};
  return v;
}

// One operand's loads through registers, for rows of any alignment.  A chunk that passes the end of its row is read
// from further back, so that it ends there, and shifted when it is stored: every load is 16 bytes and inside the
// matrix, none waits for another or is behind a branch of its own.  But for the last k tile a chunk's place in the
// tile does not change, so a load costs no address arithmetic (which took longer than the loads).
template <class T, class Ti, int R, bool KC, int THREADS>
struct Staged {
  static constexpr int kLoads = Ti::kChunks / THREADS;
  u32x4 v[kLoads];
  unsigned off[kLoads];
  int past[kLoads];  // elements of a chunk that its row does not have
  bool plain;        // rows of 8 elements and more, near enough for 32-bit offsets
  bool cut;          // some chunk passes its row's end

  __host__ __device__ void init(int tid, int64_t ld, int64_t r0, int64_t rows, int ks) {
    plain = (KC ? ks : rows) >= 8 && ld < kMostDirectLd;
    cut = !KC && r0 + R > rows;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      int row, k;
      Ti::at(j * THREADS + tid, row, k);
      if (KC) {  // a row past the last one is read as the last: what comes of it is not written
        const int left = int(rows - r0 < R ? rows - r0 : R) - 1;
        past[j] = 0;
        off[j] = unsigned(row < left ? row : left) * unsigned(ld * 2) + k * 2;
      } else {
        const int64_t valid = rows - (r0 + row);
        past[j] = valid >= 8 ? 0 : valid <= 0 ? 8 : int(8 - valid);
        // a chunk wholly past the row's end reads the tile's first eight rows or, where there are fewer, the last eight of all
        off[j] = unsigned(k) * unsigned(ld * 2) + (past[j] < 8 ? row - past[j] : rows - r0 < 8 ? int(rows - r0) - 8 : 0) * 2;
      }
    }
  }
  __host__ __device__ void load(int tid, const T* p, int64_t ld, int64_t r0, int64_t rows, int t, int ks) {
    const int64_t k0 = int64_t(t) * kBK;
    if (plain && k0 + kBK <= ks) {
      const char* base = reinterpret_cast<const char*>(KC ? p + r0 * ld + k0 : p + k0 * ld + r0);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) __builtin_memcpy(&v[j], base + int(off[j]), 16);
      return;
    }
    cut = true;
    const int64_t length = KC ? ks : rows;  // of the contiguous side
    const T* from[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      int row, k;
      Ti::at(j * THREADS + tid, row, k);
      const int64_t along = KC ? k0 + k : r0 + row, across = KC ? r0 + row : k0 + k, last = (KC ? rows : int64_t(ks)) - 1;
      const int64_t valid = across <= last ? length - along : 0;
      past[j] = valid >= 8 ? 0 : valid <= 0 ? 8 : int(8 - valid);
      from[j] = p + (across <= last ? across : last) * ld + (past[j] == 8 ? 0 : along - past[j]);
    }
    if (length >= 8) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) __builtin_memcpy(&v[j], from[j], 16);
    } else {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {  // from[j] + past[j] is the chunk's first element; what is read ends its 8
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i >= past[j] ? from[j][i] : T(0.0f);
        __builtin_memcpy(&v[j], e, 16);
      }
    }
  }
  __host__ __device__ void store(int tid, char* lds) const {
    if (!cut) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) *reinterpret_cast<u32x4*>(lds + (j * THREADS + tid) * 16) = v[j];
    } else {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) *reinterpret_cast<u32x4*>(lds + (j * THREADS + tid) * 16) = drop(v[j], past[j]);
    }
  }
};

// Lays half a tile's work out for the compiler's scheduler: LOADS memory loads, then READS LDS reads (in that order,
// which is the program's), spread among PRODUCTS matrix instructions; nothing moves past the end.
template <int LOADS, int READS, int PRODUCTS>
struct Order {
  static constexpr int kEach = PRODUCTS * 7 / 8 / (LOADS + READS) > 0 ? PRODUCTS * 7 / 8 / (LOADS + READS) : 1;
  template <int I>
  __device__ static __attribute__((always_inline)) void slot() {
    if constexpr (I < LOADS + READS) {
      __builtin_amdgcn_sched_group_barrier(I < LOADS ? 0x20 : 0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, kEach, 0);
      slot<I + 1>();
    }
  }
  __device__ static __attribute__((always_inline)) void apply() {
    slot<0>();
    __builtin_amdgcn_sched_group_barrier(0x8, PRODUCTS, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
};

// Workgroups are dealt to the XCDs in turn: give each XCD a run of neighbouring tiles.
__device__ inline int run_of(int id, int total) {
  const int per = total / kXcds, rest = total % kXcds, x = id % kXcds;
  return x * per + (x < rest ? x : rest) + id / kXcds;
}

// Tile number -> tile: in groups of 8 tile rows, column by column, so that what an XCD works on at one time shares operand
// rows in its L2.  Of a symmetric product only the tiles on and below the diagonal: a group's columns left of its
// rows' diagonal block, then that block row by row.
template <bool SYMMETRIC>
__device__ inline void tile_of(int id, const GemmArgs& g, int& tm, int& tn) {
  if constexpr (SYMMETRIC) {
    int q = int((__builtin_sqrtf(8.0f * id + 1.0f) - 1.0f) * 0.0625f);  // the groups before q hold 32 q q + 4 q tiles
    while (32 * (q + 1) * (q + 1) + 4 * (q + 1) <= id) ++q;
    while (32 * q * q + 4 * q > id) --q;
    id -= 32 * q * q + 4 * q;
    const int first = 8 * q, high = g.tiles_m - first < 8 ? g.tiles_m - first : 8;
    if (id < high * first) {
      tm = first + id % high;
      tn = id / high;
    } else {
      id -= high * first;
      int r = 0;
      while ((r + 1) * (r + 2) / 2 <= id) ++r;
      tm = first + r;
      tn = first + id - r * (r + 1) / 2;
    }
  } else {
    const int group = 8 * g.tiles_n, first = id / group * 8, high = g.tiles_m - first < 8 ? g.tiles_m - first : 8;
    tm = first + id % group % high;
    tn = id % group / high;
  }
}

// The mirrored block of a symmetric product's tile: the epilogue's values as they were written, kept in LDS row by row in
// the layout of an operand with its rows contiguous, whose transposing reads give a lane eight neighbours of a column.
// 5 of 4096 x 4096 x 4096: 345 us; written entry by entry from the lanes' accumulators 372.
template <class C>
struct Mirror {
  typedef Tile<f16, C::BN, false> Ti;
  static constexpr int kBytes = C::BM * C::BN * 2;

  __device__ static void keep(char* lds, int m, int n, const float (&v)[8]) {
    typename Vec<f16>::x8 e;
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = f16(v[j]);
    const int c = n >> 3;
    *reinterpret_cast<typename Vec<f16>::x8*>(lds + m * (C::BN * 2) + ((((c >> 1) ^ Ti::pair_hash(m)) * 2 + (c & 1)) << 4)) = e;
  }
  // THREADS threads write what all of them kept: to[n][m]
  template <int THREADS>
  __device__ static void write(const char* lds, f16* to, int64_t ld, int64_t m0, int64_t n0, const GemmArgs& g) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int kPieces = (C::BN / 16) * (C::BM / 32);
    for (int i = wave; i < kPieces; i += THREADS / 64) {
      const int r0 = i / (C::BM / 32) * 16, s = i % (C::BM / 32);
      const auto e = Ti::frag(lds, r0, s, lane);
      const int64_t n = n0 + r0 + (lane & 15), m = m0 + 32 * s + 8 * (lane >> 4);
      if (n >= g.n || m >= g.m) continue;
      if (g.m - m >= 8) {
        __builtin_memcpy(to + n * ld + m, &e, 16);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (m + j < g.m) to[n * ld + m + j] = e[j];
      }
    }
  }
};

// HOW says what is known of the tile before it runs: whole (nothing of it is past the matrix) and past the L2s.
template <bool WHOLE_, bool PAST_L2_>
struct How {
  static constexpr bool WHOLE = WHOLE_, PAST_L2 = PAST_L2_;
};
// What a lane has of a tile: FN products' four neighbours each, of FM rows.  Two products' fours, exchanged between the
// lanes 16 apart, are eight neighbours of one or the other: the epilogue takes these, 16 bytes at a time and 64 next to
// each other, from row i0 on every STEP-th; what it reads of memory is asked for four rows at a time, before anything
// of them is written.  The Q-th eight of a lane; recursive, so that acc is indexed by constants however long the epilogue is.
template <class C, int STEP, int Q, class HOW, class Epi>
__device__ __attribute__((always_inline)) inline void finish(const f32x4 (&acc)[C::FM][C::FN], int i0, const Epi& epi, int64_t m0,
                                                             int64_t n0, int z, const GemmArgs& g, char* lds) {
  constexpr int W = 8, GROUPS = C::FN / 2, ROWS = (C::FM + STEP - 1) / STEP, BATCH = ROWS < 4 ? ROWS : 4;
  static_assert(ROWS % BATCH == 0);
  const int lane = threadIdx.x & 63, wave = (threadIdx.x % C::GROUP) >> 6;
  const int64_t mw = m0 + (wave / C::WN) * (C::BM / C::WM) + (lane & 15);
  const int64_t n = n0 + (wave % C::WN) * (C::BN / C::WN) + 32 * Q + 16 * ((lane >> 4) & 1) + 8 * (lane >> 5);
  const int valid = HOW::WHOLE || g.n - n >= W ? W : g.n > n ? int(g.n - n) : 0;
  const auto col = epi.template column<W>(n, valid, z, g);
#pragma unroll
  for (int h = 0; h < ROWS / BATCH; ++h) {
    typename Epi::template Read<W> in[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int64_t m = mw + 16 * (i0 + (h * BATCH + i) * STEP);
      if (HOW::WHOLE || (m < g.m && valid > 0)) in[i] = epi.template read<W>(m, n, valid, z, g);
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int64_t m = mw + 16 * (i0 + (h * BATCH + i) * STEP);
      float v[W];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float lo = acc[h * BATCH + i][2 * Q][j], hi = acc[h * BATCH + i][2 * Q + 1][j];
        if constexpr (STEP > 1)
#pragma unroll
          for (int k = 0; k < C::FM; ++k)
            if (k == i0 + (h * BATCH + i) * STEP) lo = acc[k][2 * Q][j], hi = acc[k][2 * Q + 1][j];
        const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(lo), __float_as_uint(hi), false, false);
        v[j] = __uint_as_float(two[0]);
        v[4 + j] = __uint_as_float(two[1]);
      }
      if (HOW::WHOLE || (m < g.m && valid > 0)) {
        epi.template row<W, HOW>(m, n, v, valid, col, in[i], z, g);
        if constexpr (Epi::kSymmetric) Mirror<C>::keep(lds, int(m - m0), int(n - n0), v);
      }
    }
  }
  if constexpr (Q + 1 < GROUPS) finish<C, STEP, Q + 1, HOW>(acc, i0, epi, m0, n0, z, g, lds);
}
// An epilogue's choices are made once a tile, so that the code a tile runs through is short: it passes the
// instruction cache once for each.
template <class C, int STEP, bool PAST_L2, class Epi>
__device__ __attribute__((always_inline)) inline void finish(const f32x4 (&acc)[C::FM][C::FN], int i0, const Epi& epi, int64_t m0,
                                                             int64_t n0, int z, const GemmArgs& g, char* lds) {
  if (m0 + C::BM <= g.m && n0 + C::BN <= g.n)
    epi.chosen([&](const auto& e) __attribute__((always_inline)) { finish<C, STEP, 0, How<true, PAST_L2>>(acc, i0, e, m0, n0, z, g, lds); });
  else
    finish<C, STEP, 0, How<false, false>>(acc, i0, epi, m0, n0, z, g, lds);
}

// One workgroup's tile.  Half a tile's operands are in registers ahead of the matrix instructions: while the products of
// one half run, the other half's LDS reads are under way.  One barrier a k tile: after it the tile just read is
// overwritten by the loads of the tile after next (direct), or the next tile, stored from registers while the
// first half ran, is complete (staged).
// The n side is the first operand of the matrix instruction, so that a lane ends with neighbouring n of one m.
template <class T, class C, bool AKC, bool BKC, bool DIRECT, bool PAST_L2, class Epi>
__global__ __launch_bounds__(C::THREADS) void k_gemm(GemmArgs g, Epi epi) {
#ifdef __HIP_DEVICE_COMPILE__  // the host's pass knows no buffer resources, and wants the kernel's name only
  constexpr int FM = C::FM, FN = C::FN;
  typedef Tile<T, C::BM, AKC> TA;
  typedef Tile<T, C::BN, BKC> TB;
  constexpr int BUF = TA::kBytes + TB::kBytes, kReads = FM * (AKC ? 1 : 2) + FN * (BKC ? 1 : 2);
  typedef typename Vec<T>::x8 x8;
  constexpr int LOADS = (TA::kChunks + TB::kChunks) / C::GROUP;
  constexpr int SUMS = C::WK > 1 ? FM * FN * 16 * C::THREADS : 0, BYTES = C::WK * 2 * BUF;
  static_assert(!Epi::kSymmetric || Mirror<C>::kBytes <= BYTES);
  __shared__ __attribute__((aligned(1024))) char all_lds[BYTES > SUMS ? BYTES : SUMS];
  int id = g.first + run_of(blockIdx.x, gridDim.x), tm, tn;
  const int z = id / (g.tiles * g.splits);
  id -= z * g.tiles * g.splits;
  const int split = id / g.tiles, tile = id % g.tiles;
  tile_of<Epi::kSymmetric>(tile, g, tm, tn);
  const T* a = static_cast<const T*>(g.a) + z * g.stride_a;
  const T* b = static_cast<const T*>(g.b) + z * g.stride_b;
  const int64_t m0 = int64_t(tm) * C::BM, n0 = int64_t(tn) * C::BN;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / C::GROUP), tid = threadIdx.x % C::GROUP;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* const lds = all_lds + group * (2 * BUF);
  const int wm = (wave / C::WN) * (C::BM / C::WM), wn = (wave % C::WN) * (C::BN / C::WN);
  const int t0 = split * g.span, ks = int(g.k) < (t0 + g.span) * kBK ? int(g.k) : (t0 + g.span) * kBK;
  // a group's tiles are t0 + group, + WK, ..., numbered 0 to passes; past the last k tile the operands are 0
  const int passes = ((ks + kBK - 1) / kBK - t0 + C::WK - 1) / C::WK;
  const auto tile_at = [&](int t) { return t0 + t * C::WK + group; };
  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = {0, 0, 0, 0};
  x8 a0[FM], b0[FN], a1[FM], b1[FN];
  const auto read = [&](x8(&fa)[FM], x8(&fb)[FN], int t, int s) {
    const char* from = lds + (t & 1) * BUF;
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[j] = TB::frag(from + TA::kBytes, wn + 16 * j, s, lane);
#pragma unroll
    for (int i = 0; i < FM; ++i) fa[i] = TA::frag(from, wm + 16 * i, s, lane);
  };
  const auto multiply = [&](const x8(&fa)[FM], const x8(&fb)[FN]) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mfma(fb[j], fa[i], acc[i][j]);
  };
  if constexpr (DIRECT) {
    Direct<T, TA, C::BM, AKC, C::GROUP> la;
    Direct<T, TB, C::BN, BKC, C::GROUP> lb;
    la.init(tid, g.lda, m0, g.m);
    lb.init(tid, g.ldb, n0, g.n);
    const auto fetch = [&](int t) {
      char* to = lds + (t & 1) * BUF;
      la.issue(to, a, g.lda, m0, g.m, tile_at(t), ks, wave);
      lb.issue(to + TA::kBytes, b, g.ldb, n0, g.n, tile_at(t), ks, wave);
    };
    if (passes > 0) {
      fetch(0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      fetch(1);
      read(a0, b0, 0, 0);
      for (int t = 0; t < passes; ++t) {
        read(a1, b1, t, 1);
        multiply(a0, b0);
        Order<0, kReads, FM * FN>::apply();
        // every read of this tile is done, and the next tile has come
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        fetch(t + 2);
        read(a0, b0, t + 1, 0);
        multiply(a1, b1);
        Order<LOADS, kReads, FM * FN>::apply();
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
  } else {
    Staged<T, TA, C::BM, AKC, C::GROUP> la;
    Staged<T, TB, C::BN, BKC, C::GROUP> lb;
    la.init(tid, g.lda, m0, g.m, ks);
    lb.init(tid, g.ldb, n0, g.n, ks);
    const auto load = [&](int t) {
      la.load(tid, a, g.lda, m0, g.m, tile_at(t), ks);
      lb.load(tid, b, g.ldb, n0, g.n, tile_at(t), ks);
    };
    const auto store = [&](int t) {
      char* to = lds + (t & 1) * BUF;
      la.store(tid, to);
      lb.store(tid, to + TA::kBytes);
    };
    if (passes > 0) {
      load(0);
      store(0);
      if (passes > 1) load(1);
      __syncthreads();
      read(a0, b0, 0, 0);
      for (int t = 0; t < passes; ++t) {
        read(a1, b1, t, 1);
        multiply(a0, b0);
        if (t + 1 < passes) store(t + 1);
        if (t + 2 < passes) load(t + 2);
        __syncthreads();
        if (t + 1 < passes) read(a0, b0, t + 1, 0);
        multiply(a1, b1);
      }
    }
  }
  if constexpr (C::WK > 1) {  // the groups' sums, in their order: every group gets the rows that it finishes
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(all_lds);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) sums[((i * FN + j) * C::WK + group) * C::GROUP + tid] = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FM; ++i)
      if (i % C::WK == group)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          acc[i][j] = sums[(i * FN + j) * C::WK * C::GROUP + tid];
#pragma unroll
          for (int k = 1; k < C::WK; ++k) acc[i][j] += sums[((i * FN + j) * C::WK + k) * C::GROUP + tid];
        }
  }
  if (g.splits > 1) {
    f32x4* to = reinterpret_cast<f32x4*>(g.part) + ((int64_t(z) * g.tiles + tile) * g.splits + split) * (FM * FN * C::GROUP) + tid;
#pragma unroll
    for (int i = 0; i < FM; ++i)
      if (i % C::WK == group)
#pragma unroll
        for (int j = 0; j < FN; ++j) to[(i * FN + j) * C::GROUP] = acc[i][j];
    return;
  }
  if constexpr (Epi::kSymmetric) __syncthreads();  // the last loads have landed everywhere, the sums have been read: LDS is free
  if (group < FM) finish<C, C::WK, PAST_L2>(acc, group, epi, m0, n0, z, g, all_lds);
  if constexpr (Epi::kSymmetric)
    if (tm != tn) {
      __syncthreads();
      Mirror<C>::template write<C::THREADS>(all_lds, epi.mirrored(z, g), epi.ld, m0, n0, g);
    }
#endif
}

// The splits of a product, added in their order, and its epilogue: a workgroup a tile, its lanes as one group of k_gemm.
template <class C, class Epi>
__global__ __launch_bounds__(C::GROUP) void k_join(GemmArgs g, Epi epi) {
  int tm, tn;
  const int z = blockIdx.x / g.tiles, tile = blockIdx.x % g.tiles;
  tile_of<Epi::kSymmetric>(tile, g, tm, tn);
  const f32x4* from =
      reinterpret_cast<const f32x4*>(g.part) + (int64_t(z) * g.tiles + tile) * g.splits * (C::FM * C::FN * C::GROUP) + threadIdx.x;
  f32x4 acc[C::FM][C::FN];
#pragma unroll
  for (int i = 0; i < C::FM; ++i)
#pragma unroll
    for (int j = 0; j < C::FN; ++j) acc[i][j] = from[(i * C::FN + j) * C::GROUP];
#pragma unroll 4
  for (int s = 1; s < g.splits; ++s) {
    from += C::FM * C::FN * C::GROUP;
#pragma unroll
    for (int i = 0; i < C::FM; ++i)
#pragma unroll
      for (int j = 0; j < C::FN; ++j) acc[i][j] += from[(i * C::FN + j) * C::GROUP];
  }
  const int64_t m0 = int64_t(tm) * C::BM, n0 = int64_t(tn) * C::BN;
  __shared__ __attribute__((aligned(1024))) char lds[Epi::kSymmetric ? Mirror<C>::kBytes : 16];
  finish<C, 1, false>(acc, 0, epi, m0, n0, z, g, lds);
  if constexpr (Epi::kSymmetric)
    if (tm != tn) {
      __syncthreads();
      Mirror<C>::template write<C::GROUP>(lds, epi.mirrored(z, g), epi.ld, m0, n0, g);
    }
}

inline int64_t tiles_of(int64_t m, int64_t n, int bm, int bn, bool symmetric) {
  const int64_t tm = (m + bm - 1) / bm, tn = (n + bn - 1) / bn;
  return symmetric ? tm * (tm + 1) / 2 : tm * tn;
}

// Which tile a product takes, and over how many workgroups a tile's k is split: what costs least by what was measured.
// A round of workgroups over the CUs takes a time of its own and one per k tile:
//   256: 10 + 1.45 us (4096 x 4096 x 64, 4096: 11.7, 110 us);  128: 7.5 + 0.5 (2048 x 2048 x 64, 8192: 9.0, 70.4);
//   64: 6.5 + 0.24 up to one tile a CU (1024 x 1024 x 64, 4096: 6.6, 21.6), 6.7 + 0.33 for two (1024 tiles: 13.9, 97.3 at 8192).
// 1536 x 1536 x 4096 takes 82, 38 and 51 us with the three, 1024 x 1024 x 4096 78, 36 and 22.  A split adds a launch, and its sums
// go through memory.
struct Plan {
  int side;  // 256, 128 or 64
  int splits, span;
};
inline Plan plan_of(int64_t m, int64_t n, int64_t k, int64_t count, bool symmetric, bool may_split) {
  const int64_t kt = (k + kBK - 1) / kBK;
  const auto rounds = [](int64_t w, int64_t at_once) { return double((w + at_once - 1) / at_once); };
  const double large = rounds(tiles_of(m, n, 256, 256, symmetric) * count, kCus) * (10.0 + 1.45 * kt);
  const double medium = rounds(tiles_of(m, n, 128, 128, symmetric) * count, kCus) * (7.5 + 0.5 * kt);
  const int64_t tiles = tiles_of(m, n, 64, 64, symmetric) * count;
  const auto small = [&](int64_t w, int64_t span) { return w <= kCus ? 6.5 + 0.24 * span : rounds(w, 2 * kCus) * (6.7 + 0.33 * span); };
  Plan p{64, 1, int(kt)};
  double least = small(tiles, kt);
  for (int64_t s = 2; may_split && s <= kt / 4 && tiles * s <= 2 * kCus; ++s) {
    const int64_t span = (kt + s - 1) / s;
    const double cost = small(tiles * s, span) + 4.5 + double(tiles * s) * 0.008;
    if (cost < least) least = cost, p = {64, int((kt + span - 1) / span), int(span)};
  }
  if (medium < least) least = medium, p = {128, 1, int(kt)};
  if (large < least) p = {256, 1, int(kt)};
  return p;
}
inline size_t part_bytes(int64_t m, int64_t n, int64_t k, int64_t count, bool symmetric) {
  const Plan p = plan_of(m, n, k, count, symmetric, true);
  return p.splits > 1 ? up256(size_t(tiles_of(m, n, p.side, p.side, symmetric)) * count * p.splits * p.side * p.side * 4) : 0;
}

// Rows of copies and of workspace matrices are whole lines of 128 bytes, with zeros behind what they hold: a k tile of a row is
// one line then, not two (5 updates of 3859 x 4242 with rows of whole 64 bytes 8.66 ms, with lines 8.08).
struct Pack {
  const void* from;
  int64_t ld, rows, cols;
  void* to;
};

__host__ __device__ inline int64_t packed_ld(int64_t cols) { return (cols + 63) / 64 * 64; }
template <class T>
__global__ __launch_bounds__(256) void k_pack(Pack p0, Pack p1) {
  const Pack p = blockIdx.y ? p1 : p0;
  const unsigned pieces = unsigned(packed_ld(p.cols) / 8);
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < p.rows * pieces; i += int64_t(gridDim.x) * 256) {
    const int64_t r = i / pieces, c = (i - r * pieces) * 8;
    const T* from = static_cast<const T*>(p.from) + r * p.ld + c;
    u32x4 v;
    if (p.cols - c >= 8) {
      __builtin_memcpy(&v, from, 16);
    } else {
      T e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = j < p.cols - c ? from[j] : T(0.0f);
      __builtin_memcpy(&v, e, 16);
    }
    *reinterpret_cast<u32x4*>(static_cast<T*>(p.to) + i * 8) = v;
  }
}
// One or two (from NULL: none) matrices in one launch.
template <class T>
inline void pack(const Pack& a, const Pack& b, hipStream_t st) {
  const Pack& first = a.from ? a : b;
  if (!first.from) return;
  const bool both = a.from && b.from;
  const auto work = [](const Pack& p) { return p.rows * (packed_ld(p.cols) / 8); };
  const int64_t most = both && work(b) > work(a) ? work(b) : work(first), blocks = (most + 255) / 256;
  if (blocks > 0) k_pack<T><<<dim3(unsigned(blocks < 8192 ? blocks : 8192), both ? 2 : 1), 256, 0, st>>>(first, b);
}

inline bool direct_ok(const void* p, int64_t ld, int64_t stride, int64_t contiguous, bool padded) {
  return aligned(p, 16) && ld % 8 == 0 && stride % 8 == 0 && ld < kMostDirectLd && (contiguous % 8 == 0 || padded);
}

template <class T, class C, bool AKC, bool BKC, bool DIRECT, bool PAST_L2, class Epi>
void launch_tiles(GemmArgs g, const Epi& epi, hipStream_t st) {
  const int64_t all = int64_t(g.tiles) * g.count * g.splits, most = kMostThreads / C::THREADS;
  for (int64_t first = 0; first < all; first += most) {
    g.first = int(first);
    k_gemm<T, C, AKC, BKC, DIRECT, PAST_L2, Epi><<<unsigned(all - first < most ? all - first : most), C::THREADS, 0, st>>>(g, epi);
  }
}

template <class T, class C, bool AKC, bool BKC, class Epi>
int launch(GemmArgs g, const Epi& epi, hipStream_t st) {
  g.tiles_m = int((g.m + C::BM - 1) / C::BM);
  g.tiles_n = int((g.n + C::BN - 1) / C::BN);
  g.tiles = int(tiles_of(g.m, g.n, C::BM, C::BN, Epi::kSymmetric));
  const bool direct = direct_ok(g.a, g.lda, g.stride_a, AKC ? g.k : g.m, g.pad_a) && direct_ok(g.b, g.ldb, g.stride_b, BKC ? g.k : g.n, g.pad_b);
  if constexpr (C::BM == 256 && Epi::kPastL2)
    if (direct && epi.lines()) {
      launch_tiles<T, C, AKC, BKC, true, true>(g, epi, st);
      return launched();
    }
  if (direct)
    launch_tiles<T, C, AKC, BKC, true, false>(g, epi, st);
  else if constexpr (!Epi::kAnyRows)
    return XMEM_EINVAL;  // operands of the library's own workspace, aligned by construction
  else if constexpr (C::STAGED)
    launch_tiles<T, C, AKC, BKC, false, false>(g, epi, st);
  else
    return launch<T, Medium, AKC, BKC>(g, epi, st);  // a tile's registers would not fit
  if constexpr (C::BM == 64)
    if (g.splits > 1) k_join<C, Epi><<<unsigned(g.tiles * g.count), C::GROUP, 0, st>>>(g, epi);
  return launched();
}

// part: part_bytes() of workspace, or NULL to leave k whole.
template <class T, bool AKC, bool BKC, class Epi>
int gemm(GemmArgs g, const Epi& epi, void* part, hipStream_t st) {
  if (g.m <= 0 || g.n <= 0 || g.count <= 0) return XMEM_OK;
  const Plan p = plan_of(g.m, g.n, g.k, g.count, Epi::kSymmetric, part != nullptr);
  g.splits = p.splits;
  g.span = p.span;
  g.part = static_cast<float*>(part);
  if (p.side == 256) return launch<T, Large, AKC, BKC>(g, epi, st);
  if (p.side == 128) return launch<T, Medium, AKC, BKC>(g, epi, st);
  if (tiles_of(g.m, g.n, 64, 64, Epi::kSymmetric) * g.count * p.splits > kCus) return launch<T, Half, AKC, BKC>(g, epi, st);
  return launch<T, Small, AKC, BKC>(g, epi, st);
}

// Whether the 64 bytes that an epilogue writes of a row are one piece of memory.
inline bool whole_lines(const void* p, int64_t ld) { return aligned(p, 64) && ld % 32 == 0; }

// W neighbouring elements of a row, `valid` of which exist; whole ones move in one access of any alignment.
template <class T, int W>
__device__ inline void get(const T* p, int valid, float (&v)[W]) {
  T e[W];
  if (valid == W) {
    __builtin_memcpy(e, p, sizeof(e));
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) e[j] = j < valid ? p[j] : T(0.0f);
  }
#pragma unroll
  for (int j = 0; j < W; ++j) v[j] = float(e[j]);
}
// HOW::PAST_L2: an output of the 256 x 256 tiles stays in no L2 for long; written past them, where its rows are whole
// pieces of 64 bytes, it leaves the operands there.  8192 x 8192 and its pre-activation 283 -> 244 us, 24 steps of 8192 x 2048 18.1 -> 17.2 ms; one of 1024 x 1024,
// which the next kernel reads, 162 -> 171 us.
template <class T, int W, class HOW>
__device__ inline void put(T* p, int valid, const float (&v)[W]) {
  T e[W];
#pragma unroll
  for (int j = 0; j < W; ++j) e[j] = T(v[j]);
  if (HOW::WHOLE || valid == W) {
    if constexpr (HOW::PAST_L2) {
      typedef unsigned any4 __attribute__((ext_vector_type(4), aligned(2)));
      static_assert(sizeof(e) == 16);
      any4 q;
      __builtin_memcpy(&q, e, 16);
      __builtin_nontemporal_store(q, reinterpret_cast<any4*>(p));
    } else {
      __builtin_memcpy(p, e, sizeof(e));
    }
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < valid) p[j] = e[j];
  }
}
typedef How<false, false> Any;

// What an epilogue keeps of its W columns, or reads of a row of them.
template <int W>
struct Column {
  float v[W];
};
struct None {};

}  // namespace xops
