// norm.hip -- the norms before and after a block with its gate, scale and residual sum, and their gradients, on MI355X (gfx950).
//
// Forward, with xhat = (x - mu) rho: out = r + alpha s a(g) (hhat w1 + b1), y = outhat w2 + b2.  A row is read once: its inputs stay in
// registers, each norm takes one sum of it (two with a mean: squares are taken of what is left without it, so nothing cancels), and
// its outputs are written once.  y comes from the 32-bit sum, so that it is rounded once; the stored out is what the backward pass sees.
//
// Backward: e = dy w2, dr = dout + rho2 (e - [layer] mean(e) - outhat mean(e outhat)); with b = dr a(g) and f = alpha s b w1: dh = rho1 (f -
// [layer] mean(f) - hhat mean(f hhat)), dgate = dr alpha s (hhat w1 + b1) a'(g).  The vectors' gradients are sums over rows of b hhat, b, dy outhat
// and dy, times what a column has in common: a workgroup goes over rows with its threads on the same columns, keeps their sums, and writes
// one part a workgroup; k_norm_sums adds the parts up in order.
//
// Bound by memory.  Forward, bfloat16, both norms, gate, scale: 32768 x 4096 256 to 274 us by the card (4.9 to 5.2 TB/s of 1.34 GB; a large
// copy reaches 4.9).  Backward of the same 426 and 9 (2.15 GB, 5.0 TB/s), 8192 x 2048 56 and 6.4 (268 MB, 4.8 TB/s; with means and biases 61
// and 9; in float32 106 and 6, 108 and 9).  The norm alone 14 forward and 25 + 4.4 back (8192 x 2048).  One row of 2048 takes 2.4 us, of which a
// launch is 2.1.
// Wide gradients are not: 4096 x 16384 289 and 8 (1.07 GB, 3.7 TB/s), with means and biases 484 and 13; 2048 x 16384 in float32, no gate, 258 and 8, 430
// and 13.  One workgroup a CU, whose second loads wait for its first sums, and 124 to 352 bytes a thread in scratch memory: at 1024 threads 240 bytes
// are nearly as much as the row's eight values in 16 bits.  Narrow ones are far from the memory's rate (32768 x 40 3.3): 8.2 and 4.1, with means
// and biases 13.4 and 4.2; the 16-bit forms below a wavefront keep up to 56 bytes of scratch.
#include "rows.h"

using namespace xops;

namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct Norms {
  const void *r, *h, *gate;
  int64_t ldr, ldh, ldg;
  const float *s, *w1, *b1, *w2, *b2;
  int64_t t, n;
  int post, pre, act;
  float eps, alpha;
  void *out, *y;
  int64_t ldo, ldy;
  float* stats;
  bool past_caches;   // outputs
  int64_t first = 0;  // row of the launch
};

__device__ inline float logistic(float g) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-g * kLog2e)); }

// What a gate's value multiplies with.
__device__ inline float gate_of(float g, int act) {
  return act == XMEM_GATE_NONE ? g : act == XMEM_GATE_SIGMOID ? logistic(g) : g * logistic(g);
}

// alpha s a(g) ((h - mu) rho w + b) of a piece; `vector` reads a vector's part of it.
template <class T>
struct Branch {
  static constexpr int E = kPiece<T>;
  const Norms& p;
  float mu, rho;
  template <class Vector>
  __device__ void of(u32x4 h, u32x4 g, const Vector& vector, float (&v)[E]) const {
    float w[E], b[E], s[E];
    unpack<T>(h, v);
    if (p.post != XMEM_NORM_NONE) {
      vector(p.w1, 1.0f, w);
      vector(p.b1, 0.0f, b);
#pragma unroll
      for (int k = 0; k < E; ++k) v[k] = (v[k] - mu) * rho * w[k] + b[k];
    }
    vector(p.s, 1.0f, s);
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] *= p.alpha * s[k];
    if (p.gate) {
      float a[E];
      unpack<T>(g, a);
#pragma unroll
      for (int k = 0; k < E; ++k) v[k] *= gate_of(a[k], p.act);
    }
  }
};

// Mean and reciprocal deviation of a row: `each(f)` gives the sum of f(x) over the thread's elements of it.
template <class Sums, class Each>
__device__ inline void moments(Sums& sums, const Each& each, int kind, int64_t n, float eps, float& mu, float& rho) {
  mu = 0.0f;
  rho = 0.0f;
  if (kind == XMEM_NORM_NONE) return;
  if (kind == XMEM_NORM_LAYER) mu = sums.one(each([](float x) { return x; })) / float(n);
  rho = 1.0f / sqrtf(sums.one(each([&](float x) { return (x - mu) * (x - mu); })) / float(n) + eps);
}

// W threads of a row, with NCH pieces of it in each thread's registers; as many rows a workgroup as make 256 threads.  The last piece
// is moved down to the row's end (Place), so that no thread has a tail: 8192 x 2047 with tails 40 us, without 34.
template <class T, int W, int NCH>
__global__ __launch_bounds__(W < 256 ? 256 : W) void k_norm(Norms p) {
  constexpr int E = kPiece<T>, R = W < 256 ? 256 / W : 1;
  __shared__ typename RowSums<W, R>::Meet meet;
  const int slot = W < kWave ? threadIdx.x / W : __builtin_amdgcn_readfirstlane(threadIdx.x / W), tid = threadIdx.x % W;
  RowSums<W, R> sums(meet, slot);
  const int64_t t = p.first + int64_t(blockIdx.x) * R + slot, at = t < p.t ? t : p.t - 1;
  const bool here = t < p.t;  // a row that is not there is the last one again, and not written
  const int n = int(p.n), pieces = (n + E - 1) / E;
  const auto place = [&](int j) { return Place<E>(j * W + tid, n); };
  const auto row = [&](const void* x, int64_t ld, int j) { return piece_at(static_cast<const T*>(x) + at * ld, place(j).at); };
  const auto put = [&](void* x, int64_t ld, int j, const float (&v)[E]) {
    if (here && p.past_caches)
      put_piece_past(static_cast<T*>(x) + at * ld, place(j).at, v);
    else if (here)
      put_piece_at(static_cast<T*>(x) + at * ld, place(j).at, v);
  };
  // over the thread's elements of pieces that `piece` gives
  const auto total = [&](const auto& piece, const auto& f) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        float v[E];
        piece(j, v);
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = f(v[k]);
        place(j).counted(v);
#pragma unroll
        for (int k = 0; k < E; ++k) s += v[k];
      }
    return s;
  };
  float x[NCH][E], mu1 = 0.0f, rho1 = 0.0f, mu2, rho2;
  u32x4 cr[NCH];
#pragma unroll
  for (int j = 0; j < NCH; ++j)
    if (j * W < pieces) cr[j] = row(p.r, p.ldr, j);
  if (p.h) {
    u32x4 ch[NCH], cg[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        ch[j] = row(p.h, p.ldh, j);
        if (p.gate) cg[j] = row(p.gate, p.ldg, j);
      }
    const auto piece = [&](int j, float (&v)[E]) { unpack<T>(ch[j], v); };
    moments(sums, [&](const auto& f) { return total(piece, f); }, p.post, n, p.eps, mu1, rho1);
    // elements that two wavefronts have are read by both before one writes them
    if (W > kWave && p.post == XMEM_NORM_NONE && p.out == p.r) __syncthreads();
    const Branch<T> branch{p, mu1, rho1};
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        float v[E];
        branch.of(ch[j], cg[j], [&](const float* w, float without, float (&to)[E]) { vector_at(w, place(j).at, without, to); }, v);
        unpack<T>(cr[j], x[j]);
#pragma unroll
        for (int k = 0; k < E; ++k) x[j][k] += v[k];
        put(p.out, p.ldo, j, x[j]);
      }
  } else {
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) unpack<T>(cr[j], x[j]);
  }
  const auto piece = [&](int j, float (&v)[E]) {
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = x[j][k];
  };
  moments(sums, [&](const auto& f) { return total(piece, f); }, p.pre, n, p.eps, mu2, rho2);
  if (p.y) {
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        float w[E], b[E];
        vector_at(p.w2, place(j).at, 1.0f, w);
        vector_at(p.b2, place(j).at, 0.0f, b);
#pragma unroll
        for (int k = 0; k < E; ++k) x[j][k] = (x[j][k] - mu2) * rho2 * w[k] + b[k];
        put(p.y, p.ldy, j, x[j]);
      }
  }
  if (p.stats && tid == 0 && here) {
    p.stats[t] = mu1;
    p.stats[p.t + t] = rho1;
    p.stats[2 * p.t + t] = mu2;
    p.stats[3 * p.t + t] = rho2;
  }
}

// A row that no registers hold, or of less than a piece: its inputs are read again for each sum, and outputs written last (out may be r).
// Short rows are right here, not fast, with a workgroup each: 32768 x 7 in bfloat16 431 us, where 32768 x 8 takes 5.0.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_any(Norms p) {
  constexpr int E = kPiece<T>, THREADS = 1024;
  __shared__ typename RowSums<THREADS>::Meet meet;
  RowSums<THREADS> sums(meet);
  const int64_t t = p.first + blockIdx.x, n = p.n, pieces = (n + E - 1) / E;
  const T* r = static_cast<const T*>(p.r) + t * p.ldr;
  const T* h = p.h ? static_cast<const T*>(p.h) + t * p.ldh : nullptr;
  const T* g = p.gate ? static_cast<const T*>(p.gate) + t * p.ldg : nullptr;
  float mu1, rho1, mu2, rho2;
  const auto total = [&](const auto& piece, const auto& f) {
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < pieces; i += THREADS) {
      float v[E];
      piece(i, v);
#pragma unroll
      for (int k = 0; k < E; ++k) s += i * E + k < n ? f(v[k]) : 0.0f;
    }
    return s;
  };
  const auto block = [&](int64_t i, float (&v)[E]) { unpack<T>(piece_of(h, i, n), v); };
  moments(sums, [&](const auto& f) { return total(block, f); }, h ? p.post : XMEM_NORM_NONE, n, p.eps, mu1, rho1);
  const Branch<T> branch{p, mu1, rho1};
  const auto sum = [&](int64_t i, float (&x)[E]) {
    unpack<T>(piece_of(r, i, n), x);
    if (h) {
      float v[E];
      branch.of(piece_of(h, i, n), g ? piece_of(g, i, n) : u32x4{},
                [&](const float* w, float without, float (&to)[E]) { vector_of<E>(w, i, n, without, to); }, v);
#pragma unroll
      for (int k = 0; k < E; ++k) x[k] += v[k];
    }
  };
  moments(sums, [&](const auto& f) { return total(sum, f); }, p.pre, n, p.eps, mu2, rho2);
  for (int64_t i = threadIdx.x; i < pieces; i += THREADS) {
    float x[E], w[E], b[E];
    sum(i, x);
    if (p.out) put_piece(static_cast<T*>(p.out) + t * p.ldo, i, n, x);
    if (!p.y) continue;
    vector_of<E>(p.w2, i, n, 1.0f, w);
    vector_of<E>(p.b2, i, n, 0.0f, b);
#pragma unroll
    for (int k = 0; k < E; ++k) x[k] = (x[k] - mu2) * rho2 * w[k] + b[k];
    put_piece(static_cast<T*>(p.y) + t * p.ldy, i, n, x);
  }
  if (p.stats && threadIdx.x == 0) {
    p.stats[t] = mu1;
    p.stats[p.t + t] = rho1;
    p.stats[2 * p.t + t] = mu2;
    p.stats[3 * p.t + t] = rho2;
  }
}

// rows of a workgroup, its threads
template <class Kernel>
int launch_rows(Kernel kernel, Norms p, int per, int block, hipStream_t st) {
  const int64_t most = kMostThreads / block * per;
  for (; p.first < p.t; p.first += most) {
    const int64_t rows = p.t - p.first < most ? p.t - p.first : most;
    kernel<<<unsigned((rows + per - 1) / per), block, 0, st>>>(p);
  }
  return launched();
}

template <class T, int W, int NCH>
int launch_norm(const Norms& p, hipStream_t st) {
  return launch_rows(k_norm<T, W, NCH>, p, W < 256 ? 256 / W : 1, W < 256 ? 256 : W, st);
}
// A piece a thread up to 256 pieces (512 where rows are few), two or four beyond.  Measured in us, bfloat16 without a gate: rows of 2048 in
// 256 threads 25.0 (8192 of them) and 6.1 (1003), in a wavefront of four pieces a lane 28.2 and 8.5; of 4096 with a gate in 256 threads 264 to 272
// (32768), in 512 265 to 288, and without one 5.6 and 4.5 (200); of 8192 in 512 threads 26.3 (2048) and 5.7 (100), in 256 29.5 and 8.1, in
// 1024 27.6 and 5.5; of 16,384 in 1024 threads 27.5 (1024) and 6.8 (60), in 512 30.8 and 8.1.  Rows below a wavefront share one: 32768 of
// 40 5.4, one a wavefront 26.
template <class T>
int launch_norm(const Norms& p, hipStream_t st) {
  const int64_t pieces = (p.n + kPiece<T> - 1) / kPiece<T>;
  if (p.n < kPiece<T>) return launch_rows(k_norm_any<T>, p, 1, 1024, st);
  if (pieces <= 8) return launch_norm<T, 8, 1>(p, st);
  if (pieces <= 16) return launch_norm<T, 16, 1>(p, st);
  if (pieces <= 32) return launch_norm<T, 32, 1>(p, st);
  if (pieces <= 64) return launch_norm<T, 64, 1>(p, st);
  if (pieces <= 128) return launch_norm<T, 128, 1>(p, st);
  if (pieces <= 256) return launch_norm<T, 256, 1>(p, st);
  if (pieces <= 512) return p.t < 2048 ? launch_norm<T, 512, 1>(p, st) : launch_norm<T, 256, 2>(p, st);
  if (pieces <= 1024) return launch_norm<T, 512, 2>(p, st);
  if (pieces <= 2048) return launch_norm<T, 1024, 2>(p, st);
  if (pieces <= 4096) return launch_norm<T, 1024, 4>(p, st);
  return launch_rows(k_norm_any<T>, p, 1, 1024, st);
}

// ------------------------------------------------------------------ gradients

// What a row adds to the vectors' gradients, summed over rows: A = dout a(g) xhat1, B = dout a(g), C = dy xhat2, D = dy.
struct NormGrads {
  const void *dy, *dout, *out, *h, *gate;
  int64_t lddy, lddo, ldo, ldh, ldg;
  const float *stats, *s, *w1, *b1, *w2;
  int64_t t, n;
  int post, pre, act;
  float alpha;
  void *dr, *dh, *dg;
  int64_t lddr, lddh, lddg;
  float *part;  // [4][groups][n], NULL: none of the vectors' gradients is wanted
  bool biases;  // B and D too, and b1 is looked at
};

// One piece of a row.  `first`: what the norm after the sum adds up; `grad`: dr; `second`: what the block's norm does.
template <class T>
struct Piece {
  static constexpr int E = kPiece<T>;
  const NormGrads& p;
  float mu1, rho1, mu2, rho2;

  // e = dy w2 and xhat2
  __device__ void first(u32x4 cdy, u32x4 cout, const float (&w2)[E], float (&e)[E], float (&hat)[E], float (&dy)[E]) const {
    unpack<T>(cdy, dy);
    unpack<T>(cout, hat);
#pragma unroll
    for (int k = 0; k < E; ++k) {
      e[k] = dy[k] * w2[k];
      hat[k] = (hat[k] - mu2) * rho2;
    }
  }
  // dr from dout, e, xhat2 and the means of e and e xhat2
  __device__ void grad(u32x4 cdout, const float (&e)[E], const float (&hat)[E], float mean_e, float mean_eh, float (&d)[E]) const {
    unpack<T>(cdout, d);
#pragma unroll
    for (int k = 0; k < E; ++k) d[k] += rho2 * (e[k] - mean_e - hat[k] * mean_eh);
  }
  // from d = dr and s = alpha scale: b = d a(g), xhat1, f = s b w1 and dgate
  __device__ void second(u32x4 ch, u32x4 cg, const float (&d)[E], const float (&s)[E], const float (&w1)[E], const float (&b1)[E],
                         float (&b)[E], float (&hat)[E], float (&f)[E], float (&dg)[E]) const {
    unpack<T>(ch, hat);
    if (p.post != XMEM_NORM_NONE)
#pragma unroll
      for (int k = 0; k < E; ++k) hat[k] = (hat[k] - mu1) * rho1;
#pragma unroll
    for (int k = 0; k < E; ++k) b[k] = d[k];
    if (p.gate) {
      float g[E];
      unpack<T>(cg, g);
#pragma unroll
      for (int k = 0; k < E; ++k) {
        float a = g[k], slope = 1.0f;
        if (p.act != XMEM_GATE_NONE) {
          const float q = logistic(g[k]);
          a = p.act == XMEM_GATE_SIGMOID ? q : g[k] * q;
          slope = p.act == XMEM_GATE_SIGMOID ? q * (1.0f - q) : q * (1.0f + g[k] * (1.0f - q));
        }
        dg[k] = d[k] * s[k] * (hat[k] * w1[k] + b1[k]) * slope;
        b[k] *= a;
      }
    }
#pragma unroll
    for (int k = 0; k < E; ++k) f[k] = s[k] * b[k] * w1[k];
  }
};

// The vectors of a column: alpha scale, w1, w2 and b1.
__device__ inline float column_of(const NormGrads& p, int q, int64_t c) {
  return q == 0 ? p.alpha * (p.s ? p.s[c] : 1.0f) : q == 1 ? (p.w1 ? p.w1[c] : 1.0f) : q == 2 ? (p.w2 ? p.w2[c] : 1.0f) : (p.b1 ? p.b1[c] : 0.0f);
}

// BLOCK / W rows at a time, W threads and NCH pieces a thread each, whose columns' sums over all of the workgroup's rows stay in
// registers, half of them in LDS where they are four vectors' (BIASES), and all where a thread has more than eight columns of two.  The
// vectors are in LDS too (a thread would spend 24 to 32 registers on them), those of rows past 1024 pieces in the L2s.  With more than
// a piece a thread, what the first norm does not need is loaded after its sums.  128 registers, so that a CU has 16 wavefronts:
// 131 made 8192 x 2048 74 us instead of 55.  What they do not hold goes to scratch memory: nothing from 64 to 512 threads a row and in
// float32 below, up to 56 bytes a thread below in 16 bits, 40 and 48 at 1024 in 16 bits with biases, 124 and (with biases) 240 with two
// pieces a thread in 16 bits, 160 and 352 with four in float32.  Two workgroups of 512 a CU wait less for each other's sums than one of 1024 (55, 63); of
// 256 threads they write more parts (62 and 8.5 for the sums).
template <class T, int W, int NCH, bool BIASES, int BLOCK>
__global__ __launch_bounds__(BLOCK, 4) void k_norm_back(NormGrads p) {
  constexpr int E = kPiece<T>, R = BLOCK / W, VECTORS = BIASES ? 4 : 3;
  constexpr bool VLDS = NCH == 1, LATE = NCH > 1, APART = BIASES ? W < 1024 || NCH > 1 : NCH * E > 8;
  constexpr int HELD = BIASES ? APART ? 2 : 4 : APART ? 0 : 2;
  // vectors in LDS: as many as leave room for two workgroups of 512 on a CU
  constexpr int VL = VLDS ? (W == 512 && APART && E == 8 ? 2 : VECTORS) : 0;
  constexpr int ROWS = BLOCK / kWave * (W < kWave ? W : kWave) * E, COLUMNS = VL * W * E;  // floats
  __shared__ typename RowSums<W, R>::Meet meet;
  __shared__ float apart[APART ? 2 : 1][APART ? NCH * E : 1][APART ? BLOCK : 1];
  __shared__ __attribute__((aligned(16))) float shared[R > 1 && ROWS > COLUMNS ? ROWS : COLUMNS > 4 ? COLUMNS : 4];  // vectors, then rows' sums
  const int slot = W < kWave ? threadIdx.x / W : __builtin_amdgcn_readfirstlane(threadIdx.x / W), tid = threadIdx.x % W;
  RowSums<W, R> sums(meet, slot);
  const int n = int(p.n), pieces = (n + E - 1) / E;
  const auto place = [&](int j) { return Place<E>(j * W + tid, n); };
  if constexpr (VLDS) {  // [vector][half of a piece][thread of the row][4]
    for (int i = threadIdx.x; i < COLUMNS; i += BLOCK) {
      const int q = i / (W * E), c = i % (W * E);
      shared[((q * (E / 4) + c % E / 4) * W + c / E) * 4 + c % 4] = column_of(p, q, Place<E>(c / E, n).at + c % E);
    }
    __syncthreads();
  }
  const auto vector = [&](int q, int j, float (&v)[E]) {
    if (q < VL) {
#pragma unroll
      for (int h = 0; h < E / 4; ++h) {
        const f32x4 part = *reinterpret_cast<const f32x4*>(shared + ((q * (E / 4) + h) * W + tid) * 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[4 * h + k] = part[k];
      }
    } else {
      vector_at(q == 0 ? p.s : q == 1 ? p.w1 : q == 2 ? p.w2 : BIASES ? p.b1 : nullptr, place(j).at, q == 3 ? 0.0f : 1.0f, v);
      if (q == 0)
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] *= p.alpha;
    }
  };
  float acc[HELD ? HELD : 1][NCH][E] = {};  // A, B, C, D or A, C
  if constexpr (APART)
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int k = 0; k < NCH * E; ++k) apart[q][k][threadIdx.x] = 0.0f;
  const auto add = [&](int q, int j, int k, float v) {  // q: 0 to 3 for A to D
    if constexpr (HELD == 4)
      acc[q][j][k] += v;
    else if constexpr (!APART)
      acc[q / 2][j][k] += v;
    else if (!BIASES || (q & 1))
      apart[q / 2][j * E + k][threadIdx.x] += v;
    else
      acc[q / 2][j][k] += v;
  };
  for (int64_t t0 = int64_t(blockIdx.x) * R; t0 < p.t; t0 += int64_t(gridDim.x) * R) {
    const int64_t t = t0 + slot, at = t < p.t ? t : 0;
    const bool here = t < p.t;  // a row that is not there is one of 0, and not written
    const auto row = [&](const void* x, int64_t ld, int j) {
      return here ? piece_at(static_cast<const T*>(x) + at * ld, place(j).at) : u32x4{};
    };
    const auto put = [&](void* x, int64_t ld, int j, const float (&v)[E]) {
      if (here) put_piece_at(static_cast<T*>(x) + at * ld, place(j).at, v);
    };
    u32x4 cdy[NCH], cdo[NCH], co[NCH], ch[NCH], cg[NCH];
    const auto rest = [&](int j) {
      if (p.h) ch[j] = row(p.h, p.ldh, j);
      if (p.gate) cg[j] = row(p.gate, p.ldg, j);
    };
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        if (p.dy) {
          cdy[j] = row(p.dy, p.lddy, j);
          co[j] = row(p.out, p.ldo, j);
        }
        cdo[j] = p.dout ? row(p.dout, p.lddo, j) : u32x4{};
        if (!LATE) rest(j);
      }
    // elements that two wavefronts have are read by both before one writes them
    if (W > kWave && !p.dy && p.dr == p.dout) __syncthreads();
    // Of a row that is not there they are 0 too: another row's mean times its rho may pass 32 bits, and 0 times that is NaN.
    const auto stat = [&](int i) { return R == 1 || here ? p.stats[i * p.t + at] : 0.0f; };
    const Piece<T> q{p, stat(0), stat(1), stat(2), stat(3)};
    float s1 = 0.0f, s2 = 0.0f;
    if (p.dy) {
      float e[E], hat[E], dy[E], w[E];
#pragma unroll
      for (int j = 0; j < NCH; ++j)
        if (j * W < pieces) {
          vector(2, j, w);
          q.first(cdy[j], co[j], w, e, hat, dy);
#pragma unroll
          for (int k = 0; k < E; ++k) {
            add(2, j, k, dy[k] * hat[k]);
            if (BIASES) add(3, j, k, dy[k]);
          }
          place(j).counted(e);
#pragma unroll
          for (int k = 0; k < E; ++k) {
            s1 += e[k] * hat[k];
            s2 += e[k];
          }
        }
      if (p.pre == XMEM_NORM_LAYER)
        sums.two(s1, s2);
      else
        s1 = sums.one(s1), s2 = 0.0f;
      s1 /= float(n);
      s2 /= float(n);
    }
    float f[NCH][E], s3 = 0.0f, s4 = 0.0f;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        float e[E], hat[E], d[E], w[E], b[E], dg[E], s[E], w1[E], b1[E];
        if (LATE) rest(j);
        if (p.dy) {
          vector(2, j, w);
          q.first(cdy[j], co[j], w, e, hat, d);
          q.grad(cdo[j], e, hat, s2, s1, d);
        } else {
          unpack<T>(cdo[j], d);
        }
        put(p.dr, p.lddr, j, d);
        if (!p.h) continue;
        vector(0, j, s);
        vector(1, j, w1);
        vector(3, j, b1);
        q.second(ch[j], cg[j], d, s, w1, b1, b, hat, f[j], dg);
        if (p.dg) put(p.dg, p.lddg, j, dg);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          add(0, j, k, b[k] * hat[k]);
          if (BIASES) add(1, j, k, b[k]);
          b[k] = f[j][k];
        }
        place(j).counted(b);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          s3 += b[k] * hat[k];
          s4 += b[k];
        }
      }
    if (!p.h) continue;
    if (p.post != XMEM_NORM_NONE) {
      if (p.post == XMEM_NORM_LAYER)
        sums.two(s3, s4);
      else
        s3 = sums.one(s3), s4 = 0.0f;
      s3 /= float(n);
      s4 /= float(n);
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        if (p.post != XMEM_NORM_NONE) {
          float hat[E];
          unpack<T>(ch[j], hat);
#pragma unroll
          for (int k = 0; k < E; ++k) f[j][k] = q.rho1 * (f[j][k] - s4 - (hat[k] - q.mu1) * q.rho1 * s3);
        }
        put(p.dh, p.lddh, j, f[j]);
      }
  }
  if (!p.part) return;
  // the rows' sums, then the workgroup's part of each
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (!BIASES && (q & 1)) continue;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      float v[E];
#pragma unroll
      for (int k = 0; k < E; ++k) {
        if constexpr (APART)
          v[k] = !BIASES || (q & 1) ? apart[q / 2][j * E + k][threadIdx.x] : acc[HELD ? q / 2 : 0][j][k];
        else
          v[k] = acc[HELD == 4 ? q : q / 2][j][k];
      }
      if constexpr (R > 1) {
        constexpr int V = W < kWave ? W : kWave, PARTS = BLOCK / (W < kWave ? kWave : W);  // lanes that meet, wavefronts of one column
#pragma unroll
        for (int d = W; d < kWave; d *= 2)
#pragma unroll
          for (int k = 0; k < E; ++k) v[k] += __shfl_xor(v[k], d);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        __syncthreads();
        if (lane < V)
#pragma unroll
          for (int k = 0; k < E; ++k) shared[(k * (BLOCK / kWave) + wave) * V + lane] = v[k];
        __syncthreads();
        if (threadIdx.x < W)
#pragma unroll
          for (int k = 0; k < E; ++k)
#pragma unroll
            for (int w = 1; w < PARTS; ++w) v[k] += shared[(k * (BLOCK / kWave) + w * RowSums<W, R>::kParts + wave) * V + lane];
      }
      if (threadIdx.x < W && j * W < pieces) __builtin_memcpy(p.part + (int64_t(q) * gridDim.x + blockIdx.x) * n + place(j).at, v, sizeof(v));
    }
  }
}

// Rows that no registers hold, or of less than a piece: each is read three times, and a workgroup's sums are kept where its parts go.
// 32768 x 7 in bfloat16 take 1,290 us, where 32768 x 8 take 8.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_back_any(NormGrads p) {
  constexpr int E = kPiece<T>, THREADS = 1024;
  __shared__ typename RowSums<THREADS>::Meet meet;
  RowSums<THREADS> sums(meet);
  const int64_t n = p.n, pieces = (n + E - 1) / E;
  for (int64_t t = blockIdx.x; t < p.t; t += gridDim.x) {
    const auto row = [&](const void* x, int64_t ld, int64_t i) {
      return x ? piece_of(static_cast<const T*>(x) + t * ld, i, n) : u32x4{};
    };
    const auto vector = [&](int q, int64_t i, float (&v)[E]) {
      vector_of<E>(q == 0 ? p.s : q == 1 ? p.w1 : q == 2 ? p.w2 : p.b1, i, n, q == 3 ? 0.0f : 1.0f, v);
      if (q == 0)
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] *= p.alpha;
    };
    // behind the row's end xhat is what is left of 0, which may pass 32 bits: 0 times that is no 0
    const auto product = [&](int64_t i, int k, const float (&v)[E], const float (&xhat)[E]) { return i * E + k < n ? v[k] * xhat[k] : 0.0f; };
    const Piece<T> q{p, p.stats[t], p.stats[p.t + t], p.stats[2 * p.t + t], p.stats[3 * p.t + t]};
    float s1 = 0.0f, s2 = 0.0f, s3 = 0.0f, s4 = 0.0f, e[E], hat[E], dy[E], d[E], b[E], f[E], dg[E], s[E], w[E], add[E];
    if (p.dy) {
      for (int64_t i = threadIdx.x; i < pieces; i += THREADS) {
        vector(2, i, w);
        q.first(row(p.dy, p.lddy, i), row(p.out, p.ldo, i), w, e, hat, dy);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          s1 += product(i, k, e, hat);
          s2 += e[k];
        }
      }
      sums.two(s1, s2);
      s1 /= float(n);
      s2 = p.pre == XMEM_NORM_LAYER ? s2 / float(n) : 0.0f;
    }
    const auto grad = [&](int64_t i) {
      if (p.dy) {
        vector(2, i, w);
        q.first(row(p.dy, p.lddy, i), row(p.out, p.ldo, i), w, e, hat, dy);
        q.grad(row(p.dout, p.lddo, i), e, hat, s2, s1, d);
      } else {
        unpack<T>(row(p.dout, p.lddo, i), d);
      }
    };
    const auto second = [&](int64_t i) {
      vector(0, i, s);
      vector(1, i, w);
      vector(3, i, add);
      q.second(row(p.h, p.ldh, i), row(p.gate, p.ldg, i), d, s, w, add, b, hat, f, dg);
    };
    if (p.post != XMEM_NORM_NONE) {
      for (int64_t i = threadIdx.x; i < pieces; i += THREADS) {
        grad(i);
        second(i);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          if (i * E + k >= n) f[k] = 0.0f;
          s3 += product(i, k, f, hat);
          s4 += f[k];
        }
      }
      sums.two(s3, s4);
      s3 /= float(n);
      s4 = p.post == XMEM_NORM_LAYER ? s4 / float(n) : 0.0f;
    }
    for (int64_t i = threadIdx.x; i < pieces; i += THREADS) {
      const auto into = [&](int which, const float (&v)[E]) {
        if (!p.part) return;
        float* to = p.part + (int64_t(which) * gridDim.x + blockIdx.x) * n;
        float sum[E];
        vector_of<E>(t == blockIdx.x ? nullptr : to, i, n, 0.0f, sum);
#pragma unroll
        for (int k = 0; k < E; ++k) sum[k] += v[k];
        put_vector(to, i, n, sum);
      };
      grad(i);
      if (p.dy) {
        if (p.biases) into(3, dy);
#pragma unroll
        for (int k = 0; k < E; ++k) dy[k] *= hat[k];
        into(2, dy);
      }
      if (p.h) {
        second(i);
        if (p.dg) put_piece(static_cast<T*>(p.dg) + t * p.lddg, i, n, dg);
        if (p.biases) into(1, b);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          b[k] *= hat[k];
          if (p.post != XMEM_NORM_NONE) f[k] = q.rho1 * (f[k] - s4 - hat[k] * s3);
        }
        into(0, b);
        put_piece(static_cast<T*>(p.dh) + t * p.lddh, i, n, f);
      }
      put_piece(static_cast<T*>(p.dr) + t * p.lddr, i, n, d);
    }
  }
}

struct VectorGrads {
  const float *part, *s, *w1, *b1;
  int64_t groups, n;
  float alpha;
  float *ds, *dw1, *db1, *dw2, *db2;
};

// The groups' parts added up in a fixed order: COLS columns a workgroup, whose 1024 / COLS shares take every so many-th group each.
template <int COLS>
__global__ __launch_bounds__(1024) void k_norm_sums(VectorGrads p) {
  constexpr int SHARES = 1024 / COLS, U = 4;
  __shared__ float sums[4][16][COLS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = threadIdx.x % COLS;
  const bool wanted[4] = {p.ds || p.dw1, p.db1 || (p.ds && p.b1), p.dw2 != nullptr, p.db2 != nullptr};
  for (int64_t c0 = int64_t(blockIdx.x) * COLS; c0 < p.n; c0 += int64_t(gridDim.x) * COLS) {
    const int64_t c = c0 + col < p.n ? c0 + col : p.n - 1;
    float v[4] = {};
    for (int64_t g0 = threadIdx.x / COLS; g0 < p.groups; g0 += U * SHARES) {
      float x[4][U];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int u = 0; u < U; ++u)
          x[q][u] = wanted[q] && g0 + SHARES * u < p.groups ? p.part[(q * p.groups + g0 + SHARES * u) * p.n + c] : 0.0f;
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int u = 0; u < U; ++u) v[q] += x[q][u];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int d = COLS; d < kWave; d *= 2) v[q] += __shfl_xor(v[q], d);
      if (lane < COLS) sums[q][wave][lane] = v[q];
    }
    __syncthreads();
    if (threadIdx.x < COLS && c0 + col < p.n) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int w = 1; w < 16; ++w) v[q] += sums[q][w][col];
      const float s = p.alpha * (p.s ? p.s[c] : 1.0f);
      if (p.ds) p.ds[c] = p.alpha * ((p.w1 ? p.w1[c] : 1.0f) * v[0] + (p.b1 ? p.b1[c] * v[1] : 0.0f));
      if (p.dw1) p.dw1[c] = s * v[0];
      if (p.db1) p.db1[c] = s * v[1];
      if (p.dw2) p.dw2[c] = v[2];
      if (p.db2) p.db2[c] = v[3];
    }
    __syncthreads();
  }
}

// How rows are taken: threads of a row and pieces a thread (0: read again), and how many groups of sums there are.
template <int W> constexpr int kBackBlock = W <= 512 ? 512 : 1024;
struct Plan {
  int threads, nch;
  int64_t groups;
};
Plan plan_of(int64_t t, int64_t n, int dtype) {
  const int e = dtype == XMEM_F32 ? 4 : 8;
  const int64_t pieces = (n + e - 1) / e;
  Plan q{8, 1, 0};
  while (q.threads < 1024 && q.threads < pieces) q.threads *= 2;
  if (n < e)
    q.threads = 1024, q.nch = 0;
  else if (pieces > 1024)
    q.nch = pieces <= 2 * 1024 ? 2 : e == 4 && pieces <= 4 * 1024 ? 4 : 0;
  const int block = q.threads <= 512 ? 512 : 1024, per = block / q.threads;
  const int64_t rows = (t + per - 1) / per;
  int64_t most = kCus * 1024 / block;
  if (q.nch == 0) {  // parts of 256 MiB at most, or one group's
    const int64_t fit = (int64_t(1) << 24) / n;
    most = fit < 1 ? 1 : fit < most ? fit : most;
  }
  q.groups = rows < 2 * most ? (rows + 1) / 2 : most;  // two rounds at least: a part a round would be as much to write as the rows
  return q;
}

template <class T, int W, int NCH>
void launch_back(const NormGrads& p, const Plan& q, hipStream_t st) {
  if (p.biases)
    k_norm_back<T, W, NCH, true, kBackBlock<W>><<<unsigned(q.groups), kBackBlock<W>, 0, st>>>(p);
  else
    k_norm_back<T, W, NCH, false, kBackBlock<W>><<<unsigned(q.groups), kBackBlock<W>, 0, st>>>(p);
}
template <class T>
int launch_backward(const NormGrads& p, const Plan& q, hipStream_t st) {
  if (q.nch == 0)
    k_norm_back_any<T><<<unsigned(q.groups), 1024, 0, st>>>(p);
  else if (q.threads == 8)
    launch_back<T, 8, 1>(p, q, st);
  else if (q.threads == 16)
    launch_back<T, 16, 1>(p, q, st);
  else if (q.threads == 32)
    launch_back<T, 32, 1>(p, q, st);
  else if (q.threads == 64)
    launch_back<T, 64, 1>(p, q, st);
  else if (q.threads == 128)
    launch_back<T, 128, 1>(p, q, st);
  else if (q.threads == 256)
    launch_back<T, 256, 1>(p, q, st);
  else if (q.threads == 512)
    launch_back<T, 512, 1>(p, q, st);
  else if (q.nch == 1)
    launch_back<T, 1024, 1>(p, q, st);
  else if (q.nch == 2)
    launch_back<T, 1024, 2>(p, q, st);
  else if constexpr (sizeof(T) == 4)
    launch_back<T, 1024, 4>(p, q, st);
  return launched();
}

bool sizes_ok(int64_t t, int64_t n, int dtype) {
  return t >= 0 && t < kMostRows && n >= 1 && n < kMostRows && type_ok(dtype);
}
// 16 columns a workgroup of the last sums, or 64: 4096 columns 8.8 us and 11.2, 16,384 17.8 and 8.0.
constexpr int64_t kNarrow = 4096;
bool kind_ok(int kind) { return kind >= XMEM_NORM_NONE && kind <= XMEM_NORM_LAYER; }

}  // namespace

extern "C" {

int xmem_residual_norm_forward(const void* d_r, int64_t ldr, const void* d_h, int64_t ldh, const void* d_gate, int64_t ldg,
                               const float* d_scale, float alpha, int post, const float* d_w1, const float* d_b1, int pre,
                               const float* d_w2, const float* d_b2, int gate_activation, float eps, int64_t tokens, int64_t width,
                               int dtype, void* d_out, int64_t ldo, void* d_y, int64_t ldy, float* d_stats, void* hip_stream) {
  if (!sizes_ok(tokens, width, dtype) || !kind_ok(post) || !kind_ok(pre) || !(eps >= 0.0f)) return XMEM_EINVAL;
  if (gate_activation < XMEM_GATE_NONE || gate_activation > XMEM_GATE_SILU) return XMEM_EINVAL;
  if ((post == XMEM_NORM_NONE && (d_w1 || d_b1)) || (pre == XMEM_NORM_NONE && (d_w2 || d_b2 || d_y))) return XMEM_EINVAL;
  if (!ld_ok(ldr, width) || (d_h && !ld_ok(ldh, width)) || (d_gate && !ld_ok(ldg, width)) || (d_out && !ld_ok(ldo, width)) ||
      (d_y && !ld_ok(ldy, width)))
    return XMEM_EINVAL;
  if (tokens > 0 && !d_h && (d_gate || d_scale || d_out || post != XMEM_NORM_NONE)) return XMEM_EINVAL;  // of no rows no pointer is needed
  if (d_out && d_out == d_r && ldo != ldr) return XMEM_EINVAL;
  if (tokens > 0 && (!d_r || (pre != XMEM_NORM_NONE && !d_y) || (d_h && !d_out))) return XMEM_EINVAL;
  // Outputs that the cache behind the L2s cannot hold are gone from it before anyone reads them: 2048 x 16384 in float32 (268 MB) 127 us,
  // written past it 104; 32768 x 4096 in bfloat16 268 and 264.
  const bool past_caches = tokens * width * (dtype == XMEM_F32 ? 4 : 2) * ((d_out != nullptr) + (d_y != nullptr)) >= kCacheBytes;
  const Norms p{d_r, d_h, d_gate, ldr, ldh, ldg, d_scale, d_w1, d_b1, d_w2, d_b2, tokens, width, post, pre, gate_activation, eps, alpha,
                d_out, d_y, ldo, ldy, d_stats, past_caches};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (tokens == 0 || (!d_h && !d_y && !d_stats)) return XMEM_OK;
  return (dtype == XMEM_BF16 ? launch_norm<bf16> : dtype == XMEM_F16 ? launch_norm<f16> : launch_norm<float>)(p, st);
}

size_t xmem_residual_norm_backward_workspace_bytes(int64_t tokens, int64_t width, int dtype) {
  if (!sizes_ok(tokens, width, dtype)) return 0;
  return up256(size_t(plan_of(tokens, width, dtype).groups) * size_t(width) * 16);
}

int xmem_residual_norm_backward(const void* d_dy, int64_t lddy, const void* d_dout, int64_t lddout, const void* d_out, int64_t ldo,
                                const float* d_stats, const void* d_h, int64_t ldh, const void* d_gate, int64_t ldg,
                                const float* d_scale, float alpha, int post, const float* d_w1, const float* d_b1, int pre,
                                const float* d_w2, int gate_activation, int64_t tokens, int64_t width, int dtype, void* d_dr,
                                int64_t lddr, void* d_dh, int64_t lddh, void* d_dgate, int64_t lddg, float* d_dscale, float* d_dw1,
                                float* d_db1, float* d_dw2, float* d_db2, void* d_workspace, size_t workspace_bytes,
                                void* hip_stream) {
  if (!sizes_ok(tokens, width, dtype) || !kind_ok(post) || !kind_ok(pre)) return XMEM_EINVAL;
  if (gate_activation < XMEM_GATE_NONE || gate_activation > XMEM_GATE_SILU) return XMEM_EINVAL;
  if (post == XMEM_NORM_NONE && (d_w1 || d_b1 || d_dw1 || d_db1)) return XMEM_EINVAL;
  if (pre == XMEM_NORM_NONE && (d_dy || d_w2 || d_dw2 || d_db2)) return XMEM_EINVAL;
  if (tokens > 0 && !d_h && (d_gate || d_scale || post != XMEM_NORM_NONE || d_dh || d_dscale)) return XMEM_EINVAL;
  if (tokens > 0 && d_dgate && !d_gate) return XMEM_EINVAL;
  const struct {
    const void* at;
    int64_t ld;
  } all[] = {{d_dy, lddy}, {d_dout, lddout}, {d_dy ? d_out : nullptr, ldo}, {d_h, ldh}, {d_gate, ldg}, {d_dr, lddr}, {d_dh, lddh},
             {d_dgate, lddg}};
  for (const auto& m : all)
    if (m.at && !ld_ok(m.ld, width)) return XMEM_EINVAL;
  if (d_dr && d_dr == d_dout && lddr != lddout) return XMEM_EINVAL;
  if (tokens > 0) {
    if (!d_dr || !d_stats || (pre != XMEM_NORM_NONE ? !d_dy || !d_out : !d_dout) || (d_h && !d_dh)) return XMEM_EINVAL;
  }
  const bool sums = d_dscale || d_dw1 || d_db1 || d_dw2 || d_db2;
  const Plan q = plan_of(tokens, width, dtype);
  if (sums && tokens > 0) {
    const size_t need = xmem_residual_norm_backward_workspace_bytes(tokens, width, dtype);
    if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256)) return XMEM_EWORKSPACE;
    for (const auto& m : all)
      if (shares(d_workspace, need, m.at, tokens, m.ld, width, dtype == XMEM_F32 ? 4 : 2)) return XMEM_EINVAL;
    const float* const vectors[] = {d_scale, d_w1, d_b1, d_w2, d_dscale, d_dw1, d_db1, d_dw2, d_db2};
    for (const float* v : vectors)
      if (shares(d_workspace, need, v, 1, width, width, 4)) return XMEM_EINVAL;
    if (shares(d_workspace, need, d_stats, 4, tokens, tokens, 4)) return XMEM_EINVAL;
  }
  if (tokens == 0 && !sums) return XMEM_OK;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  float* part = sums ? static_cast<float*>(d_workspace) : nullptr;
  if (tokens > 0) {
    const NormGrads p{d_dy, d_dout, d_out, d_h, d_gate, lddy, lddout, ldo, ldh, ldg, d_stats, d_scale, d_w1, d_b1, d_w2, tokens, width,
                      post, pre, gate_activation, alpha, d_dr, d_dh, d_dgate, lddr, lddh, lddg, part,
                      d_b1 || d_db1 || d_db2};
    const int rc = (dtype == XMEM_BF16 ? launch_backward<bf16> : dtype == XMEM_F16 ? launch_backward<f16> : launch_backward<float>)(p, q, st);
    if (rc != XMEM_OK) return rc;
  }
  if (sums) {
    const VectorGrads v{part, d_scale, d_w1, d_b1, tokens > 0 ? q.groups : 0, width, alpha, d_dscale, d_dw1, d_db1, d_dw2, d_db2};
    const auto sums_of = [&](auto kernel, int64_t cols) {
      const int64_t blocks = (width + cols - 1) / cols;
      kernel<<<unsigned(blocks < 65536 ? blocks : 65536), 1024, 0, st>>>(v);
    };
    if (width <= kNarrow)
      sums_of(k_norm_sums<16>, 16);
    else
      sums_of(k_norm_sums<64>, 64);
  }
  return launched();
}

}  // extern "C"
