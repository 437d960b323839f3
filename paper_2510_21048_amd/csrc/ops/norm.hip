// norm.hip -- the norms before and after a block with its gate, scale and residual sum, and their gradients, on MI355X (gfx950).
//
// A row is read once: what it needs of its inputs stays in registers (a wavefront a row where they hold it, else a workgroup),
// two or four sums are taken of it, and its outputs are written once.  A norm's mean is taken before its squares, so nothing cancels.
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
  int64_t first = 0;  // row of the launch
};

__device__ inline float logistic(float g) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-g * kLog2e)); }

// What a gate's value multiplies with.
__device__ inline float gate_of(float g, int act) {
  return act == XMEM_GATE_NONE ? g : act == XMEM_GATE_SIGMOID ? logistic(g) : g * logistic(g);
}

// alpha s a(g) ((h - mu) rho w + b), piece by piece.
template <class T>
struct Branch {
  static constexpr int E = kPiece<T>;
  const Norms& p;
  float mu, rho;
  __device__ void of(u32x4 h, u32x4 g, int64_t i, float (&v)[E]) const {
    float w[E], b[E], s[E];
    unpack<T>(h, v);
    if (p.post != XMEM_NORM_NONE) {
      vector_of<E>(p.w1, i, p.n, 1.0f, w);
      vector_of<E>(p.b1, i, p.n, 0.0f, b);
#pragma unroll
      for (int k = 0; k < E; ++k) v[k] = (v[k] - mu) * rho * w[k] + b[k];
    }
    vector_of<E>(p.s, i, p.n, 1.0f, s);
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

template <int E>
__device__ inline float squares(const float (&v)[E], float mu, int64_t valid) {
  float s = 0.0f;
  if (valid >= E) {
#pragma unroll
    for (int k = 0; k < E; ++k) s += (v[k] - mu) * (v[k] - mu);
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) s += k < valid ? (v[k] - mu) * (v[k] - mu) : 0.0f;
  }
  return s;
}
template <int E>
__device__ inline float total(const float (&v)[E]) {
  float s = v[0];
#pragma unroll
  for (int k = 1; k < E; ++k) s += v[k];
  return s;
}

// Mean and reciprocal deviation of a row: `each(f)` calls f with every piece of the thread and the row's elements from it on.
template <int THREADS, class Each>
__device__ inline void moments(RowSums<THREADS>& sums, const Each& each, int kind, int64_t n, float eps, float& mu, float& rho) {
  mu = 0.0f;
  rho = 0.0f;
  if (kind == XMEM_NORM_NONE) return;
  float s = 0.0f;
  if (kind == XMEM_NORM_LAYER) {
    each([&](const auto& v, int64_t) { s += total(v); });
    mu = sums.one(s) / float(n);
    s = 0.0f;
  }
  each([&](const auto& v, int64_t valid) { s += squares(v, mu, valid); });
  rho = 1.0f / sqrtf(sums.one(s) / float(n) + eps);
}

template <int THREADS>
constexpr int kBlock = THREADS < 256 ? 256 : THREADS;

// THREADS of a row (64: four rows a workgroup), NCH pieces of it in each thread's registers.
template <class T, int THREADS, int NCH>
__global__ __launch_bounds__(kBlock<THREADS>) void k_norm(Norms p) {
  constexpr int E = kPiece<T>;
  __shared__ typename RowSums<THREADS>::Meet meet;
  RowSums<THREADS> sums(meet);
  const int tid = threadIdx.x % THREADS;
  const int64_t t = p.first + (THREADS < 256 ? int64_t(blockIdx.x) * (256 / THREADS) + threadIdx.x / THREADS : int64_t(blockIdx.x));
  if (t >= p.t) return;  // a whole wavefront, of those that do not meet others
  const int64_t n = p.n;
  const int pieces = int((n + E - 1) / E);
  const T* r = static_cast<const T*>(p.r) + t * p.ldr;
  float x[NCH][E], mu1 = 0.0f, rho1 = 0.0f, mu2, rho2;
  u32x4 cr[NCH];
#pragma unroll
  for (int j = 0; j < NCH; ++j)
    if (j * THREADS < pieces) cr[j] = piece_of(r, j * THREADS + tid, n);
  if (p.h) {
    const T* h = static_cast<const T*>(p.h) + t * p.ldh;
    const T* g = p.gate ? static_cast<const T*>(p.gate) + t * p.ldg : nullptr;
    u32x4 ch[NCH], cg[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * THREADS < pieces) {
        ch[j] = piece_of(h, j * THREADS + tid, n);
        if (g) cg[j] = piece_of(g, j * THREADS + tid, n);
      }
    moments<THREADS>(sums, [&](const auto& f) {
#pragma unroll
      for (int j = 0; j < NCH; ++j)
        if (j * THREADS < pieces) {
          float v[E];
          unpack<T>(ch[j], v);
          f(v, n - int64_t(j * THREADS + tid) * E);
        }
    }, p.post, n, p.eps, mu1, rho1);
    const Branch<T> branch{p, mu1, rho1};
    T* out = static_cast<T*>(p.out) + t * p.ldo;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * THREADS < pieces) {
        float v[E];
        branch.of(ch[j], cg[j], j * THREADS + tid, v);
        unpack<T>(cr[j], x[j]);
        const int64_t valid = n - int64_t(j * THREADS + tid) * E;
#pragma unroll
        for (int k = 0; k < E; ++k) x[j][k] = k < valid ? x[j][k] + v[k] : 0.0f;
        put_piece(out, j * THREADS + tid, n, x[j]);
      }
  } else {
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * THREADS < pieces) unpack<T>(cr[j], x[j]);
  }
  moments<THREADS>(sums, [&](const auto& f) {
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * THREADS < pieces) f(x[j], n - int64_t(j * THREADS + tid) * E);
  }, p.pre, n, p.eps, mu2, rho2);
  if (p.y) {
    T* y = static_cast<T*>(p.y) + t * p.ldy;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * THREADS < pieces) {
        float w[E], b[E];
        vector_of<E>(p.w2, j * THREADS + tid, n, 1.0f, w);
        vector_of<E>(p.b2, j * THREADS + tid, n, 0.0f, b);
#pragma unroll
        for (int k = 0; k < E; ++k) x[j][k] = (x[j][k] - mu2) * rho2 * w[k] + b[k];
        put_piece(y, j * THREADS + tid, n, x[j]);
      }
  }
  if (p.stats && tid == 0) {
    p.stats[t] = mu1;
    p.stats[p.t + t] = rho1;
    p.stats[2 * p.t + t] = mu2;
    p.stats[3 * p.t + t] = rho2;
  }
}

// A row that no registers hold: its inputs are read again for each sum, and outputs written last (out may be r).
template <class T>
__global__ __launch_bounds__(1024) void k_norm_long(Norms p) {
  constexpr int E = kPiece<T>, THREADS = 1024;
  __shared__ typename RowSums<THREADS>::Meet meet;
  RowSums<THREADS> sums(meet);
  const int64_t t = p.first + blockIdx.x, n = p.n, pieces = (n + E - 1) / E;
  const T* r = static_cast<const T*>(p.r) + t * p.ldr;
  const T* h = p.h ? static_cast<const T*>(p.h) + t * p.ldh : nullptr;
  const T* g = p.gate ? static_cast<const T*>(p.gate) + t * p.ldg : nullptr;
  float mu1, rho1, mu2, rho2;
  moments<THREADS>(sums, [&](const auto& f) {
    for (int64_t i = threadIdx.x; i < pieces; i += THREADS) {
      float v[E];
      unpack<T>(piece_of(h, i, n), v);
      f(v, n - i * E);
    }
  }, h ? p.post : XMEM_NORM_NONE, n, p.eps, mu1, rho1);
  const Branch<T> branch{p, mu1, rho1};
  const auto sum = [&](int64_t i, float (&x)[E]) {
    unpack<T>(piece_of(r, i, n), x);
    if (h) {
      float v[E];
      branch.of(piece_of(h, i, n), g ? piece_of(g, i, n) : u32x4{}, i, v);
#pragma unroll
      for (int k = 0; k < E; ++k) x[k] = i * E + k < n ? x[k] + v[k] : 0.0f;
    }
  };
  moments<THREADS>(sums, [&](const auto& f) {
    for (int64_t i = threadIdx.x; i < pieces; i += THREADS) {
      float x[E];
      sum(i, x);
      f(x, n - i * E);
    }
  }, p.pre, n, p.eps, mu2, rho2);
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

template <class T>
int launch_norm(const Norms& p, hipStream_t st) {
  const int64_t pieces = (p.n + kPiece<T> - 1) / kPiece<T>;
  if (pieces <= 64) return launch_rows(k_norm<T, 64, 1>, p, 4, 256, st);
  if (pieces <= 64 * 2) return launch_rows(k_norm<T, 64, 2>, p, 4, 256, st);
  if (pieces <= 64 * 4) return launch_rows(k_norm<T, 64, 4>, p, 4, 256, st);
  if (pieces <= 256 * 2) return launch_rows(k_norm<T, 256, 2>, p, 1, 256, st);
  if (pieces <= 256 * 4) return launch_rows(k_norm<T, 256, 4>, p, 1, 256, st);
  if (pieces <= 1024 * 2) return launch_rows(k_norm<T, 1024, 2>, p, 1, 1024, st);
  if (pieces <= 1024 * 4) return launch_rows(k_norm<T, 1024, 4>, p, 1, 1024, st);
  return launch_rows(k_norm_long<T>, p, 1, 1024, st);
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
  // dr from dout, e, xhat2 and the means of e and e xhat2, where `valid` elements are the row's; 0 behind them
  __device__ void grad(u32x4 cdout, const float (&e)[E], const float (&hat)[E], float mean_e, float mean_eh, int64_t valid,
                       float (&d)[E]) const {
    unpack<T>(cdout, d);
#pragma unroll
    for (int k = 0; k < E; ++k) d[k] += rho2 * (e[k] - mean_e - hat[k] * mean_eh);
    if (valid < E)
#pragma unroll
      for (int k = 0; k < E; ++k) d[k] = k < valid ? d[k] : 0.0f;
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

// BLOCK / W rows at a time, W threads and NCH pieces a thread each, whose columns' sums over all of the workgroup's rows stay
// in registers (with NCH of 2, those of B and D in LDS).
template <class T, int W, int NCH, bool BIASES, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_norm_back(NormGrads p) {
  constexpr int E = kPiece<T>, R = BLOCK / W, HELD = NCH == 1 && BIASES ? 4 : 2, VECTORS = BIASES ? 4 : 3;
  constexpr bool APART = BIASES && HELD == 2;  // B and D in LDS
  __shared__ typename RowSums<W, R>::Meet meet;
  __shared__ float apart[APART ? 2 : 1][APART ? NCH * E : 1][APART ? BLOCK : 1], rows[R > 1 ? E : 1][R > 1 ? BLOCK : 1];
  __shared__ f32x4 columns[NCH == 1 ? VECTORS : 1][NCH == 1 ? E / 4 : 1][NCH == 1 ? W : 1];
  const int slot = __builtin_amdgcn_readfirstlane(threadIdx.x / W), tid = threadIdx.x % W;
  RowSums<W, R> sums(meet, slot);
  const int n = int(p.n), pieces = (n + E - 1) / E;
  if constexpr (NCH == 1) {
    for (int i = threadIdx.x; i < VECTORS * W * E; i += BLOCK) {
      const int q = i / (W * E), c = i % (W * E);
      reinterpret_cast<float*>(&columns[q][c % E / 4][c / E])[c % 4] = c < n ? column_of(p, q, c) : 0.0f;
    }
    __syncthreads();
  }
  const auto vector = [&](int q, int j, float (&v)[E]) {
    if constexpr (NCH == 1) {
      if (q < VECTORS) {
#pragma unroll
        for (int h = 0; h < E / 4; ++h) __builtin_memcpy(v + 4 * h, &columns[q][h][tid], 16);
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = 0.0f;
      }
    } else {
#pragma unroll
      for (int k = 0; k < E; ++k) {
        const int c = (j * W + tid) * E + k;
        v[k] = q < VECTORS ? column_of(p, q, c < n ? c : n - 1) : 0.0f;
      }
    }
  };
  float acc[HELD][NCH][E] = {};  // A, B, C, D or A, C
  if constexpr (APART)
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int k = 0; k < NCH * E; ++k) apart[q][k][threadIdx.x] = 0.0f;
  const auto add = [&](int q, int j, int k, float v) {  // q: 0 to 3 for A to D
    if constexpr (HELD == 4)
      acc[q][j][k] += v;
    else if constexpr (!BIASES)
      acc[q / 2][j][k] += v;
    else if (q & 1)
      apart[q / 2][j * E + k][threadIdx.x] += v;
    else
      acc[q / 2][j][k] += v;
  };
  for (int64_t t0 = int64_t(blockIdx.x) * R; t0 < p.t; t0 += int64_t(gridDim.x) * R) {
    const int64_t t = t0 + slot, at = t < p.t ? t : 0;
    const bool here = t < p.t;  // a row that is not there is one of 0, and not written
    const auto row = [&](const void* x, int64_t ld, int j) {
      return here ? near_piece(static_cast<const T*>(x) + at * ld, j * W + tid, n) : u32x4{};
    };
    const auto put = [&](void* x, int64_t ld, int j, const float (&v)[E]) {
      if (here) put_piece(static_cast<T*>(x) + at * ld, j * W + tid, n, v);
    };
    u32x4 cdy[NCH], cdo[NCH], co[NCH], ch[NCH], cg[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        if (p.dy) {
          cdy[j] = row(p.dy, p.lddy, j);
          co[j] = row(p.out, p.ldo, j);
        }
        cdo[j] = p.dout ? row(p.dout, p.lddo, j) : u32x4{};
        if (p.h) ch[j] = row(p.h, p.ldh, j);
        if (p.gate) cg[j] = row(p.gate, p.ldg, j);
      }
    const Piece<T> q{p, p.stats[at], p.stats[p.t + at], p.stats[2 * p.t + at], p.stats[3 * p.t + at]};
    float d[NCH][E];
    if (p.dy) {
      float s1 = 0.0f, s2 = 0.0f, e[E], hat[E], dy[E], w[E];
#pragma unroll
      for (int j = 0; j < NCH; ++j)
        if (j * W < pieces) {
          vector(2, j, w);
          q.first(cdy[j], co[j], w, e, hat, dy);
#pragma unroll
          for (int k = 0; k < E; ++k) {
            s1 += e[k] * hat[k];
            s2 += e[k];
            add(2, j, k, dy[k] * hat[k]);
            if (BIASES) add(3, j, k, dy[k]);
          }
        }
      if (p.pre == XMEM_NORM_LAYER)
        sums.two(s1, s2);
      else
        s1 = sums.one(s1), s2 = 0.0f;
      s1 /= float(n);
      s2 /= float(n);
#pragma unroll
      for (int j = 0; j < NCH; ++j)
        if (j * W < pieces) {
          vector(2, j, w);
          q.first(cdy[j], co[j], w, e, hat, dy);
          q.grad(cdo[j], e, hat, s2, s1, n - (j * W + tid) * E, d[j]);
        }
    } else {
#pragma unroll
      for (int j = 0; j < NCH; ++j)
        if (j * W < pieces) unpack<T>(cdo[j], d[j]);
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) put(p.dr, p.lddr, j, d[j]);
    if (!p.h) continue;
    float s1 = 0.0f, s2 = 0.0f, b[E], hat[E], f[E], dg[E], s[E], w1[E], b1[E];
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        vector(0, j, s);
        vector(1, j, w1);
        vector(3, j, b1);
        q.second(ch[j], cg[j], d[j], s, w1, b1, b, hat, f, dg);
        if (p.dg) put(p.dg, p.lddg, j, dg);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          s1 += f[k] * hat[k];
          s2 += f[k];
          add(0, j, k, b[k] * hat[k]);
          if (BIASES) add(1, j, k, b[k]);
          d[j][k] = f[k];
        }
      }
    if (p.post != XMEM_NORM_NONE) {
      if (p.post == XMEM_NORM_LAYER)
        sums.two(s1, s2);
      else
        s1 = sums.one(s1), s2 = 0.0f;
      s1 /= float(n);
      s2 /= float(n);
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * W < pieces) {
        if (p.post != XMEM_NORM_NONE) {
          unpack<T>(ch[j], hat);
#pragma unroll
          for (int k = 0; k < E; ++k) d[j][k] = q.rho1 * (d[j][k] - s2 - (hat[k] - q.mu1) * q.rho1 * s1);
        }
        put(p.dh, p.lddh, j, d[j]);
      }
  }
  if (!p.part) return;
  // the workgroup's rows, then its part of each sum
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (!BIASES && (q & 1)) continue;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      float v[E];
#pragma unroll
      for (int k = 0; k < E; ++k) {
        if constexpr (APART)
          v[k] = q & 1 ? apart[q / 2][j * E + k][threadIdx.x] : acc[q / 2][j][k];
        else
          v[k] = acc[HELD == 4 ? q : q / 2][j][k];
      }
      if constexpr (R > 1) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < E; ++k) rows[k][threadIdx.x] = v[k];
        __syncthreads();
        if (slot == 0)
#pragma unroll
          for (int k = 0; k < E; ++k)
#pragma unroll
            for (int w = 1; w < R; ++w) v[k] += rows[k][w * W + tid];
      }
      if (slot == 0) put_vector(p.part + (int64_t(q) * gridDim.x + blockIdx.x) * n, j * W + tid, n, v);
    }
  }
}

// Rows that no registers hold: each is read three times, and a workgroup's sums are kept where its parts go.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_back_long(NormGrads p) {
  constexpr int E = kPiece<T>, THREADS = 1024;
  __shared__ typename RowSums<THREADS>::Meet meet;
  RowSums<THREADS> sums(meet);
  const int64_t n = p.n, pieces = (n + E - 1) / E;
  for (int64_t t = blockIdx.x; t < p.t; t += gridDim.x) {
    const auto row = [&](const void* x, int64_t ld, int64_t i) {
      return x ? piece_of(static_cast<const T*>(x) + t * ld, i, n) : u32x4{};
    };
    const auto vector = [&](int q, int64_t i, float (&v)[E]) {
#pragma unroll
      for (int k = 0; k < E; ++k) v[k] = column_of(p, q, i * E + k < n ? i * E + k : n - 1);
    };
    const Piece<T> q{p, p.stats[t], p.stats[p.t + t], p.stats[2 * p.t + t], p.stats[3 * p.t + t]};
    float s1 = 0.0f, s2 = 0.0f, s3 = 0.0f, s4 = 0.0f, e[E], hat[E], dy[E], d[E], b[E], f[E], dg[E], s[E], w[E], add[E];
    if (p.dy) {
      for (int64_t i = threadIdx.x; i < pieces; i += THREADS) {
        vector(2, i, w);
        q.first(row(p.dy, p.lddy, i), row(p.out, p.ldo, i), w, e, hat, dy);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          s1 += e[k] * hat[k];
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
        q.grad(row(p.dout, p.lddo, i), e, hat, s2, s1, n - i * E, d);
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
          s3 += f[k] * hat[k];
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

// The groups' parts added up in a fixed order: sixteen wavefronts a share of the groups each, then their sums.
__global__ __launch_bounds__(1024) void k_norm_sums(VectorGrads p) {
  __shared__ float sums[16][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool wanted[4] = {p.ds || p.dw1, p.db1 || (p.ds && p.b1), p.dw2 != nullptr, p.db2 != nullptr};
  for (int64_t c = int64_t(blockIdx.x) * 64 + lane; c - lane < p.n; c += int64_t(gridDim.x) * 64) {
    float v[4] = {};
    if (c < p.n)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (wanted[q])
#pragma unroll 8
          for (int64_t g = wave; g < p.groups; g += 16) v[q] += p.part[(q * p.groups + g) * p.n + c];
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[wave][q][lane] = v[q];
    __syncthreads();
    if (wave == 0 && c < p.n) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        for (int w = 1; w < 16; ++w) v[q] += sums[w][q][lane];
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
constexpr int kBackBlock = 1024;
struct Plan {
  int threads, nch;
  int64_t groups;
};
Plan plan_of(int64_t t, int64_t n, int dtype) {
  const int e = dtype == XMEM_F32 ? 4 : 8;
  const int64_t pieces = (n + e - 1) / e;
  Plan q{64, 1, 0};
  while (q.threads < kBackBlock && q.threads < pieces) q.threads *= 2;
  if (pieces > kBackBlock) q.nch = pieces <= 2 * kBackBlock ? 2 : 0;
  const int per = kBackBlock / q.threads;
  const int64_t rows = (t + per - 1) / per;
  int64_t most = kCus;
  if (q.nch == 0) {  // parts of 256 MiB at most, or one group's
    const int64_t fit = (int64_t(1) << 24) / n;
    most = fit < 1 ? 1 : fit < most ? fit : most;
  }
  q.groups = rows < most ? rows : most;
  return q;
}

template <class T, int W, int NCH>
void launch_back(const NormGrads& p, const Plan& q, hipStream_t st) {
  if (p.biases)
    k_norm_back<T, W, NCH, true, kBackBlock><<<unsigned(q.groups), kBackBlock, 0, st>>>(p);
  else
    k_norm_back<T, W, NCH, false, kBackBlock><<<unsigned(q.groups), kBackBlock, 0, st>>>(p);
}
template <class T>
int launch_backward(const NormGrads& p, const Plan& q, hipStream_t st) {
  if (q.nch == 0)
    k_norm_back_long<T><<<unsigned(q.groups), 1024, 0, st>>>(p);
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
  else
    launch_back<T, 1024, 2>(p, q, st);
  return launched();
}

bool sizes_ok(int64_t t, int64_t n, int dtype) {
  return t >= 0 && t < kMostRows && n >= 1 && n < kMostRows && type_ok(dtype);
}
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
  const Norms p{d_r, d_h, d_gate, ldr, ldh, ldg, d_scale, d_w1, d_b1, d_w2, d_b2, tokens, width, post, pre, gate_activation, eps, alpha,
                d_out, d_y, ldo, ldy, d_stats};
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
  if (sums && tokens > 0 &&
      (!d_workspace || workspace_bytes < xmem_residual_norm_backward_workspace_bytes(tokens, width, dtype) || !aligned(d_workspace, 256)))
    return XMEM_EWORKSPACE;
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
    const int64_t blocks = (width + 63) / 64;
    k_norm_sums<<<unsigned(blocks < 65536 ? blocks : 65536), 1024, 0, st>>>(v);
  }
  return launched();
}

}  // extern "C"
