// muon.hip -- momentum and the update orthogonalised by Newton-Schulz products, on MI355X (gfx950).
//
// X is kept as the caller's matrices lie: [long, short] where rows > cols, [short, long] else, so nothing is
// transposed; the matrix product reads either layout.  With P = X X^T (short by short, symmetric) and
// Q = b P + c P P, a step is X <- a X + Q X.
//
// Numbers.  The products take half-precision operands: 11 bits where bfloat16 has 8, and the range is no matter
// since |X|_F <= 1 at the start and no singular value passes 1.3 afterwards; powers of two (kX for X, kP for P and Q) keep small
// entries normal.  Three things hold the error near 7e-4 of the update (its bfloat16 rounding: 1.7e-3):
//   - the diagonals of P and Q, which are far larger than the rest, are kept apart in 32 bits and the products take
//     the matrices without them: (P P)_ij = (E E)_ij + (d_i + d_j) E_ij, and + d_i^2 on the diagonal;
//   - the linear terms (a + q_ii) X_i take X from two halves of 11 bits (but in the last two steps), so that directions in
//     which the gradient is weak, which a step multiplies by a, are not lost in the rounding of the strong ones;
//   - Q is made from the same rounded P in both terms: b + 2 c p is near 0 where P is near 1, so that its error cancels.
// On matrices of normal values the products alone, in bfloat16, leave 1e-2; in half precision without these, 1.5e-3;
// where one direction holds most of a gradient, 1.6e-1 and 2e-2.
//
// A |u| far below the 1e-7 added to it makes X as small, and its entries lose bits past half precision's range: of an update below
// a hundredth of a usual one.
//
// Bound by the products where matrices are large: 24 of 8192 x 2048 take 17.0 to 17.3 ms, of which the five X X^T 5.1 to 5.4 (800 TFLOP/s of
// the half that is computed: 864 tiles in 3.4 rounds), P P 1.3, Q X 7.6 to 9.3 (its 32 k tiles a workgroup are followed by 8 bytes read and
// written an element, which nothing hides), momentum and start 1.6 (4 GB each at 4.5 and 5.5 TB/s).  A single 1024 x 1024 takes
// 159 us: 17 launches one after another, 10 us a product.
#include "gemm.h"

using namespace xops;

namespace {

constexpr float kX = 256.0f, kP = 1024.0f;
constexpr float kNormEps = 1e-7f;
constexpr int kThreads = 256;
// The steps at the end whose X is kept in one half: a rounding there is multiplied by a^2 at most, and on a gradient of
// 16 strong directions over weak ones the error goes from 4e-4 to 1.3e-3; each such step moves 4 of 8 bytes less.
constexpr int kOneHalf = 2;
constexpr int kNormParts = 256;  // workgroups whose sums make one matrix's norm
constexpr int64_t kMostCount = 65535, kMostSide = kMostDirectLd - 64;

struct Shape {
  int64_t count, rows, cols, s, l;  // s <= l
  int64_t lds, ldx;                 // row lengths of P, Q and of X: whole lines
  bool tall;                        // rows > cols: X lies as [l, s]
};
Shape shape_of(int64_t count, int64_t rows, int64_t cols) {
  Shape h{count, rows, cols, rows < cols ? rows : cols, rows < cols ? cols : rows, 0, 0, rows > cols};
  h.lds = packed_ld(h.s);
  h.ldx = packed_ld(cols);
  return h;
}

struct Ws {
  f16 *x[2], *lo[2];  // X and its second half, before and after a step
  f16 *p, *q;         // behind their rows' ends are zeros, as behind X's
  float *dp, *dq;  // diagonals
  double* part;
  void* split;  // partial sums of products whose k is split
  size_t bytes;
};
Ws carve(void* base, const Shape& h) {
  Ws w;
  char* at = static_cast<char*>(base);
  const auto take = [&](size_t b) {
    char* r = at;
    at += up256(b);
    return r;
  };
  const size_t nx = size_t(h.count) * h.rows * h.ldx * 2, np = size_t(h.count) * h.s * h.lds * 2;
  for (int i = 0; i < 2; ++i) {
    w.x[i] = reinterpret_cast<f16*>(take(nx));
    w.lo[i] = reinterpret_cast<f16*>(take(nx));
  }
  w.p = reinterpret_cast<f16*>(take(np));
  w.q = reinterpret_cast<f16*>(take(np));
  w.dp = reinterpret_cast<float*>(take(size_t(h.count) * h.s * 4));
  w.dq = reinterpret_cast<float*>(take(size_t(h.count) * h.s * 4));
  w.part = reinterpret_cast<double*>(take(size_t(h.count) * kNormParts * 8));
  const size_t s1 = part_bytes(h.s, h.s, h.l, h.count, true), s2 = part_bytes(h.s, h.s, h.s, h.count, true),
               s3 = h.tall ? part_bytes(h.l, h.s, h.s, h.count, false) : part_bytes(h.s, h.l, h.s, h.count, false);
  w.split = take(s1 > s2 ? (s1 > s3 ? s1 : s3) : s2 > s3 ? s2 : s3);
  w.bytes = size_t(at - static_cast<char*>(base));
  return w;
}

// m <- mu m + g, and the squares of u summed in 64 bits (their range is no matter then).  Eight elements a thread at a time.
template <class G>
__global__ __launch_bounds__(kThreads) void k_momentum(const G* g, float* mom, int64_t per, float mu, bool nesterov, double* part) {
  __shared__ double sums[kThreads / kWave];
  g += int64_t(blockIdx.y) * per;
  mom += int64_t(blockIdx.y) * per;
  double sum = 0.0;
  for (int64_t i = (int64_t(blockIdx.x) * kThreads + threadIdx.x) * 8; i < per; i += int64_t(kNormParts) * kThreads * 8) {
    const int valid = per - i >= 8 ? 8 : int(per - i);
    float e[8], m[8];
    get<G, 8>(g + i, valid, e);
    get<float, 8>(mom + i, valid, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = mu * m[j] + e[j];
      const double u = nesterov ? e[j] + mu * m[j] : m[j];
      sum += u * u;
    }
    put<float, 8, Any>(mom + i, valid, m);
  }
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double v = 0.0;
    for (int i = 0; i < kThreads / kWave; ++i) v += sums[i];
    part[blockIdx.y * kNormParts + blockIdx.x] = v;
  }
}

// X = u / (|u| + eps) in two halves; 0 behind a row's end, up to a multiple of 8.
template <class G>
__global__ __launch_bounds__(kThreads) void k_start(const G* g, const float* mom, int64_t rows, int64_t cols, int64_t ldx, float mu,
                                                    bool nesterov, const double* part, f16* x, f16* lo) {
  const int64_t b = blockIdx.y;
  double v = 0.0;
#pragma unroll
  for (int i = 0; i < kNormParts / kWave; ++i) v += part[b * kNormParts + i * kWave + (threadIdx.x & 63)];
  v = wave_sum(v);
  const float inv = kX / (float(sqrt(v)) + kNormEps);
  const unsigned pieces = unsigned((cols + 7) / 8);
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < rows * pieces; i += int64_t(gridDim.x) * kThreads) {
    const int64_t r = i / pieces, c = (i - r * pieces) * 8, at = (b * rows + r) * cols + c;
    const int valid = cols - c >= 8 ? 8 : int(cols - c);
    float e[8], m[8];
    get<float, 8>(mom + at, valid, m);
    if (nesterov) get<G, 8>(g + at, valid, e);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = (nesterov ? e[j] + mu * m[j] : m[j]) * inv;
      m[j] = j < valid ? m[j] : 0.0f;  // infinities and NaN in g must not reach the padding
      e[j] = m[j] - float(f16(m[j]));
    }
    put<f16, 8, Any>(x + (b * rows + r) * ldx + c, 8, m);
    put<f16, 8, Any>(lo + (b * rows + r) * ldx + c, 8, e);
  }
}

// Clears what is behind the rows of the matrices that no kernel of the start writes, up to a multiple of 8: what a piece of
// 16 bytes reads with them.  y: the second X, P, Q.
__global__ void k_clear_pads(f16* x, f16* p, f16* q, int64_t rows_x, int64_t cols_x, int64_t ldx, int64_t rows_p, int64_t cols_p, int64_t ldp) {
  f16* at = blockIdx.y == 0 ? x : blockIdx.y == 1 ? p : q;
  const int64_t rows = blockIdx.y ? rows_p : rows_x, cols = blockIdx.y ? cols_p : cols_x, ld = blockIdx.y ? ldp : ldx, pad = -cols & 7;
  const int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i < rows * pad) at[i / pad * ld + cols + i % pad] = f16(0.0f);
}

// Which of the W columns from n on is m's own, or -1.
template <int W>
__device__ inline int diagonal(int64_t m, int64_t n) {
  return m >= n && m < n + W ? int(m - n) : -1;
}

// P = X X^T without its diagonal, which goes to d.  Only tiles on or below the diagonal are computed; the tiles below it
// are written to their mirrored places too.
struct GramEpilogue {
  static constexpr bool kSymmetric = true, kPastL2 = false, kAnyRows = false;  // what it writes is read next
  f16* p;
  float* d;
  int64_t ld;

  template <class F>
  __device__ __attribute__((always_inline)) void chosen(F f) const { f(*this); }
  __device__ f16* mirrored(int z, const GemmArgs& g) const { return p + z * g.m * ld; }
  template <int W>
  __device__ None column(int64_t, int, int, const GemmArgs&) const { return {}; }
  template <int W> using Read = None;
  template <int W>
  __device__ None read(int64_t, int64_t, int, int, const GemmArgs&) const { return {}; }
  template <int W, class HOW>
  __device__ void row(int64_t m, int64_t n, float (&v)[W], int valid, None, None, int z, const GemmArgs& g) const {
    const int here = diagonal<W>(m, n);
    float dm = 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      v[j] *= kP / (kX * kX);
      dm = j == here ? v[j] : dm;
      v[j] = j == here ? 0.0f : v[j];
    }
    if (here >= 0) d[z * g.m + m] = dm * (1.0f / kP);
    put<f16, W, HOW>(p + (z * g.m + m) * ld + n, valid, v);
  }
};

// Q = b P + c P P without its diagonal.
struct PolyEpilogue {
  static constexpr bool kSymmetric = true, kPastL2 = false, kAnyRows = false;
  const f16* p;
  const float* dp;
  f16* q;
  float* dq;
  int64_t ld;

  template <class F>
  __device__ __attribute__((always_inline)) void chosen(F f) const { f(*this); }
  __device__ f16* mirrored(int z, const GemmArgs& g) const { return q + z * g.m * ld; }
  template <int W>
  __device__ Column<W> column(int64_t n, int valid, int z, const GemmArgs& g) const {
    Column<W> c;
#pragma unroll
    for (int j = 0; j < W; ++j) c.v[j] = j < valid ? dp[z * g.m + n + j] : 0.0f;
    return c;
  }
  template <int W>
  struct Read {  // as it lies: half the registers
    typedef f16 part __attribute__((ext_vector_type(W)));
    part e;
    float dm;
  };
  template <int W>
  __device__ Read<W> read(int64_t m, int64_t n, int, int z, const GemmArgs& g) const {
    Read<W> r;
    r.dm = dp[z * g.m + m];
    // a row's storage is a multiple of 8 long: whole pieces, whatever of them is the matrix
    __builtin_memcpy(&r.e, p + (z * g.m + m) * ld + n, sizeof(r.e));
    return r;
  }
  template <int W, class HOW>
  __device__ void row(int64_t m, int64_t n, float (&v)[W], int valid, const Column<W>& dn, const Read<W>& r, int z, const GemmArgs& g) const {
    const int here = diagonal<W>(m, n);
    float ee = 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      ee = j == here ? v[j] : ee;
      const float e = float(r.e[j]);  // times kP; E_ii is 0
      v[j] = j == here ? 0.0f : XMEM_NS_B * e + XMEM_NS_C * (v[j] * (1.0f / kP) + (r.dm + dn.v[j]) * e);
    }
    if (here >= 0) dq[z * g.m + m] = XMEM_NS_B * r.dm + XMEM_NS_C * (ee * (1.0f / (kP * kP)) + r.dm * r.dm);
    put<f16, W, HOW>(q + (z * g.m + m) * ld + n, valid, v);
  }
};

// X <- (a + q_ii) X_i + (Q X)_i.  The diagonal's index is the row where X lies as [s, l], the column else.
template <bool TALL>
struct StepEpilogue {
  static constexpr bool kSymmetric = false, kPastL2 = true, kAnyRows = false;
  bool lines() const { return out ? whole_lines(out, cols) : whole_lines(nx, ld) && whole_lines(nlo, ld); }
  template <class F>
  __device__ __attribute__((always_inline)) void chosen(F f) const { f(*this); }
  const f16 *x, *lo;  // lo, nlo: NULL where X is kept in one half
  const float* dq;
  f16 *nx, *nlo;
  int64_t ld, s, cols;
  bf16* out;  // the last step writes the update instead
  float scale;

  template <int W>
  __device__ Column<W> column(int64_t n, int valid, int z, const GemmArgs&) const {
    Column<W> c;
#pragma unroll
    for (int j = 0; j < W; ++j) c.v[j] = TALL && j < valid ? XMEM_NS_A + dq[z * s + n + j] : 0.0f;
    return c;
  }
  template <int W>
  struct Read {  // as they lie: half the registers
    typedef f16 part __attribute__((ext_vector_type(W)));
    part hi, lo;
    float dm;
  };
  template <int W>
  __device__ Read<W> read(int64_t m, int64_t n, int, int z, const GemmArgs& g) const {
    const int64_t at = (z * g.m + m) * ld + n;
    Read<W> r;
    r.dm = TALL ? 0.0f : XMEM_NS_A + dq[z * s + m];
    // a row's storage is a multiple of 8 long: whole pieces, whatever of them is the matrix
    __builtin_memcpy(&r.hi, x + at, sizeof(r.hi));
    if (lo)
      __builtin_memcpy(&r.lo, lo + at, sizeof(r.lo));
    else
      r.lo = typename Read<W>::part(f16(0.0f));
    return r;
  }
  template <int W, class HOW>
  __device__ void row(int64_t m, int64_t n, float (&v)[W], int valid, const Column<W>& dn, const Read<W>& r, int z, const GemmArgs& g) const {
    const int64_t at = (z * g.m + m) * ld + n;
    float rest[W];
#pragma unroll
    for (int j = 0; j < W; ++j)
      v[j] = (TALL ? dn.v[j] : r.dm) * (float(r.hi[j]) + float(r.lo[j])) + v[j] * (1.0f / kP);  // times kX
    if (out) {
#pragma unroll
      for (int j = 0; j < W; ++j) v[j] *= scale / kX;
      put<bf16, W, HOW>(out + (z * g.m + m) * g.n + n, valid, v);
    } else {
      put<f16, W, HOW>(nx + at, valid, v);
      if (nlo) {
#pragma unroll
        for (int j = 0; j < W; ++j) rest[j] = v[j] - float(f16(v[j]));
        put<f16, W, HOW>(nlo + at, valid, rest);
      }
    }
  }
};

__global__ __launch_bounds__(kThreads) void k_scaled(const f16* x, const f16* lo, int64_t rows, int64_t cols, int64_t ldx, float scale,
                                                     bf16* out) {
  const int64_t b = blockIdx.y;
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < rows * cols; i += int64_t(gridDim.x) * kThreads) {
    const int64_t at = b * rows * ldx + i / cols * ldx + i % cols;
    out[b * rows * cols + i] = bf16((float(x[at]) + float(lo[at])) * (scale / kX));
  }
}

unsigned blocks_of(int64_t n) {
  const int64_t b = (n + kThreads - 1) / kThreads;
  return unsigned(b < 1 ? 1 : b > 4096 ? 4096 : b);
}

template <class G>
int update(const G* g, float* mom, const Shape& h, float mu, bool nesterov, int steps, float scale, bf16* out, void* base,
           hipStream_t st) {
  Ws w = carve(base, h);
  const int64_t per = h.rows * h.cols;
  const unsigned z = unsigned(h.count);
  k_momentum<G><<<dim3(kNormParts, z), kThreads, 0, st>>>(g, mom, per, mu, nesterov, w.part);
  k_start<G><<<dim3(blocks_of(h.rows * ((h.cols + 7) / 8)), z), kThreads, 0, st>>>(g, mom, h.rows, h.cols, h.ldx, mu, nesterov, w.part, w.x[0],
                                                                   w.lo[0]);
  int rc = launched();
  if (steps == 0) {
    k_scaled<<<dim3(blocks_of(per), z), kThreads, 0, st>>>(w.x[0], w.lo[0], h.rows, h.cols, h.ldx, scale, out);
    return launched();
  }
  const int64_t sx = h.rows * h.ldx, sp = h.s * h.lds;
  const int64_t pads_x = h.count * h.rows * (-h.cols & 7), pads_p = h.count * h.s * (-h.s & 7), pads = pads_x > pads_p ? pads_x : pads_p;
  if (pads > 0)
    k_clear_pads<<<dim3(unsigned((pads + 255) / 256), 3), 256, 0, st>>>(w.x[1], w.p, w.q, h.count * h.rows, h.cols, h.ldx, h.count * h.s, h.s, h.lds);
  for (int i = 0; i < steps && rc == XMEM_OK; ++i) {
    const f16 *x = w.x[i & 1], *lo = i == 0 || i < steps - kOneHalf ? w.lo[i & 1] : nullptr;
    bf16* to = i == steps - 1 ? out : nullptr;
    const auto args = [&](const f16* a, int64_t lda, int64_t sa, const f16* b, int64_t ldb, int64_t sb, int64_t m, int64_t n, int64_t k) {
      return GemmArgs{a, b, lda, ldb, sa, sb, m, n, k, true, true, h.count};
    };
    const GemmArgs gram = args(x, h.ldx, sx, x, h.ldx, sx, h.s, h.s, h.l);
    const GramEpilogue ge{w.p, w.dp, h.lds};
    const PolyEpilogue pe{w.p, w.dp, w.q, w.dq, h.lds};
    rc = h.tall ? gemm<f16, false, false>(gram, ge, w.split, st) : gemm<f16, true, true>(gram, ge, w.split, st);
    if (rc == XMEM_OK) rc = gemm<f16, true, true>(args(w.p, h.lds, sp, w.p, h.lds, sp, h.s, h.s, h.s), pe, w.split, st);
    if (rc != XMEM_OK) break;
    f16 *nx = w.x[~i & 1], *nlo = i + 1 < steps - kOneHalf ? w.lo[~i & 1] : nullptr;
    if (h.tall)
      rc = gemm<f16, true, true>(args(x, h.ldx, sx, w.q, h.lds, sp, h.l, h.s, h.s),
                                 StepEpilogue<true>{x, lo, w.dq, nx, nlo, h.ldx, h.s, h.cols, to, scale}, w.split, st);
    else
      rc = gemm<f16, true, false>(args(w.q, h.lds, sp, x, h.ldx, sx, h.s, h.l, h.s),
                                  StepEpilogue<false>{x, lo, w.dq, nx, nlo, h.ldx, h.s, h.cols, to, scale}, w.split, st);
  }
  return rc;
}

bool sizes_ok(int64_t count, int64_t rows, int64_t cols) {
  return count >= 0 && count <= kMostCount && rows >= 0 && cols >= 0 && rows < kMostSide && cols < kMostSide &&
         rows * cols < (int64_t(1) << 40) && count * ((rows + 63) / 64) * ((cols + 63) / 64) < (int64_t(1) << 28);
}

}  // namespace

extern "C" {

size_t xmem_muon_update_workspace_bytes(int64_t count, int64_t rows, int64_t cols) {
  if (!sizes_ok(count, rows, cols) || count == 0 || rows == 0 || cols == 0) return 0;
  return carve(nullptr, shape_of(count, rows, cols)).bytes;
}

int xmem_muon_update(const void* d_grad, int grad_dtype, float* d_momentum, int64_t count, int64_t rows, int64_t cols,
                     float mu, int nesterov, int steps, float scale, void* d_update, void* d_workspace,
                     size_t workspace_bytes, void* hip_stream) {
  if (!sizes_ok(count, rows, cols) || grad_dtype < XMEM_BF16 || grad_dtype > XMEM_F32 || steps < 0 || steps > XMEM_NS_MAX_STEPS)
    return XMEM_EINVAL;
  if (count == 0 || rows == 0 || cols == 0) return XMEM_OK;
  if (!d_grad || !d_momentum || !d_update) return XMEM_EINVAL;
  const Shape h = shape_of(count, rows, cols);
  if (!d_workspace || workspace_bytes < xmem_muon_update_workspace_bytes(count, rows, cols) || !aligned(d_workspace, 256))
    return XMEM_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  bf16* out = static_cast<bf16*>(d_update);
  if (grad_dtype == XMEM_BF16) return update(static_cast<const bf16*>(d_grad), d_momentum, h, mu, nesterov, steps, scale, out, d_workspace, st);
  if (grad_dtype == XMEM_F16) return update(static_cast<const f16*>(d_grad), d_momentum, h, mu, nesterov, steps, scale, out, d_workspace, st);
  return update(static_cast<const float*>(d_grad), d_momentum, h, mu, nesterov, steps, scale, out, d_workspace, st);
}

}  // extern "C"
