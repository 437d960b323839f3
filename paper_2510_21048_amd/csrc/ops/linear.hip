// linear.hip -- y = act(x w^T + b) + r and its gradients on MI355X (gfx950).
//
//   z = x w^T + b, y = act(z) + r          one product, its epilogue (gemm.h); z is written where the backward pass wants it
//   dz = dy act'(z), db = sum over m dz    k_dz: one pass over dy and z, column sums of bands of rows; k_db adds the bands
//   dx = dz w, dw = dz^T x                 two products, either operand as it lies
//
// dz is rounded to 16 bits, as the matrix instructions take it (the products' outputs are rounded to as many: 1.4 times
// their error without); db sums it before that.  No sum's order depends on when a workgroup runs.
// 8192 x 8192 x 2048 with gelu and z: 262 to 282 us by the card (975 to 1,050 TFLOP/s; its 268 MB of outputs alone take 55 at a
// large copy's rate); the gradients 572 to 615 us, of which k_dz 88 (402 MB at 4.6 TB/s).  32768 x 4096 x 16384 with a residual: 3.4 ms.
// One token through 4096 x 1024: 8.5 us.
#include "gemm.h"

using namespace xops;

namespace {

constexpr float kGelu = 0.7978845608028654f, kCube = 0.044715f;  // sqrt(2 / pi)

// (1 + tanh(u)) / 2 is the logistic function of 2u, without a difference of near numbers: gelu(z) = z s(2u), as
// silu(z) = z s(z).  exp and 1/x are the hardware's; 1/x is good to 2^-22 of its value, exp(v) to |v| 2^-24 more, since
// v log2(e) is rounded before the power of two (2^-18 at v = 80, where the logistic function is next to nothing).
__device__ inline float logistic(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }
__device__ inline float gelu_argument(float z) { return z * (2.0f * kGelu + (2.0f * kGelu * kCube) * (z * z)); }

__device__ inline float activate(float z, int act) {
  if (act == XMEM_ACT_RELU) return z < 0.0f ? 0.0f : z;  // NaN stays
  if (act == XMEM_ACT_GELU) return z * logistic(gelu_argument(z));
  if (act == XMEM_ACT_SILU) return z * logistic(z);
  return z;
}

__device__ inline float slope(float z, int act) {
  if (act == XMEM_ACT_RELU) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
  if (act == XMEM_ACT_GELU) {
    const float s = logistic(gelu_argument(z)), w = s * (1.0f - s);  // 0 where the cube overflows
    return w == 0.0f ? s : s + z * w * (2.0f * kGelu + (6.0f * kGelu * kCube) * (z * z));
  }
  if (act == XMEM_ACT_SILU) {
    const float s = logistic(z), w = s * (1.0f - s);
    return w == 0.0f ? s : s + z * w;
  }
  return 1.0f;
}

// ACT < 0: the activation is `act`.
template <class T, int ACT = -1>
struct LinearEpilogue {
  static constexpr bool kSymmetric = false, kPastL2 = true, kAnyRows = true;
  const float* bias;
  const T* r;
  T* y;
  T* z;
  int64_t ldr, ldy, ldz;
  int act;

  bool lines() const { return whole_lines(y, ldy) && whole_lines(z, ldz); }
  template <class F>
  __device__ __attribute__((always_inline)) void chosen(F f) const {
    if (act == XMEM_ACT_GELU)
      f(LinearEpilogue<T, XMEM_ACT_GELU>{bias, r, y, z, ldr, ldy, ldz, act});
    else if (act == XMEM_ACT_SILU)
      f(LinearEpilogue<T, XMEM_ACT_SILU>{bias, r, y, z, ldr, ldy, ldz, act});
    else if (act == XMEM_ACT_RELU)
      f(LinearEpilogue<T, XMEM_ACT_RELU>{bias, r, y, z, ldr, ldy, ldz, act});
    else
      f(LinearEpilogue<T, XMEM_ACT_NONE>{bias, r, y, z, ldr, ldy, ldz, act});
  }
  template <int W>
  __device__ Column<W> column(int64_t n, int valid, int, const GemmArgs&) const {
    Column<W> c;
#pragma unroll
    for (int j = 0; j < W; ++j) c.v[j] = bias && j < valid ? bias[n + j] : 0.0f;
    return c;
  }
  template <int W>
  struct Read {  // of the residual, as it lies: half the registers
    T v[W];
  };
  template <int W>
  __device__ Read<W> read(int64_t m, int64_t n, int valid, int, const GemmArgs&) const {
    Read<W> e;
    if (!r) return e;
    if (valid == W) {
      __builtin_memcpy(e.v, r + m * ldr + n, sizeof(e.v));
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) e.v[j] = j < valid ? r[m * ldr + n + j] : T(0.0f);
    }
    return e;
  }
  template <int W, class HOW>
  __device__ void row(int64_t m, int64_t n, float (&v)[W], int valid, const Column<W>& c, const Read<W>& e, int, const GemmArgs&) const {
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] += c.v[j];
    if (z) put<T, W, HOW>(z + m * ldz + n, valid, v);
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = activate(v[j], ACT < 0 ? act : ACT);
    if (r)
#pragma unroll
      for (int j = 0; j < W; ++j) v[j] += float(e.v[j]);
    put<T, W, HOW>(y + m * ldy + n, valid, v);
  }
};

template <class T>
struct StoreEpilogue {
  static constexpr bool kSymmetric = false, kPastL2 = true, kAnyRows = true;
  T* y;
  int64_t ldy;

  bool lines() const { return whole_lines(y, ldy); }
  template <class F>
  __device__ __attribute__((always_inline)) void chosen(F f) const { f(*this); }
  template <int W> using Read = None;
  template <int W>
  __device__ None column(int64_t, int, int, const GemmArgs&) const { return {}; }
  template <int W>
  __device__ None read(int64_t, int64_t, int, int, const GemmArgs&) const { return {}; }
  template <int W, class HOW>
  __device__ void row(int64_t m, int64_t n, float (&v)[W], int valid, None, None, int, const GemmArgs&) const {
    put<T, W, HOW>(y + m * ldy + n, valid, v);
  }
};

constexpr int kBandCols = 512;  // columns of a workgroup of k_dz, eight a lane

// Rows whose column sums one workgroup of k_dz takes: 64, or 16 where that makes fewer than four workgroups a CU (128 are a third
// slower there, and 2 to 8% faster only from 4,096 workgroups of 64 on).  us with db and, with gelu, dw of 8 columns, 16 rows and 64: 128 x 4096 21.4 and 24.9, 2048 x 4096 29.3 and
// 41.3, 4096 x 4096 38.6 and 50.4, 8192 x 4096 (1,024 workgroups of 64) 61.2 and 61.5, 8192 x 8192 130.5 and 122.8.
inline int64_t band_rows(int64_t m, int64_t n) { return (m + 63) / 64 * ((n + kBandCols - 1) / kBandCols) < 4 * kCus ? 16 : 64; }
inline int64_t bands(int64_t m, int64_t n) { return (m + band_rows(m, n) - 1) / band_rows(m, n); }

// Whether a matrix of `cols` columns is copied to rows of 16 bytes' alignment before a product of m n k multiplications: the
// copy costs a launch and a pass over it.  float16, with the copies and without: 501 x 1023 x 511 13.6 and 9.0 us,
// 1003 x 2047 x 1021 (2.1e9) 21.1 and 17.2, 1601 x 1603 x 1605 (4.1e9) 30.1 and 30.8, 4099 x 4097 x 4095 221 and 303.
constexpr double kPackFrom = 4.0e9;
inline bool packs(int64_t cols, int64_t ld, int64_t m, int64_t n, int64_t k) {
  return (cols % 8 || ld % 8) && double(m) * double(n) * double(k) >= kPackFrom;
}
inline size_t packed_bytes(int64_t rows, int64_t cols) { return up256(size_t(rows) * packed_ld(cols) * 2); }
inline size_t sums_bytes(int64_t m, int64_t n) { return up256(size_t(bands(m, n)) * n * 4); }
// dz is kept where it is not dy, or dy's rows allow no 16-byte loads
inline bool keeps_dz(int64_t m, int64_t n, int64_t k, int64_t lddy, int act) { return act != XMEM_ACT_NONE || packs(n, lddy, m, n, k); }

// dz = dy act'(z), and the column sums of each band of rows before dz is rounded.  A wavefront takes every fourth row of
// the band, 16 bytes a lane; what pads a row of dz is 0, since the product that sums along it reads it.
template <class T, int ACT>
__global__ __launch_bounds__(256) void k_dz(const T* dy, int64_t lddy, const T* z, int64_t ldz, int64_t m, int64_t n, T* dz, int64_t lddz,
                                            float* part, int band) {
  __shared__ float sums[3][kBandCols];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = int64_t(blockIdx.x) * kBandCols + lane * 8, r0 = int64_t(blockIdx.y) * band;
  const int valid = n - c >= 8 ? 8 : n > c ? int(n - c) : 0;
  const int64_t end = m < r0 + band ? m : r0 + band;
  float sum[8] = {};
  if (valid > 0) {
#pragma unroll 2  // rows' loads on their way: 8192 x 8192 in 88 us, with four 109, with eight 106
    for (int64_t r = r0 + wave; r < end; r += 4) {
      float v[8], w[8];
      get<T, 8>(dy + r * lddy + c, valid, v);
      if constexpr (ACT != XMEM_ACT_NONE) {
        get<T, 8>(z + r * ldz + c, valid, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= slope(w[j], ACT);
      }
      if (dz) {
        if (valid < 8)  // where z is read as 0 past the end, dy is too
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = j < valid ? v[j] : 0.0f;
        put<T, 8, Any>(dz + r * lddz + c, 8, v);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[j];
    }
  }
  if (!part) return;
  if (wave > 0)
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[wave - 1][lane * 8 + j] = sum[j];
  __syncthreads();
  if (wave == 0)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j < valid) part[int64_t(blockIdx.y) * n + c + j] = ((sum[j] + sums[0][lane * 8 + j]) + sums[1][lane * 8 + j]) + sums[2][lane * 8 + j];
    }
}

// The bands' sums of the columns from `first` on, 16 runs of bands to a column and those in order.
__global__ __launch_bounds__(1024) void k_db(const float* part, int64_t nb, int64_t first, int64_t n, float* db) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = first + int64_t(blockIdx.x) * 64 + lane;
  float sum = 0.0f;
  if (c < n)
#pragma unroll 8
    for (int64_t b = wave; b < nb; b += 16) sum += part[b * n + c];
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave > 0 || c >= n) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) sum += sums[i][lane];
  db[c] = sum;
}

constexpr int64_t kMostSize = int64_t(1) << 30;
constexpr int64_t kMostLd = int64_t(1) << 40;

bool sizes_ok(int64_t m, int64_t n, int64_t k) {
  return m >= 0 && n >= 0 && k >= 0 && m < kMostSize && n < kMostSize && k < kMostSize &&
         ((m + 63) / 64) * ((n + 63) / 64) < kMostSize && ((m + 63) / 64) * ((k + 63) / 64) < kMostSize &&
         ((n + 63) / 64) * ((k + 63) / 64) < kMostSize;
}
bool ld_ok(int64_t ld, int64_t cols) { return ld >= cols && ld < kMostLd; }

// The workspace, part after part.
struct Carve {
  char* at;
  template <class P>
  P* take(size_t bytes) {
    char* r = at;
    at += bytes;
    return reinterpret_cast<P*>(r);
  }
};

size_t forward_bytes(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
  return (packs(k, ldx, m, n, k) ? packed_bytes(m, k) : 0) + (packs(k, ldw, m, n, k) ? packed_bytes(n, k) : 0) + part_bytes(m, n, k, 1, false);
}

template <class T>
int forward(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias, const void* r, int64_t ldr, int64_t m,
            int64_t n, int64_t k, int act, void* y, int64_t ldy, void* z, int64_t ldz, void* ws, hipStream_t st) {
  Carve at{static_cast<char*>(ws)};
  GemmArgs g{x, w, ldx, ldw, 0, 0, m, n, k};
  Pack px{}, pw{};
  if (packs(k, ldx, m, n, k)) {
    px = {x, ldx, m, k, at.take<char>(packed_bytes(m, k))};
    g.a = px.to, g.lda = packed_ld(k), g.pad_a = true;
  }
  if (packs(k, ldw, m, n, k)) {
    pw = {w, ldw, n, k, at.take<char>(packed_bytes(n, k))};
    g.b = pw.to, g.ldb = packed_ld(k), g.pad_b = true;
  }
  pack<T>(px, pw, st);
  const LinearEpilogue<T> e{bias, static_cast<const T*>(r), static_cast<T*>(y), static_cast<T*>(z), ldr, ldy, ldz, act};
  return gemm<T, true, true>(g, e, at.at, st);
}

size_t backward_bytes(int64_t m, int64_t n, int64_t k, int64_t lddy, int64_t ldx, int64_t ldw, int act) {
  const size_t sx = part_bytes(m, k, n, 1, false), sw = part_bytes(n, k, m, 1, false);
  return sums_bytes(m, n) + (keeps_dz(m, n, k, lddy, act) ? packed_bytes(m, n) : 0) + (packs(k, ldx, m, n, k) ? packed_bytes(m, k) : 0) +
         (packs(k, ldw, m, n, k) ? packed_bytes(n, k) : 0) + (sx > sw ? sx : sw);
}

template <class T>
int backward(const void* dy, int64_t lddy, const void* z, int64_t ldz, const void* x, int64_t ldx, const void* w, int64_t ldw,
             int64_t m, int64_t n, int64_t k, int act, void* dx, int64_t lddx, void* dw, int64_t lddw, float* db, void* ws,
             hipStream_t st) {
  Carve at{static_cast<char*>(ws)};
  float* part = at.take<float>(sums_bytes(m, n));
  const void* d = dy;
  int64_t ldd = lddy;
  T* dz = nullptr;
  if (keeps_dz(m, n, k, lddy, act)) {
    T* to = at.take<T>(packed_bytes(m, n));
    if (dx || dw) {
      dz = to;
      d = to;
      ldd = packed_ld(n);
    }
  }
  if ((dz || db) && m > 0 && n > 0)
    for (int64_t b0 = 0; b0 < bands(m, n); b0 += 32768) {  // grid y is at most 65535
      const int64_t r0 = b0 * band_rows(m, n), high = bands(m, n) - b0 < 32768 ? bands(m, n) - b0 : 32768;
      float* sums = !db ? nullptr : bands(m, n) == 1 ? db : part + b0 * n;
      (act == XMEM_ACT_NONE   ? k_dz<T, XMEM_ACT_NONE>
       : act == XMEM_ACT_RELU ? k_dz<T, XMEM_ACT_RELU>
       : act == XMEM_ACT_GELU ? k_dz<T, XMEM_ACT_GELU>
                              : k_dz<T, XMEM_ACT_SILU>)<<<dim3(unsigned((n + kBandCols - 1) / kBandCols), unsigned(high)), 256, 0, st>>>(
          static_cast<const T*>(dy) + r0 * lddy, lddy, z ? static_cast<const T*>(z) + r0 * ldz : nullptr, ldz, m - r0, n,
          dz ? dz + r0 * ldd : nullptr, ldd, sums, int(band_rows(m, n)));
    }
  if (db && bands(m, n) != 1)
    for (int64_t c = 0; c < n; c += kMostThreads / 1024 * 64)
      k_db<<<unsigned((n - c < kMostThreads / 1024 * 64 ? n - c + 63 : kMostThreads / 1024 * 64) / 64), 1024, 0, st>>>(part, bands(m, n), c, n, db);
  GemmArgs gx{d, w, ldd, ldw, 0, 0, m, k, n, dz != nullptr}, gw{d, x, ldd, ldx, 0, 0, n, k, m, dz != nullptr};
  Pack px{}, pw{};
  if (packs(k, ldx, m, n, k)) {
    px = {dw ? x : nullptr, ldx, m, k, at.take<char>(packed_bytes(m, k))};
    gw.b = px.to, gw.ldb = packed_ld(k), gw.pad_b = true;
  }
  if (packs(k, ldw, m, n, k)) {
    pw = {dx ? w : nullptr, ldw, n, k, at.take<char>(packed_bytes(n, k))};
    gx.b = pw.to, gx.ldb = packed_ld(k), gx.pad_b = true;
  }
  if (m > 0 && n > 0) pack<T>(px, pw, st);
  int rc = launched();
  if (rc == XMEM_OK && dx) rc = gemm<T, true, false>(gx, StoreEpilogue<T>{static_cast<T*>(dx), lddx}, at.at, st);
  if (rc == XMEM_OK && dw) rc = gemm<T, false, false>(gw, StoreEpilogue<T>{static_cast<T*>(dw), lddw}, at.at, st);
  return rc;
}

bool known(int dtype, int act) { return (dtype == XMEM_BF16 || dtype == XMEM_F16) && act >= XMEM_ACT_NONE && act <= XMEM_ACT_SILU; }

}  // namespace

extern "C" {

size_t xmem_linear_forward_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
  return sizes_ok(m, n, k) && ld_ok(ldx, k) && ld_ok(ldw, k) ? forward_bytes(m, n, k, ldx, ldw) : 0;
}

int xmem_linear_forward(const void* d_x, int64_t ldx, const void* d_w, int64_t ldw, const float* d_bias,
                        const void* d_residual, int64_t ldr, int64_t m, int64_t n, int64_t k, int dtype,
                        int activation, void* d_y, int64_t ldy, void* d_z, int64_t ldz, void* d_workspace,
                        size_t workspace_bytes, void* hip_stream) {
  if (!sizes_ok(m, n, k) || !known(dtype, activation)) return XMEM_EINVAL;
  if (!ld_ok(ldx, k) || !ld_ok(ldw, k) || !ld_ok(ldy, n) || (d_residual && !ld_ok(ldr, n)) || (d_z && !ld_ok(ldz, n)))
    return XMEM_EINVAL;
  if (m == 0 || n == 0) return XMEM_OK;
  if (!d_y || (k > 0 && (!d_x || !d_w))) return XMEM_EINVAL;
  const size_t need = forward_bytes(m, n, k, ldx, ldw);
  if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256))) return XMEM_EWORKSPACE;
  if (!need) d_workspace = nullptr;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return (dtype == XMEM_BF16 ? forward<bf16> : forward<f16>)(d_x, ldx, d_w, ldw, d_bias, d_residual, ldr, m, n, k, activation,
                                                             d_y, ldy, d_z, ldz, d_workspace, st);
}

size_t xmem_linear_backward_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t lddy, int64_t ldx, int64_t ldw, int activation) {
  return sizes_ok(m, n, k) && ld_ok(lddy, n) && ld_ok(ldx, k) && ld_ok(ldw, k) && known(XMEM_BF16, activation)
             ? backward_bytes(m, n, k, lddy, ldx, ldw, activation)
             : 0;
}

int xmem_linear_backward(const void* d_dy, int64_t lddy, const void* d_z, int64_t ldz, const void* d_x, int64_t ldx,
                         const void* d_w, int64_t ldw, int64_t m, int64_t n, int64_t k, int dtype, int activation,
                         void* d_dx, int64_t lddx, void* d_dw, int64_t lddw, float* d_db, void* d_workspace,
                         size_t workspace_bytes, void* hip_stream) {
  if (!sizes_ok(m, n, k) || !known(dtype, activation)) return XMEM_EINVAL;
  if (activation == XMEM_ACT_NONE) d_z = nullptr;  // its slope is 1 everywhere
  if (!ld_ok(lddy, n) || (d_z && !ld_ok(ldz, n)) || !ld_ok(ldx, k) || !ld_ok(ldw, k) ||
      (d_dx && !ld_ok(lddx, k)) || (d_dw && !ld_ok(lddw, k)))
    return XMEM_EINVAL;
  if (!d_dx && !d_dw && !d_db) return XMEM_OK;
  if (m > 0 && n > 0) {
    if (!d_dy || (activation != XMEM_ACT_NONE && !d_z)) return XMEM_EINVAL;
    if (k > 0 && ((d_dx && !d_w) || (d_dw && !d_x))) return XMEM_EINVAL;
  }
  const size_t need = backward_bytes(m, n, k, lddy, ldx, ldw, activation);
  if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256))) return XMEM_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return (dtype == XMEM_BF16 ? backward<bf16> : backward<f16>)(d_dy, lddy, d_z, ldz, d_x, ldx, d_w, ldw, m, n, k, activation,
                                                               d_dx, lddx, d_dw, lddw, d_db, d_workspace, st);
}

}  // extern "C"
