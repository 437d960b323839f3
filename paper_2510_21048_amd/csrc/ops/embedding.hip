// embedding.hip -- scaled rows of a table, and the table's gradient, on MI355X (gfx950).
#include "rows.h"

using namespace xops;

namespace {

struct Lookup {
  const void* table;
  int64_t ldt;
  const int64_t* ids;
  int64_t t, vocab, n;
  float scale;
  int64_t padding;
  void* y;
  int64_t ldy;
  int lanes;  // of a row, a power of two: 64 / lanes rows a wavefront
  int64_t first = 0;  // workgroup of the launch
};

constexpr int kSlab = 4;  // pieces a lane

// A wavefront takes 64 / lanes rows, or one of more pieces than its lanes hold: lanes * kSlab of them at a time, which blockIdx.y counts.
template <class T>
__global__ __launch_bounds__(256) void k_lookup(Lookup p) {
  constexpr int E = kPiece<T>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = ((p.first + blockIdx.x) * 4 + wave) * (64 / p.lanes) + lane / p.lanes;
  if (t >= p.t) return;
  const int64_t id = p.ids[t], pieces = (p.n + E - 1) / E;
  const bool in = id >= 0 && id < p.vocab && id != p.padding;
  const T* row = static_cast<const T*>(p.table) + (in ? id : 0) * p.ldt;
  T* y = static_cast<T*>(p.y) + t * p.ldy;
  for (int64_t i0 = int64_t(blockIdx.y) * (64 * kSlab) + lane % p.lanes; i0 < pieces; i0 += int64_t(gridDim.y) * (64 * kSlab)) {
    u32x4 c[kSlab];
#pragma unroll
    for (int j = 0; j < kSlab; ++j) {
      const int64_t i = i0 + j * p.lanes;
      c[j] = in && i < pieces ? piece_of(row, i, p.n) : u32x4{};
    }
#pragma unroll
    for (int j = 0; j < kSlab; ++j) {
      const int64_t i = i0 + j * p.lanes;
      if (i < pieces) {
        float v[E];
        unpack<T>(c[j], v);
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = in ? p.scale * v[k] : id == p.padding ? 0.0f : NAN;
        put_piece(y, i, p.n, v);
      }
    }
  }
}

template <class T>
int launch_lookup(Lookup p, hipStream_t st) {
  const int64_t pieces = (p.n + kPiece<T> - 1) / kPiece<T>;
  p.lanes = 1;
  while (p.lanes < 64 && p.lanes * kSlab < pieces) p.lanes *= 2;
  const int64_t all = (pieces + 64 * kSlab - 1) / (64 * kSlab), slabs = all < 4096 ? all : 4096;
  const int64_t rows = 4 * (64 / p.lanes), blocks = (p.t + rows - 1) / rows, wide = kMostThreads / 256 / slabs;
  for (; p.first < blocks; p.first += wide)
    k_lookup<T><<<dim3(unsigned(blocks - p.first < wide ? blocks - p.first : wide), unsigned(slabs)), 256, 0, st>>>(p);
  return launched();
}

// ------------------------------------------------------------------ gradient

struct TableGrad {
  const void* dy;
  int64_t lddy;
  const int64_t* ids;
  int64_t t, vocab, n;
  float scale;
  int64_t padding;
  bool add;
  void* out;
  int64_t ldd;
};

constexpr int kIds = 1024;  // tokens looked at together

// A wavefront has one row of the table, 64 pieces of it at a time, and looks at every token.
template <class T, class O>
__global__ __launch_bounds__(256) void k_scan(TableGrad p) {
  constexpr int E = kPiece<T>;
  __shared__ int ids[kIds];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t slabs = (p.n + 64 * E - 1) / (64 * E), rows = (p.vocab + 3) / 4;
  for (int64_t item = blockIdx.x; item < rows * slabs; item += gridDim.x) {
    const int64_t v = item / slabs * 4 + wave, i = item % slabs * 64 + lane;
    float sum[E] = {};
    bool any = false;
    for (int64_t t0 = 0; t0 < p.t; t0 += kIds) {
      __syncthreads();
      for (int k = threadIdx.x; k < kIds; k += 256) {
        const int64_t id = t0 + k < p.t ? p.ids[t0 + k] : -1;
        ids[k] = id >= 0 && id < p.vocab && id != p.padding ? int(id) : -1;
      }
      __syncthreads();
      for (int k = 0; k < kIds && t0 + k < p.t; k += 64) {
        uint64_t hit = __ballot(ids[k + lane] == int(v));
        any = any || hit;
        while (hit) {
          const int at = __builtin_ctzll(hit);
          hit &= hit - 1;
          float g[E];
          unpack<T>(piece_of(static_cast<const T*>(p.dy) + (t0 + k + at) * p.lddy, i, p.n), g);
#pragma unroll
          for (int q = 0; q < E; ++q) sum[q] += g[q];
        }
      }
    }
    if (v >= p.vocab || (p.add && !any)) continue;
    O* out = static_cast<O*>(p.out) + v * p.ldd;
    O e[E];
#pragma unroll
    for (int q = 0; q < E; ++q) {
      float s = p.scale * sum[q];
      if (p.add && i * E + q < p.n) s += float(out[i * E + q]);
      e[q] = O(s);
    }
    if ((i + 1) * E <= p.n) {
      __builtin_memcpy(out + i * E, e, sizeof(e));
    } else {
#pragma unroll
      for (int q = 0; q < E; ++q)
        if (i * E + q < p.n) out[i * E + q] = e[q];
    }
  }
}

template <class T, class O>
int launch_grad(const TableGrad& p, hipStream_t st) {
  const int64_t items = (p.vocab + 3) / 4 * ((p.n + 64 * kPiece<T> - 1) / (64 * kPiece<T>)), most = 1 << 20;
  k_scan<T, O><<<unsigned(items < most ? items : most), 256, 0, st>>>(p);
  return launched();
}

bool sizes_ok(int64_t t, int64_t vocab, int64_t n) {
  return t >= 0 && t < kMostRows && vocab >= 1 && vocab < kMostRows && n >= 1 && n < kMostRows;
}

}  // namespace

extern "C" {

int xmem_embedding_forward(const void* d_table, int64_t ldt, const int64_t* d_ids, int64_t tokens, int64_t vocab, int64_t width,
                           int dtype, float scale, int64_t padding_id, void* d_y, int64_t ldy, void* hip_stream) {
  if (!sizes_ok(tokens, vocab, width) || !type_ok(dtype) || !ld_ok(ldt, width) || !ld_ok(ldy, width)) return XMEM_EINVAL;
  if (tokens == 0) return XMEM_OK;
  if (!d_table || !d_ids || !d_y) return XMEM_EINVAL;
  const Lookup p{d_table, ldt, d_ids, tokens, vocab, width, scale, padding_id, d_y, ldy, 1};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return (dtype == XMEM_BF16 ? launch_lookup<bf16> : dtype == XMEM_F16 ? launch_lookup<f16> : launch_lookup<float>)(p, st);
}

size_t xmem_embedding_backward_workspace_bytes(int64_t tokens, int64_t vocab, int64_t width) {
  return 0;
}

int xmem_embedding_backward(const void* d_dy, int64_t lddy, const int64_t* d_ids, int64_t tokens, int64_t vocab, int64_t width,
                            int dtype, float scale, int64_t padding_id, int add, int out_dtype, void* d_dtable, int64_t ldd,
                            void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (!sizes_ok(tokens, vocab, width) || !type_ok(dtype) || (out_dtype != dtype && out_dtype != XMEM_F32)) return XMEM_EINVAL;
  if (!ld_ok(lddy, width) || !ld_ok(ldd, width)) return XMEM_EINVAL;
  if (tokens == 0 && add) return XMEM_OK;
  if (!d_dtable || (tokens > 0 && (!d_dy || !d_ids))) return XMEM_EINVAL;
  if (workspace_bytes < xmem_embedding_backward_workspace_bytes(tokens, vocab, width) || !aligned(d_workspace, 256)) return XMEM_EWORKSPACE;
  const TableGrad p{d_dy, lddy, d_ids, tokens, vocab, width, scale, padding_id, add != 0, d_dtable, ldd};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (dtype == XMEM_F32) return launch_grad<float, float>(p, st);
  if (out_dtype == XMEM_F32) return (dtype == XMEM_BF16 ? launch_grad<bf16, float> : launch_grad<f16, float>)(p, st);
  return (dtype == XMEM_BF16 ? launch_grad<bf16, bf16> : launch_grad<f16, f16>)(p, st);
}

}  // extern "C"
