// clip.hip -- the norm of many gradients as one vector, and their scaling, on MI355X (gfx950).
//
// norm = scale sqrt(sum g^2), g <- scale min(1, max_norm / (norm + 1e-6)) g.  The gradients' places and sizes travel as kernel arguments, kTable of
// them a launch: nothing is copied to the device, and a captured graph holds them.  Squares are added up in 64 bits (their range
// is no matter then, and 64-bit products cost nothing beside the memory), in a fixed order: each workgroup's share, then every workgroup of the
// scaling adds up all shares for itself, which saves a launch between the two.  A gradient is looked at from the 16-byte boundary
// before it, so that its loads are aligned wherever it begins.
//
// Bound by memory: the norm has to be known before the first gradient is written, so all are read twice.  147 gradients of 2.03 GB:
// squares 360 to 384 us by the card (5.3 to 5.6 TB/s), scaling 747 to 761 (4.05 GB, 5.4 TB/s).  The scaling begins with the last gradients,
// which the caches may still hold; with the first ones 8 us more.  27 gradients of 5 MB take 4.6 and 7.2; 425 MB in float32 96 and 129.
#include <math.h>

#include <algorithm>
#include <vector>

#include "rows.h"

using namespace xops;

namespace {

constexpr int kTable = 128;          // gradients of a launch: two a lane
constexpr int kThreads = 256;
constexpr int kParts = 2048;         // workgroups of a norm at most, each with a sum of its own (425 MB in float32, partly in the caches, 70 us; with 1024 82)
constexpr int kLoads = 4;            // of 16 bytes, a thread and piece of work
constexpr int kSpan = kThreads * kLoads * 16;  // bytes of a piece of work
constexpr int64_t kMostSize = int64_t(1) << 48;

// What a launch works on.  A gradient's pieces of work begin at the 16-byte boundary at or before it.
struct Table {
  void* at[kTable];
  int64_t size[kTable];  // elements
  int64_t first[kTable + 1];  // pieces of work before the gradient's
  unsigned char type[kTable];
  int count;
};
static_assert(sizeof(Table) < 3584);

__host__ __device__ inline int bytes_of(int type) { return type == XMEM_F32 ? 4 : 2; }

// The gradient that piece of work w is of: every lane holds two of the table's ends.
struct Finder {
  int64_t end[2];
  __device__ explicit Finder(const Table& t) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < 2; ++k) end[k] = 64 * k + lane < t.count ? t.first[64 * k + lane + 1] : INT64_MAX;
  }
  __device__ int of(int64_t w) const {
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(end[0] <= w)) + __popcll(__ballot(end[1] <= w)));
  }
};

// Calls f with each 16 bytes of a piece of work: where they lie, which of their elements are the gradient's.
template <class T, class F>
__device__ inline void pieces(const Table& t, int i, int64_t w, const F& f) {
  constexpr int E = kPiece<T>;
  const uintptr_t at = reinterpret_cast<uintptr_t>(t.at[i]);
  const int head = int(at & 15) / int(sizeof(T));  // elements between the boundary and the gradient
  T* base = reinterpret_cast<T*>(at & ~uintptr_t(15));
  const int64_t n = head + t.size[i], p0 = (w - t.first[i]) * (kThreads * kLoads);
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int64_t e = (p0 + j * kThreads + threadIdx.x) * E;
    if (e < n) f(base + e, e < head ? int(head - e) : 0, n - e < E ? int(n - e) : E, j);
  }
}

template <class T>
__device__ inline u32x4 some(const T* p, int from, int to) {
  constexpr int E = kPiece<T>;
  u32x4 c;
  if (from == 0 && to == E) {
    c = *reinterpret_cast<const u32x4*>(p);
  } else {
    T e[E];
#pragma unroll
    for (int k = 0; k < E; ++k) e[k] = k >= from && k < to ? p[k] : T(0.0f);
    __builtin_memcpy(&c, e, 16);
  }
  return c;
}

template <class T>
__device__ inline double squares_of(const Table& t, int i, int64_t w) {
  u32x4 c[kLoads] = {};
  pieces<T>(t, i, w, [&](const T* p, int from, int to, int j) { c[j] = some(p, from, to); });
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    float v[kPiece<T>];
    unpack<T>(c[j], v);
#pragma unroll
    for (int k = 0; k < kPiece<T>; ++k) s = fma(double(v[k]), double(v[k]), s);
  }
  return s;
}

__device__ inline double block_sum(double v) {
  __shared__ double meet[kThreads / kWave];
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = v;
  __syncthreads();
  v = meet[0];
#pragma unroll
  for (int i = 1; i < kThreads / kWave; ++i) v += meet[i];
  return v;
}

// Each workgroup's share of the squares, added to what it has of the launches before.
__global__ __launch_bounds__(kThreads) void k_squares(Table t, bool first, double* part) {
  const Finder find(t);
  const int64_t all = t.first[t.count];
  double s = 0.0;
  for (int64_t w = blockIdx.x; w < all; w += gridDim.x) {
    const int i = find.of(w);
    s += t.type[i] == XMEM_BF16 ? squares_of<bf16>(t, i, w) : t.type[i] == XMEM_F16 ? squares_of<f16>(t, i, w) : squares_of<float>(t, i, w);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) part[blockIdx.x] = first ? s : part[blockIdx.x] + s;
}

// norm and factor from the shares, every workgroup for itself
__device__ inline float factor_of(const double* part, int parts, float max_norm, float scale, float* stats) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
  const double norm = double(scale) * sqrt(block_sum(s)), cut = double(max_norm) / (norm + 1e-6);
  // NaN stays NaN; an infinite norm under an infinite limit is no reason to clip
  const double factor = max_norm == INFINITY || cut > 1.0 ? double(scale) : double(scale) * cut;
  const float f = norm != norm ? float(norm) : float(factor);
  if (stats && blockIdx.x == 0 && threadIdx.x == 0) {
    stats[0] = float(norm);
    stats[1] = f;
  }
  return f;
}

template <class T>
__device__ inline void scale_of(const Table& t, int i, int64_t w, float f) {
  constexpr int E = kPiece<T>;
  u32x4 c[kLoads] = {};
  pieces<T>(t, i, w, [&](const T* p, int from, int to, int j) { c[j] = some(p, from, to); });
  pieces<T>(t, i, w, [&](T* p, int from, int to, int j) {
    float v[E];
    unpack<T>(c[j], v);
    T e[E];
#pragma unroll
    for (int k = 0; k < E; ++k) e[k] = T(f * v[k]);
    if (from == 0 && to == E) {
      u32x4 q;
      __builtin_memcpy(&q, e, 16);
      *reinterpret_cast<u32x4*>(p) = q;
    } else {
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (k >= from && k < to) p[k] = e[k];
    }
  });
}

__global__ __launch_bounds__(kThreads) void k_scale(Table t, const double* part, int parts, float max_norm, float scale, float* stats) {
  const float f = factor_of(part, parts, max_norm, scale, stats);
  if (f == 1.0f) return;
  const Finder find(t);
  for (int64_t w = t.first[t.count] - 1 - blockIdx.x; w >= 0; w -= gridDim.x) {
    const int i = find.of(w);
    if (t.type[i] == XMEM_BF16)
      scale_of<bf16>(t, i, w, f);
    else if (t.type[i] == XMEM_F16)
      scale_of<f16>(t, i, w, f);
    else
      scale_of<float>(t, i, w, f);
  }
}

__global__ __launch_bounds__(kThreads) void k_stats(const double* part, int parts, float scale, float* stats) {
  factor_of(part, parts, INFINITY, scale, stats);
}

int64_t pieces_of(const void* at, int64_t size, int dtype) {
  return (int64_t(reinterpret_cast<uintptr_t>(at) & 15) + size * bytes_of(dtype) + kSpan - 1) / kSpan;
}

// A launch's gradients, from the list's `at`-th on; empty ones are left out.
Table table_of(void* const* tensors, const int64_t* sizes, const int* dtypes, int64_t count, int64_t at) {
  Table t;
  t.count = 0;
  t.first[0] = 0;
  for (; at < count && t.count < kTable; ++at) {
    if (sizes[at] == 0) continue;
    const int i = t.count++;
    t.at[i] = tensors[at];
    t.size[i] = sizes[at];
    t.type[i] = static_cast<unsigned char>(dtypes[at]);
    t.first[i + 1] = t.first[i] + pieces_of(tensors[at], sizes[at], dtypes[at]);
  }
  return t;
}

bool overlap(void* const* tensors, const int64_t* sizes, const int* dtypes, int64_t count) {
  typedef std::pair<uintptr_t, uintptr_t> Range;
  std::vector<Range> all;
  all.reserve(size_t(count));
  for (int64_t i = 0; i < count; ++i)
    if (sizes[i] > 0) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(tensors[i]);
      all.emplace_back(at, at + uintptr_t(sizes[i]) * bytes_of(dtypes[i]));
    }
  std::sort(all.begin(), all.end());
  for (size_t i = 1; i < all.size(); ++i)
    if (all[i].first < all[i - 1].second) return true;
  return false;
}

}  // namespace

extern "C" {

size_t xmem_clip_grad_norm_workspace_bytes(void) { return kParts * sizeof(double); }

int xmem_clip_grad_norm(void* const* d_tensors, const int64_t* sizes, const int* dtypes, int64_t count, float max_norm, float scale,
                        float* d_stats, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (count < 0 || count >= kMostRows || (count > 0 && (!d_tensors || !sizes || !dtypes)) || !d_stats) return XMEM_EINVAL;
  if (!(max_norm >= 0.0f) || !(scale >= 0.0f) || scale == INFINITY) return XMEM_EINVAL;
  for (int64_t i = 0; i < count; ++i)
    if (sizes[i] < 0 || sizes[i] >= kMostSize || !type_ok(dtypes[i]) || (sizes[i] > 0 && !d_tensors[i]) ||
        reinterpret_cast<uintptr_t>(d_tensors[i]) % bytes_of(dtypes[i]))
      return XMEM_EINVAL;
  const bool writes = max_norm != INFINITY || scale != 1.0f;
  struct Launch {
    int64_t start, pieces;  // its first gradient, its pieces of work
  };
  std::vector<Launch> launches;
  int64_t parts = 1;
  try {
    if (writes && overlap(d_tensors, sizes, dtypes, count)) return XMEM_EINVAL;
    for (int64_t at = 0; at < count || launches.empty();) {
      Launch next{at, 0};
      for (int taken = 0; at < count && taken < kTable; ++at)
        if (sizes[at] > 0) {
          next.pieces += pieces_of(d_tensors[at], sizes[at], dtypes[at]);
          ++taken;
        }
      launches.push_back(next);
      parts = std::max(parts, std::min(next.pieces, int64_t(kParts)));
    }
  } catch (...) {  // no memory on the host
    return XMEM_EINVAL;
  }
  const size_t need = xmem_clip_grad_norm_workspace_bytes();
  if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256)) return XMEM_EWORKSPACE;
  if (shares(d_workspace, need, d_stats, 1, 2, 2, 4)) return XMEM_EINVAL;
  for (int64_t i = 0; i < count; ++i)
    if (sizes[i] > 0 && shares(d_workspace, need, d_tensors[i], 1, sizes[i], sizes[i], bytes_of(dtypes[i]))) return XMEM_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  double* part = static_cast<double*>(d_workspace);
  const auto table = [&](size_t i) { return table_of(d_tensors, sizes, dtypes, count, launches[i].start); };
  for (size_t i = 0; i < launches.size(); ++i) k_squares<<<unsigned(parts), kThreads, 0, st>>>(table(i), i == 0, part);
  if (!writes) {
    k_stats<<<1, kThreads, 0, st>>>(part, int(parts), scale, d_stats);
    return launched();
  }
  // the last gradients first, which the caches may still hold
  for (size_t i = launches.size(); i-- > 0;) {
    const int64_t grid = std::max(int64_t(1), std::min(launches[i].pieces, int64_t(kParts)));
    k_scale<<<unsigned(grid), kThreads, 0, st>>>(table(i), part, int(parts), max_norm, scale, i == 0 ? d_stats : nullptr);
  }
  return launched();
}

}  // extern "C"
