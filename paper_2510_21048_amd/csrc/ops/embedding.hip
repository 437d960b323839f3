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

// ---- many tokens: grouped by row first

// Rows are spread over groups of kKeys or fewer by a multiplication: key = id * mul mod 2^bits, of which the upper bits are
// the group, so that frequent tokens (whose numbers are often neighbours) do not meet in one.
constexpr int kGroups = 256, kKeys = 1024, kWaves = 16;
constexpr int kRun = 32;  // entries of the sorted list that one wavefront adds up

struct Groups {
  int bits, low;  // of a key, and of its place in the group
  unsigned mul, inverse;
  int64_t count() const { return int64_t(1) << (bits - low); }
  __host__ __device__ unsigned key(unsigned id) const { return (id * mul) & mask(); }
  __host__ __device__ unsigned id(unsigned key) const { return (key * inverse) & mask(); }
  __host__ __device__ unsigned mask() const { return (1u << bits) - 1; }
};
Groups groups_of(int64_t vocab) {
  Groups g{0, 0, 0, 0};
  while ((int64_t(1) << g.bits) < vocab) ++g.bits;
  g.mul = unsigned(0.6180339887 * double(int64_t(1) << g.bits)) | 1;
  g.inverse = 1;
  for (int i = 0; i < 5; ++i) g.inverse *= 2 - g.mul * g.inverse;  // twice the bits a step
  while ((int64_t(1) << (g.bits - g.low)) > kGroups && (1 << g.low) < kKeys) ++g.low;
  return g;
}

struct Lists {
  int *token, *row;  // sorted: tokens of one row together and in their order
  int* count;        // entries
  int* state;        // of a run of kRun entries, see k_sum
  float* part;       // two rows a run
  size_t bytes;
};
Lists carve(void* base, int64_t t, int64_t n) {
  Lists w;
  char* at = static_cast<char*>(base);
  const auto take = [&](size_t b) {
    char* r = at;
    at += up256(b);
    return r;
  };
  const int64_t runs = (t + kRun - 1) / kRun;
  w.token = reinterpret_cast<int*>(take(size_t(t) * 4));
  w.row = reinterpret_cast<int*>(take(size_t(t) * 4));
  w.count = reinterpret_cast<int*>(take(4));
  w.state = reinterpret_cast<int*>(take(size_t(runs) * 4));
  w.part = reinterpret_cast<float*>(take(size_t(runs) * 2 * size_t(n) * 4));
  w.bytes = size_t(at - static_cast<char*>(base));
  return w;
}

// A workgroup has the rows of one group.  It looks at every token twice, each wavefront at a sixteenth of them in order: first it
// counts its own rows' and those of the groups before, then it puts its own where these counts say.  Rows without a token are cleared.
template <class O>
__global__ __launch_bounds__(kWaves * 64) void k_group(TableGrad p, Groups groups, Lists lists) {
  __shared__ int hist[kWaves][kKeys], meet[kWaves][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int keys = 1 << groups.low;
  const unsigned mine = blockIdx.x;
  for (int i = threadIdx.x; i < kWaves * keys; i += kWaves * 64) hist[i / keys][i % keys] = 0;
  __syncthreads();
  const int64_t share = ((p.t + kWaves - 1) / kWaves + 63) / 64 * 64, from = wave * share, to = from + share < p.t ? from + share : p.t;
  // the key, or all bits where the token adds nothing
  const auto key_at = [&](int64_t i) {
    const int64_t id = i < to ? p.ids[i] : -1;
    return id >= 0 && id < p.vocab && id != p.padding ? groups.key(unsigned(id)) : ~0u;
  };
  int before = 0, all = 0;
#pragma unroll 8
  for (int64_t i = from + lane; i < to; i += 64) {
    const unsigned key = key_at(i);
    const unsigned group = key == ~0u ? ~0u : key >> groups.low;
    before += group < mine;
    all += key != ~0u;
    if (group == mine) atomicAdd(&hist[wave][key & (keys - 1)], 1);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    before += __shfl_xor(before, d);
    all += __shfl_xor(all, d);
  }
  if (lane == 0) {
    meet[wave][0] = before;
    meet[wave][1] = all;
  }
  __syncthreads();
  int base = 0, count = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    base += meet[w][0];
    count += meet[w][1];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *lists.count = count;
  // the places of a row's tokens: behind those of the group's rows before it, a wavefront's behind the earlier ones'
  __shared__ int sums[kWaves];
  int own = 0;
  if (int(threadIdx.x) < keys)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) own += hist[w][threadIdx.x];
  int place = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(place, d);
    if (lane >= d) place += up;
  }
  if (lane == 63) sums[wave] = place;
  __syncthreads();
  for (int w = 0; w < wave; ++w) place += sums[w];
  place += base - own;
  if (int(threadIdx.x) < keys)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = hist[w][threadIdx.x];
      hist[w][threadIdx.x] = place;
      place += c;
    }
  const bool empty = int(threadIdx.x) < keys && own == 0;
  __syncthreads();
#pragma unroll 4
  for (int64_t i0 = from; i0 < to; i0 += 64) {
    const unsigned key = key_at(i0 + lane);
    const int local = int(key & (keys - 1));
    uint64_t left = __ballot(key != ~0u && (key >> groups.low) == mine);
    while (left) {
      const int leader = __builtin_ctzll(left);
      const uint64_t same = left & __ballot(local == __shfl(local, leader));
      int at = 0;
      if (lane == leader) at = atomicAdd(&hist[wave][local], __popcll(same));
      at = __shfl(at, leader) + __popcll(same & ((uint64_t(1) << lane) - 1));
      if (same >> lane & 1) {
        lists.token[at] = int(i0 + lane);
        lists.row[at] = int(groups.id(key));
      }
      left &= ~same;
    }
  }
  if (p.add) return;
  // a wavefront clears the rows of its 64 threads' keys
  uint64_t clear = __ballot(empty && groups.id((mine << groups.low) + threadIdx.x) < unsigned(p.vocab));
  __shared__ uint64_t cleared[kWaves];
  if (lane == 0) cleared[wave] = clear;
  __syncthreads();
  int turn = 0;
  for (int w = 0; w < kWaves; ++w) {
    clear = cleared[w];
    while (clear) {
      const int k = __builtin_ctzll(clear);
      clear &= clear - 1;
      if (turn++ % kWaves != wave) continue;
      O* out = static_cast<O*>(p.out) + int64_t(groups.id((mine << groups.low) + w * 64 + k)) * p.ldd;
      const float zero[kPiece<O>] = {};
      for (int64_t i = lane; i * kPiece<O> < p.n; i += 64) put_piece(out, i, p.n, zero);
    }
  }
}

// scale times a row's sum, added to what is there or not
template <class O, int E>
__device__ inline void put_sum(const TableGrad& p, int64_t row, int64_t c, int valid, const float (&sum)[E]) {
  O* out = static_cast<O*>(p.out) + row * p.ldd + c;
  O e[E];
  if (p.add) {
    if (valid >= E) {
      __builtin_memcpy(e, out, sizeof(e));
    } else {
#pragma unroll
      for (int k = 0; k < E; ++k) e[k] = k < valid ? out[k] : O(0.0f);
    }
#pragma unroll
    for (int k = 0; k < E; ++k) e[k] = O(float(e[k]) + p.scale * sum[k]);
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) e[k] = O(p.scale * sum[k]);
  }
  if (valid >= E) {
    __builtin_memcpy(out, e, sizeof(e));
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (k < valid) out[k] = e[k];
  }
}

constexpr int kBegins = 1, kPasses = 2;  // state of a run: its last row goes on in the next run; all of it is one row that does and has begun before

// A wavefront adds up kRun entries of the list over 64 pieces of their rows.  A row all of whose entries it has is done; one that
// goes on leaves a part: where the run begins in part row 2 r, else in 2 r + 1.
template <class T, class O>
__global__ __launch_bounds__(256) void k_sum(TableGrad p, Lists lists, int64_t first) {
  constexpr int E = kPiece<T>, U = 8;
  const int lane = threadIdx.x & 63;
  const int64_t run = first + blockIdx.x, start = run * kRun, count = *lists.count;
  if (start >= count) return;
  const int mine = int(count - start < kRun ? count - start : kRun);
  const int row = lane < mine ? lists.row[start + lane] : -1, token = lane < mine ? lists.token[start + lane] : 0;
  const int before = start > 0 ? lists.row[start - 1] : -1, after = start + kRun < count ? lists.row[start + kRun] : -1;
  for (int64_t c0 = (int64_t(blockIdx.y) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 64 * E; c0 < p.n; c0 += int64_t(gridDim.y) * 4 * 64 * E) {
    const int n = int(p.n - c0 < 64 * E ? p.n - c0 : 64 * E), valid = n - lane * E;
    const T* dy = static_cast<const T*>(p.dy) + c0;
    u32x4 c[2][U];
    const auto load = [&](int g, u32x4 (&to)[U]) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + u < mine) to[u] = near_piece(dy + int64_t(__builtin_amdgcn_readlane(token, g + u)) * p.lddy, lane, n);
    };
    float sum[E] = {};
    bool open = __builtin_amdgcn_readlane(row, 0) == before;
    int state = 0;
    const auto add = [&](int g, const u32x4 (&from)[U]) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (g + u >= mine) break;
        float v[E];
        unpack<T>(from[u], v);
#pragma unroll
        for (int k = 0; k < E; ++k) sum[k] += v[k];
        const int e = g + u, id = __builtin_amdgcn_readlane(row, e), next = e + 1 < kRun ? __builtin_amdgcn_readlane(row, e + 1) : after;
        if (id == next) {
          if (e + 1 < kRun) continue;
          state = open ? kPasses : kBegins;
        }
        if (open || state) {
          if (valid > 0) put_vector(lists.part + (2 * run + (open ? 0 : 1)) * p.n + c0, lane, n, sum);
        } else if (valid > 0) {
          put_sum<O>(p, id, c0 + lane * E, valid, sum);
        }
        open = false;
#pragma unroll
        for (int k = 0; k < E; ++k) sum[k] = 0.0f;
      }
    };
    load(0, c[0]);
#pragma unroll
    for (int g = 0; g < kRun; g += 2 * U) {
      load(g + U, c[1]);
      add(g, c[0]);
      load(g + 2 * U, c[0]);
      add(g + U, c[1]);
    }
    if (c0 == 0 && lane == 0) lists.state[run] = state;
  }
}

// The parts of a row that went on from run to run, added up in order: eight wavefronts a share of them each, then their sums.
template <class O>
__global__ __launch_bounds__(512) void k_join(TableGrad p, Lists lists, int64_t first) {
  __shared__ f32x4 sums[8][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t run = first + blockIdx.x, count = *lists.count, runs = (count + kRun - 1) / kRun;
  if (run >= runs || lists.state[run] != kBegins) return;
  const int64_t row = lists.row[run * kRun + kRun - 1];
  int64_t last = run + 1;  // the run in which the row ends
  for (;;) {
    const bool ends = last + lane >= runs || lists.state[last + lane] != kPasses;
    const uint64_t which = __ballot(ends);
    if (which) {
      last += __builtin_ctzll(which);
      break;
    }
    last += 64;
  }
  const int64_t parts = last - run + 1, share = (parts + 7) / 8, from = wave * share, to = from + share < parts ? from + share : parts;
  for (int64_t c0 = int64_t(blockIdx.y) * 256; c0 < p.n; c0 += int64_t(gridDim.y) * 256) {
    const int n = int(p.n - c0 < 256 ? p.n - c0 : 256), valid = n - lane * 4;
    f32x4 sum = {};
#pragma unroll 8
    for (int64_t k = from; k < to; ++k) {
      float v[4];
      vector_of<4>(lists.part + (k == 0 ? 2 * run + 1 : 2 * (run + k)) * p.n + c0, lane, n, 0.0f, v);
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[q] += v[q];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && valid > 0) {
      float v[4];
#pragma unroll
      for (int w = 1; w < 8; ++w) sum += sums[w][lane];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = sum[q];
      put_sum<O>(p, row, c0 + lane * 4, valid, v);
    }
    __syncthreads();
  }
}

constexpr int64_t kFewTokens = 256;
inline bool scans(int64_t t, int64_t vocab) { return t <= kFewTokens || vocab > (int64_t(1) << 22); }

template <class T, class O>
int launch_grad(const TableGrad& p, void* workspace, hipStream_t st) {
  if (scans(p.t, p.vocab)) {
    const int64_t items = (p.vocab + 3) / 4 * ((p.n + 64 * kPiece<T> - 1) / (64 * kPiece<T>)), most = 1 << 20;
    k_scan<T, O><<<unsigned(items < most ? items : most), 256, 0, st>>>(p);
    return launched();
  }
  const Lists lists = carve(workspace, p.t, p.n);
  const Groups groups = groups_of(p.vocab);
  k_group<O><<<unsigned(groups.count()), kWaves * 64, 0, st>>>(p, groups, lists);
  const int64_t runs = (p.t + kRun - 1) / kRun, wide = int64_t(1) << 20;
  const auto slabs = [&](int64_t of, int64_t most) {
    const int64_t all = (p.n + of - 1) / of;
    return unsigned(all < most ? all : most);
  };
  const unsigned y = slabs(4 * 64 * kPiece<T>, 8), z = slabs(256, 8);
  for (int64_t first = 0; first < runs; first += wide)
    k_sum<T, O><<<dim3(unsigned(runs - first < wide ? runs - first : wide), y), 256, 0, st>>>(p, lists, first);
  for (int64_t first = 0; first < runs - 1; first += wide / 2)
    k_join<O><<<dim3(unsigned(runs - first < wide / 2 ? runs - first : wide / 2), z), 512, 0, st>>>(p, lists, first);
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
  if (!sizes_ok(tokens, vocab, width) || scans(tokens, vocab)) return 0;
  return carve(nullptr, tokens, width).bytes;
}

int xmem_embedding_backward(const void* d_dy, int64_t lddy, const int64_t* d_ids, int64_t tokens, int64_t vocab, int64_t width,
                            int dtype, float scale, int64_t padding_id, int add, int out_dtype, void* d_dtable, int64_t ldd,
                            void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (!sizes_ok(tokens, vocab, width) || !type_ok(dtype) || (out_dtype != dtype && out_dtype != XMEM_F32)) return XMEM_EINVAL;
  if (!ld_ok(lddy, width) || !ld_ok(ldd, width)) return XMEM_EINVAL;
  if (tokens == 0 && add) return XMEM_OK;
  if (!d_dtable || (tokens > 0 && (!d_dy || !d_ids))) return XMEM_EINVAL;
  const size_t need = xmem_embedding_backward_workspace_bytes(tokens, vocab, width);
  if (need > 0 && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256))) return XMEM_EWORKSPACE;
  const TableGrad p{d_dy, lddy, d_ids, tokens, vocab, width, scale, padding_id, add != 0, d_dtable, ldd};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (dtype == XMEM_F32) return launch_grad<float, float>(p, d_workspace, st);
  if (out_dtype == XMEM_F32) return (dtype == XMEM_BF16 ? launch_grad<bf16, float> : launch_grad<f16, float>)(p, d_workspace, st);
  return (dtype == XMEM_BF16 ? launch_grad<bf16, bf16> : launch_grad<f16, f16>)(p, d_workspace, st);
}

}  // extern "C"
