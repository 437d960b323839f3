// embedding.hip -- scaled rows of a table, and the table's gradient, on MI355X (gfx950).
//
// Lookup: y_t = c E[id_t], 16 bytes a lane.  Bound by memory: 32768 rows of 4096 in bfloat16 75 us (7.2 TB/s of rows read and written: frequent
// tokens' rows are in the caches).  One row takes 2.3 us, of which a launch is 2.1.
//
// Gradient: dE_v = c sum over id_t = v of dy_t.  The tokens are sorted by row in one launch (k_group), so that a row's gradient is added up
// in registers, in a fixed order and without atomics on numbers, and written once; rows without a token are cleared beside that.  A frequent
// token may have thousands of rows of dy and most have one or two, so wavefronts take equal runs of the sorted list, whoever's they are
// (k_sum), and rows that go past two runs are joined from 32-bit parts (k_join).
// 32768 x 2048 into 50304 rows in bfloat16, tokens by 1 / (rank + 1): k_group 19 us, k_sum 44, k_join 6.6 (340 MB in all: 69 at a large copy's
// rate).  8192 x 1024 added to float32: 8.1, 13 and 4.4, each bound by the latency of what it reads one after another (k_sum the list's length,
// then the places around its run, then dy).
// Few tokens of a small table take one launch (k_scan), in which each row of the table looks at all of them: 37 x 515 4.9 us.
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
  bool past_caches;  // the rows without a token
};

// W columns of a row of n >= W from c on: the last place is moved so far down that it ends with the row.  Two lanes of a wavefront have
// its columns twice then, and write the same values to them.
__device__ inline int64_t place_of(int64_t c, int64_t n, int w) { return c < n - w ? c : n - w; }

// What one lane of a wavefront wrote is there for the others, and what it read is not yet what they write.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- few tokens: every row looks at all of them

constexpr int kTile = 2048;  // tokens looked at together

// A workgroup has four rows of the table (far apart: neighbours may all be frequent) and 64 pieces of them.  Each wavefront looks at every
// fourth 64 of the tokens, notes those of the four rows, loads their rows of dy eight at a time and adds them up; then each has one of the
// rows and the four sums of it.  E: elements of a piece, one where rows have fewer than eight.
template <class T, class O, int E>
__global__ __launch_bounds__(256) void k_scan(TableGrad p) {
  constexpr int U = 8, QUARTER = kTile / 4, PER = QUARTER / 64;
  __shared__ unsigned short notes[4][QUARTER];  // token behind the wavefront's first, row
  __shared__ float parts[4][4][E][64];
  __shared__ unsigned touched[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t pieces = (p.n + E - 1) / E, slabs = (pieces + 63) / 64, apart = (p.vocab + 3) / 4;
  for (int64_t item = blockIdx.x; item < apart * slabs; item += gridDim.x) {
    const int64_t row0 = item / slabs, slab = item % slabs, p0 = pieces * slab / slabs, c0 = p0 * E;
    const int wide = int(pieces * (slab + 1) / slabs - p0), off = int(place_of(c0 + (lane < wide ? lane : wide - 1) * E, p.n, E) - c0);
    const T* dy = static_cast<const T*>(p.dy) + c0;
    float sum[4][E] = {};
    unsigned mine = 0;  // rows with a token
    for (int64_t t0 = wave * 64; t0 < p.t; t0 += kTile) {
      uint64_t id[PER];
      const int here = int(p.t - t0 < kTile ? p.t - t0 : kTile);
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (j * 256 < here) id[j] = p.ids[t0 + (j * 256 + lane < here ? j * 256 + lane : here - 1)];
      int own = 0;
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (j * 256 < here) {
          // which of the four rows
          const unsigned low = unsigned(id[j]), far = low - unsigned(row0);
          const int r = far == 0 ? 0 : far == unsigned(apart) ? 1 : far == 2 * unsigned(apart) ? 2 : 3;
          const uint64_t hit = __ballot(far == r * unsigned(apart) && (id[j] >> 32) == 0 && low < unsigned(p.vocab) && int64_t(id[j]) != p.padding &&
                                        j * 256 + lane < here);
          if (hit) {
            if (hit >> lane & 1) notes[wave][own + __popcll(hit & ((uint64_t(1) << lane) - 1))] = static_cast<unsigned short>((j * 256 + lane) << 2 | r);
            own += __popcll(hit);
          }
        }
      wave_sync();
#pragma unroll 1
      for (int k = 0; k < own; k += U) {
        const int note = notes[wave][k + (lane & (U - 1)) < own ? k + (lane & (U - 1)) : k];
        u32x4 c[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k + u < own)
            __builtin_memcpy(&c[u], dy + (t0 + (__builtin_amdgcn_readlane(note, u) >> 2)) * p.lddy + unsigned(off), E * sizeof(T));
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k + u < own) {
            const int r = __builtin_amdgcn_readlane(note, u) & 3;
            mine |= 1u << r;
            T piece[E];
            __builtin_memcpy(piece, &c[u], sizeof(piece));
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (r == q)
#pragma unroll
                for (int e = 0; e < E; ++e) sum[q][e] += float(piece[e]);
          }
      }
      wave_sync();
    }
    if (lane == 0) touched[wave] = mine;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (mine >> q & 1)
#pragma unroll
        for (int e = 0; e < E; ++e) parts[wave][q][e][lane] = sum[q][e];
    __syncthreads();
    const int64_t row = row0 + wave * apart;
    bool any = false;
    float total[E] = {};
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (touched[w] >> wave & 1) {
        any = true;
#pragma unroll
        for (int e = 0; e < E; ++e) total[e] += parts[w][wave][e][lane];
      }
    if (row < p.vocab && (any || !p.add) && lane < wide) {
      O* out = static_cast<O*>(p.out) + row * p.ldd + c0 + off;
      O o[E];
      if (p.add) __builtin_memcpy(o, out, sizeof(o));
      wave_sync();  // elements that two lanes have are read by both before one writes them
      const float scale = any ? p.scale : 0.0f;  // of no token nothing is scaled: 0 times a factor that is not finite is NaN
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = O(p.add ? float(o[e]) + scale * total[e] : scale * total[e]);
      __builtin_memcpy(out, o, sizeof(o));
    }
    __syncthreads();
  }
}

// ---- many tokens: grouped by row first

// Rows are spread over groups of kKeys or fewer by a multiplication: key = id * mul mod 2^bits, of which the upper bits are
// the group, so that frequent tokens (whose numbers are often neighbours) do not meet in one.  256 groups or more, one a CU (of 64 and
// 128 the grouping of 32768 tokens took 27.6 and 23.3 us where it took 21.7).
constexpr int kGroups = 256, kKeyBits = 10, kKeys = 1 << kKeyBits, kWaves = 16;
// Entries of the sorted list that one wavefront adds up: 8 where few tokens are added to a gradient, each row of which is read first, else
// 16.  Sums and joins in us, of 16 and 8: added, 8192 x 1024 19.7 and 17.4, 4096 x 256 14.5 and 11.1, 16384 x 1024 24.9 and 25.6, 32768 x 2048
// 61 and 67; written, 8192 x 1024 22.7 and 25.1, 32768 x 2048 50 and 64.  32 are slower in all of them.
constexpr int kRun = 16, kShortRun = 8;
constexpr int64_t kShortTokens = 16384;  // fewer

struct Groups {
  int bits, low;  // of a key, and of its place in the group
  unsigned mul, inverse;
  __host__ __device__ int64_t count() const { return int64_t(1) << (bits - low); }
  __host__ __device__ int words() const { return low > 6 ? 1 << (low - 6) : 1; }  // of 64 keys, in a group
  __host__ __device__ unsigned mask() const { return (1u << bits) - 1; }
  __device__ unsigned key(unsigned id) const { return id * mul & mask(); }
  __device__ unsigned id(unsigned key) const { return key * inverse & mask(); }
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
  int* count;        // entries, and rows that go past two runs
  int* state;        // of a run, see k_sum
  int* begin;        // the runs in which those rows begin, in any order
  uint64_t* empty;   // a bit for each key whose row is in the table and has no token
  float* part;       // two rows a run
  size_t bytes;
};
Lists carve(void* base, int64_t t, const Groups& groups, int64_t n) {
  Lists w;
  char* at = static_cast<char*>(base);
  const auto take = [&](size_t b) {
    char* r = at;
    at += up256(b);
    return r;
  };
  // room for the runs of any batch of so many tokens or fewer: few tokens may make more runs
  const int64_t few = ((t < kShortTokens ? t : kShortTokens - 1) + kShortRun - 1) / kShortRun, many = (t + kRun - 1) / kRun;
  const int64_t runs = few > many ? few : many;
  w.token = reinterpret_cast<int*>(take(size_t(t) * 4));
  w.row = reinterpret_cast<int*>(take(size_t(t) * 4));
  w.count = reinterpret_cast<int*>(take(8));
  w.state = reinterpret_cast<int*>(take(size_t(runs) * 4));
  w.begin = reinterpret_cast<int*>(take(size_t(runs) * 4));
  w.empty = reinterpret_cast<uint64_t*>(take(size_t(groups.count()) * groups.words() * 8));
  w.part = reinterpret_cast<float*>(take(size_t(runs) * 2 * size_t(n) * 4));
  w.bytes = size_t(at - static_cast<char*>(base));
  return w;
}

// A wavefront clears a row: 16 bytes a lane, the last ones moved down to the row's end.
__device__ inline void clear_row(char* row, int64_t bytes, bool past_caches) {
  const int lane = threadIdx.x & 63;
  const u32x4 zero = {};
  if (bytes < 16) {
    if (lane < bytes / 2) reinterpret_cast<short*>(row)[lane] = 0;
  } else if (past_caches) {
#pragma unroll 4
    for (int64_t i = lane * 16; i < bytes; i += 64 * 16) store_past(row + (i < bytes - 16 ? i : bytes - 16), zero);
  } else {
#pragma unroll 4
    for (int64_t i = lane * 16; i < bytes; i += 64 * 16) __builtin_memcpy(row + (i < bytes - 16 ? i : bytes - 16), &zero, 16);
  }
}

// The table's rows, by bytes.  Those from `early` on are cleared beside the grouping, whether they have tokens or not, the others without
// a token beside the sums.
struct Clear {
  char* table;
  int64_t row, distance, early, vocab;
  bool past_caches;
  __device__ void at(int64_t v) const { clear_row(table + v * distance, row, past_caches); }
};

// Sorting.  A workgroup has the rows of one group.  It looks at every token, each wavefront at a sixteenth of them in order, counts those of the
// groups before and notes its own in LDS; then it counts its rows' tokens and puts them where these counts say.  Where a wavefront has
// more than `most` of its own, its workgroup reads the tokens again for each of the two.  This takes few of the memory's cycles: workgroups
// past the groups' clear rows beside it.
__global__ __launch_bounds__(kWaves * 64) void k_group(const int64_t* ids, int64_t t, unsigned vocab, unsigned padding, Groups groups, Lists lists,
                                                       int most, Clear clear) {
  __shared__ int meet[kWaves][2], sums[kWaves];
  extern __shared__ int dynamic[];  // counts of each wavefront and row, then notes: place in the group, and the token's number in the share
  if (blockIdx.x >= groups.count()) {
    const int64_t step = (int64_t(gridDim.x) - groups.count()) * kWaves;
    const int64_t mine = (blockIdx.x - groups.count()) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t v = clear.early + mine; v < clear.vocab; v += step) clear.at(v);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int keys = 1 << groups.low;
  const unsigned mine = blockIdx.x, width = groups.bits - groups.low;
  int* const hist = dynamic + wave * keys;
  unsigned* const notes = reinterpret_cast<unsigned*>(dynamic + kWaves * keys) + wave * most;
  for (int i = threadIdx.x; i < kWaves * keys; i += kWaves * 64) dynamic[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) lists.count[1] = 0;
  const int64_t share = ((t + kWaves - 1) / kWaves + 63) / 64 * 64, from = wave * share < t ? wave * share : t;
  const int n = int(from + share < t ? share : t - from);
  ids += from;
  int before = 0, own = 0;
  // calls f(the lanes whose token is of this group, a lane's place in it, the first lane's token) for 64 tokens at a time
  const auto each = [&](const auto& f) {
    constexpr int kBatch = 8;
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += kBatch * 64) {
      uint64_t id[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) id[j] = ids[i0 + j * 64 + lane < n ? i0 + j * 64 + lane : 0];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const unsigned low = unsigned(id[j]), high = unsigned(id[j] >> 32), key = groups.key(low);
        const uint64_t there = __ballot(high == 0) & __ballot(low < vocab) & __ballot(low != padding) & __ballot(i0 + j * 64 + lane < n);
        const unsigned group = __builtin_amdgcn_ubfe(key, groups.low, width);
        f(there & __ballot(group == mine), there & __ballot(group < mine), int(key & (keys - 1)), i0 + j * 64);
      }
    }
  };
  const bool noted = share < (int64_t(1) << (32 - kKeyBits));
  each([&](uint64_t hit, uint64_t less, int local, int i0) {
    before += __popcll(less);
    if (hit) {
      const int at = own + __popcll(hit & ((uint64_t(1) << lane) - 1));
      if (hit >> lane & 1 && at < most) notes[at] = unsigned(i0 + lane) << kKeyBits | unsigned(local);
      own += __popcll(hit);
    }
  });
  if (lane == 0) {
    meet[wave][0] = before;
    meet[wave][1] = own;
  }
  __syncthreads();
  int base = 0;
  bool fits = noted;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    base += meet[w][0];
    fits = fits && meet[w][1] <= most;
  }
  if (fits) {
    for (int i = lane; i < own; i += 64) atomicAdd(&hist[notes[i] & (kKeys - 1)], 1);
  } else {
    each([&](uint64_t hit, uint64_t, int local, int) {
      if (hit >> lane & 1) atomicAdd(&hist[local], 1);
    });
  }
  __syncthreads();
  // the places of a row's tokens: behind those of the group's rows before it, a wavefront's behind the earlier ones'
  int here = 0;
  if (int(threadIdx.x) < keys)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) here += dynamic[w * keys + threadIdx.x];
  int place = here;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(place, d);
    if (lane >= d) place += up;
  }
  const uint64_t empty = __ballot(int(threadIdx.x) < keys && here == 0 && groups.id((mine << groups.low) + threadIdx.x) < clear.early);
  if (lane == 0 && wave < groups.words()) lists.empty[mine * groups.words() + wave] = empty;
  if (lane == 63) sums[wave] = place;
  __syncthreads();
  for (int w = 0; w < wave; ++w) place += sums[w];
  place += base;
  if (mine + 1 == groups.count() && int(threadIdx.x) == keys - 1) *lists.count = place;  // all of them
  place -= here;
  if (int(threadIdx.x) < keys)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = dynamic[w * keys + threadIdx.x];
      dynamic[w * keys + threadIdx.x] = place;
      place += c;
    }
  __syncthreads();
  // up to 64 tokens in their order, those of one row at a time
  const auto put = [&](uint64_t left, int local, int token) {
    while (left) {
      const int leader = __builtin_ctzll(left), which = __builtin_amdgcn_readlane(local, leader);
      const uint64_t same = left & __ballot(local == which);
      const int first = hist[which];
      wave_sync();
      if (lane == leader) hist[which] = first + __popcll(same);
      wave_sync();
      if (same >> lane & 1) {
        const int at = first + __popcll(same & ((uint64_t(1) << lane) - 1));
        lists.token[at] = int(from) + token;
        lists.row[at] = int(groups.id((mine << groups.low) + unsigned(which)));
      }
      left &= ~same;
    }
  };
  if (fits) {
#pragma unroll 1
    for (int i = 0; i < own; i += 64) {
      const unsigned note = notes[i + lane < own ? i + lane : i];
      put(__ballot(i + lane < own), int(note & (kKeys - 1)), int(note >> kKeyBits));
    }
  } else {
    each([&](uint64_t hit, uint64_t, int local, int i0) { put(hit, local, i0 + lane); });
  }
}

// What a run leaves: its last row begins in it and ends past the next run; all of it is one row that began before and goes on.
constexpr int kBegins = 1, kPasses = 2;

// A wavefront adds up the entries of a run over 64 pieces of their rows, as many of them alike as slabs come to.  A row that begins in
// the run and ends in the next is finished here, and left out there.  A longer one leaves its part in part row 2 r + 1 where it
// begins and in 2 r where it goes on or ends.  The next entries' loads are on their way while a batch is added up.
// Workgroups past the launch's `runs` clear the rows without a token, those of 64 keys at a time.
// E: elements of a piece, one where rows have fewer than eight.  In 16 bits eight, of what is added to a gradient four: its rows, which are
// read first, may have 32 bits, and few tokens make more wavefronts.  Whole calls in us, of four and eight: added, 8192 x 1024 25.6 and 27.9,
// 16384 x 1024 35.8 and 37.8; written, 8192 x 1024 29.5 and 30.6, 32768 x 2048 94 and 84, 32768 x 4096 179 and 163.
template <class T, class O, bool ADD, int E, int RUN>
__global__ __launch_bounds__(256) void k_sum(TableGrad p, Groups groups, Lists lists, int64_t first_run, unsigned runs, Clear clear) {
  constexpr int U = 4;
  if (!ADD && blockIdx.x >= runs) {
    const unsigned words = unsigned(groups.words());
    const int64_t all = groups.count() * words, step = int64_t(gridDim.x - runs) * gridDim.y;
    for (int64_t word = int64_t(blockIdx.x - runs) * gridDim.y + blockIdx.y; word < all; word += step) {
      uint64_t left = lists.empty[word];
      const unsigned key = (unsigned(word / words) << groups.low) + unsigned(word % words) * 64;
      for (int turn = 0; left; ++turn) {
        const int k = __builtin_ctzll(left);
        left &= left - 1;
        if (turn % 4 == __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) clear.at(groups.id(key + k));
      }
    }
    return;
  }
  const int lane = threadIdx.x & 63;
  const int64_t run = first_run + blockIdx.x, start = run * RUN, count = *lists.count;
  if (start >= count) return;
  const int row = start + lane < count ? lists.row[start + lane] : -1, token = start + lane < count ? lists.token[start + lane] : 0;
  const int before = start > 0 ? lists.row[start - 1] : -1, earlier = start > RUN ? lists.row[start - RUN - 1] : -1;
  const int after = start + 2 * RUN < count ? lists.row[start + 2 * RUN] : -1;
  const auto row_at = [&](int e) { return __builtin_amdgcn_readlane(row, e); };
  const int head = row_at(0), tail = row_at(RUN - 1);
  const bool on = tail >= 0 && tail == row_at(RUN);  // the run's last row goes on
  const bool open = head == before, passes = open && on && head == tail, part = open && (passes || head == earlier);
  int begin = 0, end = int(count - start < RUN ? count - start : RUN);
  if (open && !part) begin = __builtin_ctzll(__ballot(row != head));
  int state = passes ? kPasses : 0;
  if (on && !passes) {
    if (tail == row_at(2 * RUN - 1) && tail == after) {
      state = kBegins;
    } else {
      const uint64_t other = __ballot(row != tail) >> RUN;
      end = other ? RUN + __builtin_ctzll(other) : 2 * RUN;
    }
  }
  // entries that are their row's last here
  const uint64_t last = __ballot(row != __shfl_down(row, 1)) | uint64_t(1) << (end - 1);
  if (blockIdx.y == 0 && threadIdx.x == 0) {
    lists.state[run] = state;
    if (state == kBegins) lists.begin[atomicAdd(lists.count + 1, 1)] = int(run);
  }
  const int64_t pieces = (p.n + E - 1) / E, slabs = (pieces + 63) / 64;
  for (int64_t slab = int64_t(blockIdx.y) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); slab < slabs; slab += int64_t(gridDim.y) * 4) {
    const int64_t p0 = pieces * slab / slabs, c0 = p0 * E;
    const int wide = int(pieces * (slab + 1) / slabs - p0);
    const int off = int(place_of(c0 + (lane < wide ? lane : wide - 1) * E, p.n, E) - c0);
    const T* dy = static_cast<const T*>(p.dy) + c0;
    O* out = static_cast<O*>(p.out) + c0;
    struct Batch {
      T dy[U][E];
      O old[ADD ? U : 1][E];
    };
    const auto load = [&](int g, Batch& to) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + u < end) {
          __builtin_memcpy(to.dy[u], dy + int64_t(__builtin_amdgcn_readlane(token, g + u)) * p.lddy + unsigned(off), sizeof(to.dy[u]));
          if constexpr (ADD)
            if (last >> (g + u) & 1) __builtin_memcpy(to.old[u], out + int64_t(row_at(g + u)) * p.ldd + unsigned(off), sizeof(to.old[u]));
        }
    };
    float sum[E] = {};
    Batch now, next;
    load(begin, now);
#pragma unroll 1
    for (int g = begin; g < end; g += U) {
      load(g + U, next);
      if (ADD) wave_sync();  // elements that two lanes have are read by both before one writes them
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = g + u;
        if (e >= end) break;
#pragma unroll
        for (int k = 0; k < E; ++k) sum[k] += float(now.dy[u][k]);
        if (!(last >> e & 1)) continue;
        const int id = row_at(e);
        const bool to_part = (part && id == head) || (state == kBegins && e == end - 1);
        if (lane < wide) {
          if (to_part) {
            __builtin_memcpy(lists.part + (2 * run + (part && id == head ? 0 : 1)) * p.n + c0 + off, sum, sizeof(sum));
          } else {
            O o[E];
#pragma unroll
            for (int k = 0; k < E; ++k) o[k] = O(ADD ? float(now.old[ADD ? u : 0][k]) + p.scale * sum[k] : p.scale * sum[k]);
            __builtin_memcpy(out + int64_t(id) * p.ldd + unsigned(off), o, sizeof(o));
          }
        }
#pragma unroll
        for (int k = 0; k < E; ++k) sum[k] = 0.0f;
      }
      now = next;
    }
  }
}

// The parts of the rows that went past two runs, added up in order: four wavefronts a share of them each, then their sums.
template <class O, int E, int RUN>
__global__ __launch_bounds__(256) void k_join(TableGrad p, Lists lists) {
  constexpr int U = 8;
  __shared__ __attribute__((aligned(16))) float sums[3][64][E];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t runs = (*lists.count + RUN - 1) / RUN, rows = lists.count[1];
  const int64_t pieces = (p.n + E - 1) / E, slabs = (pieces + 63) / 64;
  for (int64_t item = blockIdx.x; item < rows * slabs; item += gridDim.x) {
    const int64_t run = lists.begin[item / slabs], slab = item % slabs, row = lists.row[run * RUN + RUN - 1];
    int64_t last = run + 1;  // the run in which the row ends
    for (;;) {
      const uint64_t which = __ballot(last + lane >= runs || lists.state[last + lane] != kPasses);
      if (which) {
        last += __builtin_ctzll(which);
        break;
      }
      last += 64;
    }
    const int64_t parts = last - run + 1, share = (parts + 3) / 4, from = wave * share, to = from + share < parts ? from + share : parts;
    const int64_t p0 = pieces * slab / slabs, wide = pieces * (slab + 1) / slabs - p0;
    const int64_t c = place_of((p0 + (lane < wide ? lane : wide - 1)) * E, p.n, E);
    float sum[E] = {};
    for (int64_t k0 = from; k0 < to; k0 += U) {
      float v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 + u < to) __builtin_memcpy(v[u], lists.part + (k0 + u == 0 ? 2 * run + 1 : 2 * (run + k0 + u)) * p.n + c, sizeof(v[u]));
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 + u < to)
#pragma unroll
          for (int k = 0; k < E; ++k) sum[k] += v[u][k];
    }
    if (wave > 0) __builtin_memcpy(sums[wave - 1][lane], sum, sizeof(sum));
    __syncthreads();
    if (wave == 0) {
      O* out = static_cast<O*>(p.out) + row * p.ldd + c;
      O o[E];
      if (p.add) __builtin_memcpy(o, out, sizeof(o));
      wave_sync();  // elements that two lanes have are read by both before one writes them
#pragma unroll
      for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int k = 0; k < E; ++k) sum[k] += sums[w][lane][k];
#pragma unroll
      for (int k = 0; k < E; ++k) o[k] = O(p.add ? float(o[k]) + p.scale * sum[k] : p.scale * sum[k]);
      if (lane < wide) __builtin_memcpy(out, o, sizeof(o));
    }
    __syncthreads();
  }
}

// Looking at every token for every row takes one launch, grouping three.  In us, 895 rows of 147: 16 tokens 4.2 against 11.3, 600 7.6 against
// 17.1, 2000 15.8 against 18.2; 1224 rows of 3904: 10.4 and 12.9, 13.4 and 19.6, 21.6 and 22.4; 8 tokens of 50304 rows of 1024 67 and 22.
constexpr int64_t kFewTokens = 2048, kFewItems = 2560;
inline bool scans(int64_t t, int64_t vocab, int64_t n) {
  return t <= kFewTokens && (vocab + 3) / 4 * ((n + 511) / 512) <= kFewItems;
}

template <class T, class O, bool ADD, int E, int RUN>
void launch_runs(const TableGrad& p, const Groups& groups, const Lists& lists, const Clear& clear, hipStream_t st) {
  constexpr int J = E == 1 ? 1 : 4;  // columns of a lane in the joins
  const int64_t runs = (p.t + RUN - 1) / RUN, most = int64_t(1) << 19;
  const int64_t slabs = ((p.n + E - 1) / E + 63) / 64, four = (slabs + 3) / 4, high = four < 8 ? four : 8;
  for (int64_t first = 0; first == 0 || first < runs; first += most) {  // no tokens: the table is cleared all the same
    const int64_t here = runs - first < most ? runs - first : most, words = (groups.count() * groups.words() + high - 1) / high;
    const int64_t beside = ADD || first || clear.early == 0 ? 0 : words < most ? words : most;
    if (here + beside > 0)
      k_sum<T, O, ADD, E, RUN><<<dim3(unsigned(here + beside), unsigned(high)), 256, 0, st>>>(p, groups, lists, first, unsigned(here), clear);
  }
  if (runs > 2) {
    const int64_t items = (runs - 2) * ((p.n + 64 * J - 1) / (64 * J));
    k_join<O, J, RUN><<<unsigned(items < 2048 ? items : 2048), 256, 0, st>>>(p, lists);
  }
}

template <class T, class O, bool WHOLE>
void launch_sums(const TableGrad& p, const Groups& groups, const Lists& lists, const Clear& clear, hipStream_t st) {
  if (!p.add)
    launch_runs<T, O, false, WHOLE ? kPiece<T> : 1, kRun>(p, groups, lists, clear, st);
  else if (p.t < kShortTokens)
    launch_runs<T, O, true, WHOLE ? 4 : 1, kShortRun>(p, groups, lists, clear, st);
  else
    launch_runs<T, O, true, WHOLE ? 4 : 1, kRun>(p, groups, lists, clear, st);
}

template <class T, class O>
int launch_grad(const TableGrad& p, void* workspace, hipStream_t st) {
  if (scans(p.t, p.vocab, p.n)) {
    constexpr int E = kPiece<T>;
    const int64_t items = (p.vocab + 3) / 4 * ((p.n + 64 * E - 1) / (64 * E)), most = 1 << 20;
    const unsigned grid = unsigned(items < most ? items : most);
    if (p.n < 8)
      k_scan<T, O, 1><<<grid, 256, 0, st>>>(p);
    else
      k_scan<T, O, E><<<grid, 256, 0, st>>>(p);
    return launched();
  }
  const Groups groups = groups_of(p.vocab);
  const Lists lists = carve(workspace, p.t, groups, p.n);
  const unsigned vocab = unsigned(p.vocab), padding = p.padding >= 0 && p.padding < p.vocab ? unsigned(p.padding) : ~0u;
  const int64_t share = (p.t + kWaves - 1) / kWaves;
  const int notes = share >= 4096 ? 1024 : share >= 256 ? int(share / 4) : 64;
  // Grouping many tokens leaves the memory idle for as long as it takes to clear 1,500 bytes a token: 32768 x 2048 88.3 us without, 84.1
  // with, 85.5 with 2,500.  With 8192 tokens it is not worth the rows that are then written twice (31.0, 32.1).
  const int64_t row = p.n * int64_t(sizeof(O)), early = p.add || p.t < 16384 ? 0 : p.t * 1500 / row;
  const Clear clear{static_cast<char*>(p.out), row, p.ldd * int64_t(sizeof(O)), early < p.vocab ? p.vocab - early : 0, p.vocab, p.past_caches};
  const unsigned grid = unsigned(groups.count()) + (early ? kCus : 0);
  k_group<<<grid, kWaves * 64, size_t(kWaves) * ((1 << groups.low) + notes) * 4, st>>>(p.ids, p.t, vocab, padding, groups, lists, notes, clear);
  if (p.n < 8)
    launch_sums<T, O, false>(p, groups, lists, clear, st);
  else
    launch_sums<T, O, true>(p, groups, lists, clear, st);
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
  if (!sizes_ok(tokens, vocab, width) || scans(tokens, vocab, width)) return 0;
  return carve(nullptr, tokens, groups_of(vocab), width).bytes;
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
  const int element = dtype == XMEM_F32 ? 4 : 2, out_element = out_dtype == XMEM_F32 ? 4 : 2;
  if (shares(d_workspace, need, d_dy, tokens, lddy, width, element) || shares(d_workspace, need, d_ids, 1, tokens, tokens, 8) ||
      shares(d_workspace, need, d_dtable, vocab, ldd, width, out_element))
    return XMEM_EINVAL;
  // Clearing a table of 206 MB past the caches leaves them to the sums' reads (with them 64.8 us, past them 53.9); one of 103 MB
  // stays in the cache behind the L2s (18.2 and 21.9).
  const bool past_caches = vocab * width * out_element >= kCacheBytes / 2;
  const TableGrad p{d_dy, lddy, d_ids, tokens, vocab, width, scale, padding_id, add != 0, d_dtable, ldd, past_caches};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (dtype == XMEM_F32) return launch_grad<float, float>(p, d_workspace, st);
  if (out_dtype == XMEM_F32) return (dtype == XMEM_BF16 ? launch_grad<bf16, float> : launch_grad<f16, float>)(p, d_workspace, st);
  return (dtype == XMEM_BF16 ? launch_grad<bf16, bf16> : launch_grad<f16, f16>)(p, d_workspace, st);
}

}  // extern "C"
