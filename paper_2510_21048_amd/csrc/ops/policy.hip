// policy.hip -- the clipped policy loss with a KL term over a vocabulary, on MI355X (gfx950).
//
// With m the row's largest logit and s = sum_j exp(x_j - m), the token's log-probability is (x_y - m) - log s, every other
// number of a row follows from it and four scalars, and dx_j = c (1[j = y] - exp(x_j - m) / s) with one c a row.  So a row is
// read once and its gradient written once: a workgroup keeps it in registers between the two (52 a thread for 50,304 logits of
// 16 bits in 512 threads).  Rows past 16,384 pieces of 16 bytes (131,072 logits of 16 bits, 65,536 of 32) do not fit there: those are
// read twice where a gradient is wanted, 2048 x 131072 in float32 in 583 us.
// Exponentials and sums are in 32 bits, the batch's sums in 64 and in a fixed order (k_policy_sums).  exp(x - m) is a power of two of
// (x - m) log2(e), whose rounding adds |x - m| 2^-24 to a term's relative error: terms that count are near m.
// Bound by memory: 32768 x 50304 in bfloat16, 30% of the rows masked, 5.6 GB in 1.08 ms (5.2 TB/s; a large copy reaches 4.9);
// log-probabilities of 2048 x 50304 42 us (4.9 TB/s).  A row and its sums take 8 us at least: two launches.
#include "common.h"

using namespace xops;

namespace {

struct Policy {
  const void* x;
  int64_t ldl;
  const int64_t* y;
  const float *w, *old_lp, *adv, *ref;
  int64_t tokens, vocab;
  float low, high, kl_coef, grad_scale;
  float* lp;
  void* dx;
  int64_t ldd;
  float* part;  // [3][tokens]
  int64_t first = 0;  // row of the launch
};

constexpr float kLog2e = 1.4426950408889634f;

template <class T> constexpr int kPer = 16 / sizeof(T);  // elements of a chunk

// Chunk i of a row of `vocab` elements; what the row does not have is -inf, whose exponential is 0.
template <class T>
__device__ inline u32x4 chunk_of(const T* x, int64_t i, int64_t vocab) {
  constexpr int E = kPer<T>;
  u32x4 c;
  if ((i + 1) * E <= vocab) {
    __builtin_memcpy(&c, x + i * E, 16);
  } else {
    T e[E];
#pragma unroll
    for (int k = 0; k < E; ++k) e[k] = i * E + k < vocab ? x[i * E + k] : T(-INFINITY);
    __builtin_memcpy(&c, e, 16);
  }
  return c;
}
template <class T>
__device__ inline void store_chunk(T* dx, int64_t i, int64_t vocab, const float* v) {
  constexpr int E = kPer<T>;
  T e[E];
#pragma unroll
  for (int k = 0; k < E; ++k) e[k] = T(v[k]);
  if ((i + 1) * E <= vocab) {
    __builtin_memcpy(dx + i * E, e, 16);
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (i * E + k < vocab) dx[i * E + k] = e[k];
  }
}
template <class T>
__device__ inline void values(u32x4 c, float (&v)[kPer<T>]) {
  T e[kPer<T>];
  __builtin_memcpy(e, &c, 16);
#pragma unroll
  for (int k = 0; k < kPer<T>; ++k) v[k] = float(e[k]);
}

struct Max {
  __device__ static float of(float a, float b) { return fmaxf(a, b); }
};
struct Sum {
  __device__ static float of(float a, float b) { return a + b; }
};
// Over the threads of a row: a wavefront, or a workgroup (whose wavefronts' values meet in `meet`).
template <class Op, int THREADS>
__device__ inline float over_row(float v, float* meet) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = Op::of(v, __shfl_xor(v, d));
  if constexpr (THREADS > kWave) {
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = v;
    __syncthreads();
    v = meet[0];
#pragma unroll
    for (int i = 1; i < THREADS / kWave; ++i) v = Op::of(v, meet[i]);
  }
  return v;
}

// THREADS of a row (64: four rows a workgroup), NCH chunks of the row in each thread's registers: the logits are read
// once and their gradient is written once.  NCH = 0: a row too long for that is read again for each of the largest
// logit (with the sum, rescaled when a larger one comes) and the gradient.
template <class T, int THREADS, int NCH>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS, THREADS == 1024 ? 4 : THREADS == 64 ? 5 : 6) void k_policy(Policy p) {
  constexpr int E = kPer<T>;
  __shared__ float meet[2][THREADS / kWave], at_y;  // neither where a row is a wavefront
  const int tid = threadIdx.x % THREADS, slot = threadIdx.x / THREADS;
  const int64_t t = p.first + (THREADS < 256 ? int64_t(blockIdx.x) * (256 / THREADS) + slot : int64_t(blockIdx.x));
  if (t >= p.tokens) return;  // a whole wavefront, of those that do not meet others
  const int64_t vocab = p.vocab, chunks = (vocab + E - 1) / E;
  // the token's scalars, asked for together
  const float wt = p.w ? p.w[t] : 1.0f / float(p.tokens);
  const int64_t y = p.y[t];
  const bool loss = p.old_lp;
  const float old_lp = loss ? p.old_lp[t] : 0.0f, adv = loss ? p.adv[t] : 0.0f, ref = p.ref ? p.ref[t] : 0.0f;
  const T* x = static_cast<const T*>(p.x) + t * p.ldl;
  T* dx = p.dx ? static_cast<T*>(p.dx) + t * p.ldd : nullptr;
  if (wt == 0.0f) {
    const float zero[E] = {};
    if (dx)
      for (int64_t i = tid; i < chunks; i += THREADS) store_chunk<T>(dx, i, vocab, zero);
    if (tid == 0) {
      p.lp[t] = 0.0f;
      if (p.part) p.part[t] = p.part[p.tokens + t] = p.part[2 * p.tokens + t] = 0.0f;
    }
    return;
  }
  const bool in = y >= 0 && y < vocab;
  const int64_t cy = in ? y / E : -1;
  if (THREADS > kWave && !in && tid == 0) at_y = NAN;
  float m = -INFINITY, s = 0.0f, xy = NAN, v[E];
  // the sampled token's logit, from the thread that has it: the row may be overwritten
  const auto note = [&](int64_t i) {
    if (i == cy)
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (i * E + k == y) (THREADS > kWave ? at_y : xy) = v[k];
  };
  u32x4 c[NCH > 0 ? NCH : 1];
  if constexpr (NCH > 0) {
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int i = j * THREADS + tid;
      if (j * THREADS < chunks) c[j] = chunk_of(x, i, vocab);
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * THREADS < chunks) {
        values<T>(c[j], v);
        note(j * THREADS + tid);
#pragma unroll
        for (int k = 0; k < E; ++k) m = fmaxf(m, v[k]);
      }
    m = over_row<Max, THREADS>(m, meet[0]);
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * THREADS < chunks) {
        values<T>(c[j], v);
#pragma unroll
        for (int k = 0; k < E; ++k) s += __builtin_amdgcn_exp2f((v[k] - m) * kLog2e);
      }
    s = over_row<Sum, THREADS>(s, meet[1]);
  } else {
    bool nan = false;
    for (int64_t i = tid; i < chunks; i += THREADS) {
      values<T>(chunk_of(x, i, vocab), v);
      note(i);
      float top = m;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        top = fmaxf(top, v[k]);
        nan |= v[k] != v[k];
      }
      if (top > m) {
        s *= __builtin_amdgcn_exp2f((m - top) * kLog2e);
        m = top;
      }
      if (m > -INFINITY)
#pragma unroll
        for (int k = 0; k < E; ++k) s += __builtin_amdgcn_exp2f((v[k] - m) * kLog2e);
    }
    const float top = over_row<Max, THREADS>(m, meet[0]);
    // a thread with nothing but -inf adds 0, unless no thread has more
    s = nan ? NAN : m > -INFINITY || top == -INFINITY ? s * __builtin_amdgcn_exp2f((m - top) * kLog2e) : 0.0f;
    m = top;
    s = over_row<Sum, THREADS>(s, meet[1]);
  }
  // a row's own wavefront passes it between lanes (chunk i is lane i % 64's); a workgroup's has met the others' since
  xy = THREADS > kWave ? at_y : __shfl(xy, int(cy & (kWave - 1)));
  const float lp = (xy - m) - logf(s);
  float grad = 0.0f;
  if (loss) {
    const float rho = expf(lp - old_lp);
    // a ratio past 32 bits times 0 is 0, and so is a KL term past them whose coefficient is 0
    const float free = adv == 0.0f && rho == INFINITY ? 0.0f : rho * adv, held = fminf(fmaxf(rho, 1.0f - p.low), 1.0f + p.high) * adv;
    const bool clipped = held < free;
    float kl = 0.0f;
    grad = clipped ? 0.0f : -free;
    if (p.ref) {
      const float d = ref - lp, e = expm1f(d);
      kl = e - d;
      if (p.kl_coef != 0.0f) grad -= p.kl_coef * e;
    }
    grad *= wt;
    if (tid == 0) {
      p.part[t] = wt * -(clipped ? held : free);
      p.part[p.tokens + t] = wt * kl;
      p.part[2 * p.tokens + t] = clipped ? wt : 0.0f;
    }
  }
  if (tid == 0) p.lp[t] = lp;
  if (!dx) return;
  grad *= p.grad_scale;
  const float per = -grad / s;
  const auto emit = [&](u32x4 q, int64_t i) {
    values<T>(q, v);
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = per * __builtin_amdgcn_exp2f((v[k] - m) * kLog2e);
    if (i == cy)
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (i * E + k == y) v[k] += grad;
    store_chunk<T>(dx, i, vocab, v);
  };
  if constexpr (NCH > 0) {
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if (j * THREADS < chunks) emit(c[j], j * THREADS + tid);
  } else {
    for (int64_t i = tid; i < chunks; i += THREADS) emit(chunk_of(x, i, vocab), i);
  }
}

// The sums of the three parts, in 64 bits and a fixed order.
__global__ __launch_bounds__(1024) void k_policy_sums(const float* part, int64_t tokens, float kl_coef, float* stats) {
  __shared__ double sums[3][16];
  double v[3] = {0, 0, 0};
#pragma unroll 8
  for (int64_t t = threadIdx.x; t < tokens; t += 1024)
#pragma unroll
    for (int q = 0; q < 3; ++q) v[q] += part[q * tokens + t];
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    v[q] = wave_sum(v[q]);
    if ((threadIdx.x & 63) == 0) sums[q][threadIdx.x >> 6] = v[q];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 0; q < 3; ++q) {
      v[q] = 0.0;
      for (int i = 0; i < 16; ++i) v[q] += sums[q][i];
    }
    stats[0] = float(kl_coef != 0.0f ? v[0] + double(kl_coef) * v[1] : v[0]);
    stats[1] = float(v[0]), stats[2] = float(v[1]), stats[3] = float(v[2]);
  }
}

template <class T, int THREADS, int NCH>
int launch_rows(Policy p, hipStream_t st) {
  constexpr int per = THREADS < 256 ? 256 / THREADS : 1, block = per * THREADS;
  constexpr int64_t most = kMostThreads / block * per;
  for (; p.first < p.tokens; p.first += most) {
    const int64_t rows = p.tokens - p.first < most ? p.tokens - p.first : most;
    k_policy<T, THREADS, NCH><<<unsigned((rows + per - 1) / per), block, 0, st>>>(p);
  }
  return launched();
}

// The fewest threads whose registers hold a row: 4 pieces of 16 bytes a thread where a row is a wavefront; 8 of 256 threads; 13 of
// 512, the most that leave six wavefronts a SIMD their registers (80); 16 of 1024.  Measured in us at each limit, 16 bits, with a gradient and
// without: 32768 rows of 2048 52 and 28, in 256 threads 72 and 46; 4096 rows of 16,384 48 and 24, in 512 threads 51 and 30; of 50,304 168 and
// 77, in 1024 threads 239 and 145 (in 512 with 16 pieces and four wavefronts a SIMD 159 and 87); of 131,072 545 and 281, read again
// 563 and 266.  So without a gradient, where nothing is read again, a row past 512 x 13 pieces is not kept either (100,000: 209, kept 237).
template <class T>
int launch_policy(const Policy& p, hipStream_t st) {
  const int64_t chunks = (p.vocab + kPer<T> - 1) / kPer<T>;
  if (chunks <= 64 * 4) return launch_rows<T, 64, 4>(p, st);
  if (chunks <= 256 * 8) return launch_rows<T, 256, 8>(p, st);
  if (chunks <= 512 * 13) return launch_rows<T, 512, 13>(p, st);
  if (chunks <= 1024 * 16 && p.dx) return launch_rows<T, 1024, 16>(p, st);
  return launch_rows<T, 1024, 0>(p, st);
}

constexpr int64_t kMost = int64_t(1) << 31;

}  // namespace

extern "C" {

size_t xmem_policy_loss_workspace_bytes(int64_t tokens, int64_t vocab) {
  if (tokens < 0 || tokens >= kMost || vocab < 0 || vocab >= kMost) return 0;
  return up256(size_t(tokens) * 12);
}

int xmem_policy_loss(const void* d_logits, int64_t ldl, const int64_t* d_tokens, const float* d_weights,
                     const float* d_old_logp, const float* d_advantages, const float* d_ref_logp, int64_t tokens,
                     int64_t vocab, int dtype, float clip_low, float clip_high, float kl_coef, float grad_scale,
                     float* d_stats, float* d_logp, void* d_dlogits, int64_t ldd, void* d_workspace,
                     size_t workspace_bytes, void* hip_stream) {
  if (tokens < 0 || tokens >= kMost || vocab < 1 || vocab >= kMost || dtype < XMEM_BF16 || dtype > XMEM_F32) return XMEM_EINVAL;
  if (ldl < vocab || ldl >= (int64_t(1) << 40) || (d_dlogits && (ldd < vocab || ldd >= (int64_t(1) << 40)))) return XMEM_EINVAL;
  if (!(clip_low >= 0.0f) || !(clip_high >= 0.0f)) return XMEM_EINVAL;
  const bool loss = d_old_logp || d_advantages || d_stats;
  if (loss ? (!d_stats || (tokens > 0 && (!d_old_logp || !d_advantages))) : (d_ref_logp || d_dlogits)) return XMEM_EINVAL;
  if (tokens > 0 && (!d_logits || !d_tokens || !d_logp)) return XMEM_EINVAL;
  if (d_dlogits == d_logits && d_dlogits && ldd != ldl) return XMEM_EINVAL;
  if (loss && tokens > 0 &&
      (!d_workspace || workspace_bytes < xmem_policy_loss_workspace_bytes(tokens, vocab) || !aligned(d_workspace, 256)))
    return XMEM_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  Policy p{d_logits, ldl, d_tokens, d_weights, d_old_logp, d_advantages, d_ref_logp, tokens, vocab, clip_low, clip_high, kl_coef,
           grad_scale, d_logp, d_dlogits, ldd, loss ? static_cast<float*>(d_workspace) : nullptr};
  if (tokens > 0) {
    const int rc = (dtype == XMEM_BF16 ? launch_policy<bf16> : dtype == XMEM_F16 ? launch_policy<f16> : launch_policy<float>)(p, st);
    if (rc != XMEM_OK) return rc;
  }
  if (loss) k_policy_sums<<<1, 1024, 0, st>>>(p.part, tokens, d_ref_logp ? kl_coef : 0.0f, d_stats);
  return launched();
}

}  // extern "C"
