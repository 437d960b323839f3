// policy.hip -- the clipped policy loss with a KL term over a vocabulary, on MI355X (gfx950).
#include "common.h"

using namespace xops;

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;

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
};

// (largest, sum of exp(. - largest)) of two sets of logits; the largest of no logits is -inf.
__device__ inline void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  s = (m == top ? s : s * __expf(m - top)) + (m2 == top ? s2 : s2 * __expf(m2 - top));
  m = top;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_policy(Policy p) {
  __shared__ float sm[kWaves], ss[kWaves];
  const int64_t t = blockIdx.x;
  const float wt = p.w ? p.w[t] : 1.0f / float(p.tokens);
  const T* x = static_cast<const T*>(p.x) + t * p.ldl;
  T* dx = p.dx ? static_cast<T*>(p.dx) + t * p.ldd : nullptr;
  if (wt == 0.0f) {
    if (dx)
      for (int64_t j = threadIdx.x; j < p.vocab; j += kThreads) dx[j] = T(0.0f);
    if (threadIdx.x == 0) {
      p.lp[t] = 0.0f;
      if (p.part) p.part[t] = p.part[p.tokens + t] = p.part[2 * p.tokens + t] = 0.0f;
    }
    return;
  }
  float m = -INFINITY, s = 0.0f;
  bool nan = false;
  for (int64_t j = threadIdx.x; j < p.vocab; j += kThreads) {
    const float v = float(x[j]);
    nan |= v != v;
    if (v > m) s = s * __expf(m - v), m = v;
    if (v > -INFINITY) s += __expf(v - m);
  }
  if (nan) m = INFINITY, s = NAN;
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const float m2 = __shfl_xor(m, d), s2 = __shfl_xor(s, d);
    join(m, s, m2, s2);
  }
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m, ss[threadIdx.x >> 6] = s;
  const int64_t y = p.y[t];
  const bool in = y >= 0 && y < p.vocab;
  const float xy = in ? float(x[in ? y : 0]) : NAN;  // before the row may be overwritten
  __syncthreads();
  m = sm[0], s = ss[0];
  for (int i = 1; i < kWaves; ++i) join(m, s, sm[i], ss[i]);
  const float lp = (xy - m) - logf(s);
  float grad = 0.0f;
  if (p.old_lp) {
    const float adv = p.adv[t], rho = expf(lp - p.old_lp[t]);
    const float free = rho * adv, held = fminf(fmaxf(rho, 1.0f - p.low), 1.0f + p.high) * adv;
    const bool clipped = held < free;
    float kl = 0.0f;
    grad = clipped ? 0.0f : -free;
    if (p.ref) {
      const float d = p.ref[t] - lp, e = expm1f(d);
      kl = e - d;
      grad -= p.kl_coef * e;
    }
    grad *= wt;
    if (threadIdx.x == 0) {
      p.part[t] = wt * -(clipped ? held : free);
      p.part[p.tokens + t] = wt * kl;
      p.part[2 * p.tokens + t] = clipped ? wt : 0.0f;
    }
  }
  if (threadIdx.x == 0) p.lp[t] = lp;
  if (!dx) return;
  grad *= p.grad_scale;
  const float per = grad / s;
  for (int64_t j = threadIdx.x; j < p.vocab; j += kThreads) {
    const float v = float(x[j]);
    dx[j] = T((j == y ? grad : 0.0f) - per * __expf(v - m));
  }
}

__global__ __launch_bounds__(1024) void k_policy_sums(const float* part, int64_t tokens, float kl_coef, float* stats) {
  __shared__ double sums[3][16];
  for (int q = 0; q < 3; ++q) {
    double v = 0.0;
    for (int64_t t = threadIdx.x; t < tokens; t += 1024) v += part[q * tokens + t];
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) sums[q][threadIdx.x >> 6] = v;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double v[3] = {0, 0, 0};
    for (int q = 0; q < 3; ++q)
      for (int i = 0; i < 16; ++i) v[q] += sums[q][i];
    stats[0] = float(v[0] + double(kl_coef) * v[1]);
    stats[1] = float(v[0]), stats[2] = float(v[1]), stats[3] = float(v[2]);
  }
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
  if (tokens > 0)
    (dtype == XMEM_BF16 ? k_policy<bf16> : dtype == XMEM_F16 ? k_policy<f16> : k_policy<float>)<<<unsigned(tokens), kThreads, 0, st>>>(p);
  if (loss) k_policy_sums<<<1, 1024, 0, st>>>(p.part, tokens, d_ref_logp ? kl_coef : 0.0f, d_stats);
  return launched();
}

}  // extern "C"
