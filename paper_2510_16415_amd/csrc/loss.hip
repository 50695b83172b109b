// Losses over token log-probabilities and their gradient with respect to every one of them: the preference loss of paired
// log ratios and the clipped policy loss with a KL term.  Tokens lie packed one sequence behind the other; `offsets` says where
// each begins, and a mask which tokens count.  A few bytes per token: the launches and the latency of the loads are what they
// take, so every sequence is cut into slices, a workgroup each, in two launches: one takes the sums that the gradient of a
// token depends on (its sequence's ratio, the number of counted tokens), the other the tokens' gradients.  Sums are held in 64
// bits, each added up in an order that only the sizes decide.
#include <math.h>

#include "../../include/mecefo.h"
#include "mecefo_internal.h"

namespace mecefo {
namespace {

constexpr int kThreads = 256;
constexpr int kSliceTokens = 2048;   // tokens of a slice, in a sequence of mean length
constexpr int kMaxSlices = 64;

struct Part { double sum; double count; };

struct Range { int64_t lo, hi; };
// Slice `j` of `n` of sequence `k`; offsets outside [0, tokens], or that decrease, give ranges inside it.
__device__ inline Range sequence(const int64_t* offsets, int64_t tokens, int k) {
  const int64_t a = offsets[k], b = offsets[k + 1];
  Range r;
  r.lo = a < 0 ? 0 : (a > tokens ? tokens : a);
  r.hi = b < r.lo ? r.lo : (b > tokens ? tokens : b);
  return r;
}
__device__ inline Range slice(Range r, int j, int n) {
  const int64_t len = r.hi - r.lo;
  return Range{r.lo + len * j / n, r.lo + len * (j + 1) / n};
}

__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// The sum over the workgroup, in every thread.
__device__ inline double block_sum(double v, double* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = red[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) s += red[w];
  return s;
}

// log(1 + exp(t)) without overflow; sigmoid.
__device__ inline double softplus(double t) { return (t > 0 ? t : 0.0) + log1p(exp(-fabs(t))); }
__device__ inline double sigmoid(double t) { return 1.0 / (1.0 + exp(-t)); }

struct PrefArgs {
  const float *logp, *ref;
  const uint8_t* mask;
  const int64_t* offsets;
  float *loss, *margins, *rewards, *dlogp;
  Part* parts;          // [2 * pairs][slices]
  int64_t tokens;
  int pairs, slices, mean;
  double beta, smooth, margin, grad_scale;
};

__device__ inline Part add_slices(const Part* p, int n) {
  Part s = {0.0, 0.0};
  for (int j = 0; j < n; ++j) { s.sum += p[j].sum; s.count += p[j].count; }
  return s;
}
// Sum over a slice of the counted tokens' log ratios, and how many there are.
__device__ inline Part ratio_sum(const PrefArgs& a, Range r) {
  Part s = {0.0, 0.0};
  for (int64_t t = r.lo + threadIdx.x; t < r.hi; t += blockDim.x) {
    const bool on = !a.mask || a.mask[t];
    const double x = (double)a.logp[t] - (a.ref ? (double)a.ref[t] : 0.0);
    s.sum += on ? x : 0.0;
    s.count += on ? 1.0 : 0.0;
  }
  return s;
}
// beta times the sum, or the mean, of the ratios of one sequence, and what one of its tokens contributes to that.
__device__ inline double reward(const PrefArgs& a, Part p, double* per_token) {
  *per_token = a.mean ? a.beta / (p.count > 1.0 ? p.count : 1.0) : a.beta;
  return p.sum * *per_token;
}
__device__ inline double pair_loss(const PrefArgs& a, double h) { return (1.0 - a.smooth) * softplus(-h) + a.smooth * softplus(h); }
__device__ inline double pair_slope(const PrefArgs& a, double h) { return a.smooth * sigmoid(h) - (1.0 - a.smooth) * sigmoid(-h); }

__global__ __launch_bounds__(kThreads) void preference_sums_kernel(const PrefArgs a) {
  __shared__ double red[kThreads / 64];
  const int k = blockIdx.x / a.slices, j = blockIdx.x - k * a.slices;
  const Part p = ratio_sum(a, slice(sequence(a.offsets, a.tokens, k), j, a.slices));
  const double sum = block_sum(p.sum, red), count = block_sum(p.count, red);
  if (threadIdx.x == 0) a.parts[blockIdx.x] = Part{sum, count};
}

// Zeros for the tokens in front of the first sequence and behind the last one.
__device__ inline void clear_outside(const int64_t* offsets, int64_t tokens, int n, float* dlogp) {
  const int64_t first = n > 0 ? sequence(offsets, tokens, 0).lo : tokens, last = n > 0 ? sequence(offsets, tokens, n - 1).hi : tokens;
  for (int64_t t = threadIdx.x; t < first; t += blockDim.x) dlogp[t] = 0.f;
  for (int64_t t = last + threadIdx.x; t < tokens; t += blockDim.x) dlogp[t] = 0.f;
}

// Workgroups 0 .. 2 * pairs * slices - 1: the gradients of a slice; the one behind them: the mean loss, every pair's margin and
// rewards, and the tokens of no sequence.
__global__ __launch_bounds__(kThreads) void preference_grad_kernel(const PrefArgs a) {
  __shared__ double red[kThreads / 64];
  const int grads = 2 * a.pairs * a.slices;
  if ((int)blockIdx.x == grads) {
    double total = 0.0;
    for (int i = threadIdx.x; i < a.pairs; i += kThreads) {
      double w;
      const double rc = reward(a, add_slices(a.parts + (int64_t)(2 * i) * a.slices, a.slices), &w);
      const double rr = reward(a, add_slices(a.parts + (int64_t)(2 * i + 1) * a.slices, a.slices), &w);
      const double h = rc - rr - a.margin;
      total += pair_loss(a, h);
      if (a.margins) a.margins[i] = (float)h;
      if (a.rewards) { a.rewards[2 * i] = (float)rc; a.rewards[2 * i + 1] = (float)rr; }
    }
    total = block_sum(total, red);
    if (threadIdx.x == 0) a.loss[0] = a.pairs > 0 ? (float)(total / a.pairs) : 0.f;
    clear_outside(a.offsets, a.tokens, 2 * a.pairs, a.dlogp);
    return;
  }
  const int k = blockIdx.x / a.slices, j = blockIdx.x - k * a.slices;
  double wc, wr;
  const int c = k & ~1;
  const double rc = reward(a, add_slices(a.parts + (int64_t)c * a.slices, a.slices), &wc);
  const double rr = reward(a, add_slices(a.parts + (int64_t)(c + 1) * a.slices, a.slices), &wr);
  const double slope = pair_slope(a, rc - rr - a.margin) * a.grad_scale / a.pairs;
  const float g = (float)(k & 1 ? -slope * wr : slope * wc);
  const Range r = slice(sequence(a.offsets, a.tokens, k), j, a.slices);
  for (int64_t t = r.lo + threadIdx.x; t < r.hi; t += kThreads) a.dlogp[t] = !a.mask || a.mask[t] ? g : 0.f;
}

struct PolicyArgs {
  const float *logp, *old, *ref, *advantage;
  const uint8_t* mask;
  const int64_t* offsets;
  float *loss, *kl, *clipped, *dlogp;
  double* counts;       // [sequences][slices]: counted tokens
  double* sums;         // [sequences * slices][3]: loss, KL, clipped tokens, weighted
  int64_t tokens;
  int seqs, slices, by_sequence, per_token;
  float low, high;              // bounds of the ratio
  double log_low, log_high;     // their logarithms
  float kl_coef, grad_scale;
};

__global__ __launch_bounds__(kThreads) void policy_counts_kernel(const PolicyArgs a) {
  __shared__ double red[kThreads / 64];
  const int k = blockIdx.x / a.slices, j = blockIdx.x - k * a.slices;
  const Range r = slice(sequence(a.offsets, a.tokens, k), j, a.slices);
  double n = 0.0;
  if (a.mask) {
    for (int64_t t = r.lo + threadIdx.x; t < r.hi; t += kThreads) n += a.mask[t] ? 1.0 : 0.0;
    n = block_sum(n, red);
  } else {
    n = (double)(r.hi - r.lo);
  }
  if (threadIdx.x == 0) a.counts[blockIdx.x] = n;
}

// exp(q) - q - 1, which is q^2 / 2 and more: the series where the difference would cancel.
__device__ inline float exp_excess(float q) {
  if (fabsf(q) > 0.5f) return expm1f(q) - q;
  float s = 1.f / 3628800.f;      // 1 / 10!; the term behind it is below 2^-24 of the first
  s = s * q + 1.f / 362880.f;
  s = s * q + 1.f / 40320.f;
  s = s * q + 1.f / 5040.f;
  s = s * q + 1.f / 720.f;
  s = s * q + 1.f / 120.f;
  s = s * q + 1.f / 24.f;
  s = s * q + 1.f / 6.f;
  s = s * q + 0.5f;
  return s * q * q;
}

__global__ __launch_bounds__(kThreads) void policy_grad_kernel(const PolicyArgs a) {
  __shared__ double red[kThreads / 64];
  const int grads = a.seqs * a.slices;
  if ((int)blockIdx.x == grads) return clear_outside(a.offsets, a.tokens, a.seqs, a.dlogp);
  const int k = blockIdx.x / a.slices, j = blockIdx.x - k * a.slices;
  // the weight of a counted token: 1 / all of them, or 1 / (those of its sequence x sequences that have any)
  double own = 0.0, n = 0.0;
  for (int i = 0; i < a.slices; ++i) own += a.counts[(int64_t)k * a.slices + i];
  for (int i = threadIdx.x; i < a.seqs; i += kThreads) {
    double c = 0.0;
    for (int q = 0; q < a.slices; ++q) c += a.counts[(int64_t)i * a.slices + q];
    n += a.by_sequence ? (c > 0.0 ? 1.0 : 0.0) : c;
  }
  n = block_sum(n, red);
  if (a.by_sequence) n *= own;
  const double w = n > 0.0 ? 1.0 / n : 0.0;
  const Range r = slice(sequence(a.offsets, a.tokens, k), j, a.slices);
  double loss = 0.0, kl = 0.0, clipped = 0.0;
  for (int64_t t = r.lo + threadIdx.x; t < r.hi; t += kThreads) {
    float g = 0.f;
    if (!a.mask || a.mask[t]) {
      const float A = a.advantage[a.per_token ? t : k];
      // which side of a bound the ratio lies on is decided by the difference itself, in 64 bits
      const double diff = (double)a.logp[t] - (double)a.old[t];
      const bool over = (A > 0.f && diff > a.log_high) || (A < 0.f && diff < a.log_low);
      const float rho = expf((float)diff);
      const float kept = over ? (A > 0.f ? a.high : a.low) : rho;
      float q = 0.f, excess = 0.f, slope = 0.f;
      if (a.ref) {
        q = (float)((double)a.ref[t] - (double)a.logp[t]);
        excess = exp_excess(q);
        slope = expm1f(q);
      }
      g = (float)w * a.grad_scale * ((over ? 0.f : -rho * A) - a.kl_coef * slope);
      loss += (double)(a.kl_coef * excess - kept * A);
      kl += (double)excess;
      clipped += over ? 1.0 : 0.0;
    }
    a.dlogp[t] = g;
  }
  loss = block_sum(loss, red);
  kl = block_sum(kl, red);
  clipped = block_sum(clipped, red);
  if (threadIdx.x == 0) {
    double* o = a.sums + (int64_t)blockIdx.x * 3;
    o[0] = loss * w; o[1] = kl * w; o[2] = clipped * w;
  }
}

__global__ __launch_bounds__(kThreads) void policy_total_kernel(const PolicyArgs a) {
  __shared__ double red[kThreads / 64];
  double s[3] = {0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < a.seqs * a.slices; i += kThreads)
    for (int q = 0; q < 3; ++q) s[q] += a.sums[(int64_t)i * 3 + q];
  for (int q = 0; q < 3; ++q) s[q] = block_sum(s[q], red);
  if (threadIdx.x == 0) {
    a.loss[0] = (float)s[0];
    if (a.kl) a.kl[0] = (float)s[1];
    if (a.clipped) a.clipped[0] = (float)s[2];
  }
}

int slices_of(int64_t tokens, int64_t sequences) {
  const int64_t mean = sequences > 0 ? tokens / sequences : 0;
  const int64_t n = (mean + kSliceTokens - 1) / kSliceTokens;
  return (int)(n < 1 ? 1 : n > kMaxSlices ? kMaxSlices : n);
}

mecefo_status_t check_sizes(int64_t tokens, int64_t sequences) {
  if (tokens < 0 || sequences < 0) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "tokens and the number of sequences must be >= 0");
  if (tokens * 4 >= (int64_t)1 << 31 || sequences > 1 << 20) return (mecefo_status_t)fail(MECEFO_ERR_UNSUPPORTED, "a token array reaches 2 GiB, or there are more than 2^20 sequences");
  return MECEFO_OK;
}
mecefo_status_t check_align(const void* p, const char* name, int align, bool required) {
  if (!p) return required ? (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "%s is NULL", name) : MECEFO_OK;
  if ((uintptr_t)p % align) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "%s is not %d-byte aligned", name, align);
  return MECEFO_OK;
}
mecefo_status_t check(const mecefo_preference_desc_t* d) {
  if (!d) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "descriptor is NULL");
  const mecefo_status_t st = check_sizes(d->tokens, (int64_t)d->pairs * 2);
  if (st != MECEFO_OK) return st;
  if (!isfinite(d->beta) || !isfinite(d->margin) || !isfinite(d->grad_scale)) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "beta, margin and grad_scale must be finite");
  if (!(d->label_smoothing >= 0.f && d->label_smoothing <= 1.f)) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "label_smoothing must be in [0, 1]");
  return MECEFO_OK;
}
mecefo_status_t check(const mecefo_policy_desc_t* d) {
  if (!d) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "descriptor is NULL");
  const mecefo_status_t st = check_sizes(d->tokens, d->sequences);
  if (st != MECEFO_OK) return st;
  if (!(d->clip_low >= 0.f && d->clip_low <= 1.f) || !(d->clip_high >= 0.f && isfinite(d->clip_high)))
    return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "clip_low must be in [0, 1], clip_high finite and >= 0");
  if (!isfinite(d->kl_coef) || !isfinite(d->grad_scale)) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "kl_coef and grad_scale must be finite");
  if (d->mean != MECEFO_MEAN_TOKENS && d->mean != MECEFO_MEAN_SEQUENCES) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "mean must be MECEFO_MEAN_TOKENS or MECEFO_MEAN_SEQUENCES");
  return MECEFO_OK;
}
mecefo_status_t check_ws(size_t need, const void* ws, size_t ws_bytes) {
  if (need > ws_bytes) return (mecefo_status_t)fail(MECEFO_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu needed", ws_bytes, need);
  if (!ws) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "workspace is NULL");
  return MECEFO_OK;
}
void* aligned(void* ws) { return (void*)(((uintptr_t)ws + 255) / 256 * 256); }

size_t preference_bytes(const mecefo_preference_desc_t* d) {
  return (size_t)2 * d->pairs * slices_of(d->tokens, (int64_t)d->pairs * 2) * sizeof(Part) + 256;
}
size_t policy_bytes(const mecefo_policy_desc_t* d) { return (size_t)d->sequences * slices_of(d->tokens, d->sequences) * 4 * sizeof(double) + 256; }

}  // namespace
}  // namespace mecefo

using namespace mecefo;

#define TRY(x) do { mecefo_status_t st__ = (x); if (st__ != MECEFO_OK) return st__; } while (0)
#define LAUNCHED(what) do { hipError_t e__ = hipGetLastError(); if (e__ != hipSuccess) return (mecefo_status_t)fail(MECEFO_ERR_LAUNCH, "%s: %s", what, hipGetErrorString(e__)); } while (0)

extern "C" {

mecefo_status_t mecefo_preference_workspace_bytes(const mecefo_preference_desc_t* desc, size_t* out_bytes) {
  TRY(check(desc));
  if (!out_bytes) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "out_bytes is NULL");
  *out_bytes = preference_bytes(desc);
  return MECEFO_OK;
}

mecefo_status_t mecefo_preference_loss(const mecefo_preference_desc_t* desc, const float* logp, const float* ref_logp,
                                       const uint8_t* mask, const int64_t* offsets, float* loss, float* margins,
                                       float* rewards, float* dlogp, void* ws, size_t ws_bytes, void* hip_stream) {
  TRY(check(desc));
  const bool any = desc->tokens > 0;
  TRY(check_align(logp, "logp", 4, any)); TRY(check_align(ref_logp, "ref_logp", 4, false));
  TRY(check_align(offsets, "offsets", 8, desc->pairs > 0)); TRY(check_align(loss, "loss", 4, true));
  TRY(check_align(margins, "margins", 4, false)); TRY(check_align(rewards, "rewards", 4, false));
  TRY(check_align(dlogp, "dlogp", 4, any));
  TRY(check_ws(preference_bytes(desc), ws, ws_bytes));
  hipStream_t s = (hipStream_t)hip_stream;
  const int slices = slices_of(desc->tokens, (int64_t)desc->pairs * 2), grads = 2 * desc->pairs * slices;
  const PrefArgs a = {logp, ref_logp, mask, offsets, loss, margins, rewards, dlogp, (Part*)aligned(ws), desc->tokens, desc->pairs,
                      slices, desc->length_mean, desc->beta, desc->label_smoothing, desc->margin, desc->grad_scale};
  if (grads > 0) {
    hipLaunchKernelGGL(preference_sums_kernel, dim3(grads), dim3(kThreads), 0, s, a);
    LAUNCHED("preference_loss");
  }
  hipLaunchKernelGGL(preference_grad_kernel, dim3(grads + 1), dim3(kThreads), 0, s, a);
  LAUNCHED("preference_loss");
  return MECEFO_OK;
}

mecefo_status_t mecefo_policy_workspace_bytes(const mecefo_policy_desc_t* desc, size_t* out_bytes) {
  TRY(check(desc));
  if (!out_bytes) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "out_bytes is NULL");
  *out_bytes = policy_bytes(desc);
  return MECEFO_OK;
}

mecefo_status_t mecefo_policy_loss(const mecefo_policy_desc_t* desc, const float* logp, const float* old_logp,
                                   const float* ref_logp, const float* advantage, const uint8_t* mask, const int64_t* offsets,
                                   float* loss, float* kl, float* clipped, float* dlogp, void* ws, size_t ws_bytes,
                                   void* hip_stream) {
  TRY(check(desc));
  const bool any = desc->tokens > 0;
  TRY(check_align(logp, "logp", 4, any)); TRY(check_align(old_logp, "old_logp", 4, any)); TRY(check_align(ref_logp, "ref_logp", 4, false));
  TRY(check_align(advantage, "advantage", 4, any && desc->sequences > 0)); TRY(check_align(offsets, "offsets", 8, desc->sequences > 0));
  TRY(check_align(loss, "loss", 4, true)); TRY(check_align(kl, "kl", 4, false)); TRY(check_align(clipped, "clipped", 4, false));
  TRY(check_align(dlogp, "dlogp", 4, any));
  if (!ref_logp && desc->kl_coef != 0.f) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "kl_coef needs ref_logp");
  TRY(check_ws(policy_bytes(desc), ws, ws_bytes));
  hipStream_t s = (hipStream_t)hip_stream;
  const int slices = slices_of(desc->tokens, desc->sequences), grads = desc->sequences * slices;
  double* counts = (double*)aligned(ws);
  const PolicyArgs a = {logp, old_logp, ref_logp, advantage, mask, offsets, loss, kl, clipped, dlogp, counts, counts + grads,
                        desc->tokens, desc->sequences, slices, desc->mean == MECEFO_MEAN_SEQUENCES, desc->advantage_per_token,
                        (float)(1.0 - (double)desc->clip_low), (float)(1.0 + (double)desc->clip_high), log1p(-(double)desc->clip_low),
                        log1p((double)desc->clip_high), desc->kl_coef, desc->grad_scale};
  if (grads > 0) {
    hipLaunchKernelGGL(policy_counts_kernel, dim3(grads), dim3(kThreads), 0, s, a);
    LAUNCHED("policy_loss");
  }
  hipLaunchKernelGGL(policy_grad_kernel, dim3(grads + 1), dim3(kThreads), 0, s, a);
  LAUNCHED("policy_loss");
  hipLaunchKernelGGL(policy_total_kernel, dim3(1), dim3(kThreads), 0, s, a);
  LAUNCHED("policy_loss");
  return MECEFO_OK;
}

}  // extern "C"
