// Losses over token log-probabilities and their gradient with respect to every one of them: the preference loss of paired
// log ratios and the clipped policy loss with a KL term.  Tokens lie packed one sequence behind the other; `offsets` says where
// each begins, and a mask which tokens count.  A few bytes per token: the launches and the latency of the loads are what they
// take, so every sequence is cut into slices, a workgroup each, in two launches: one takes the sums that the gradient of a
// token depends on (its sequence's ratio, the number of counted tokens), the other the tokens' gradients.  A small batch is one
// workgroup's, and one launch's; a policy batch of many sequences has a launch in between.  Sums are held in 64 bits, each added up
// in an order that only the sizes decide; exponentials of the policy in 32 bits where they hold them, else in 64.
#include <math.h>

#include <type_traits>

#include "../../include/mecefo.h"
#include "loss_ranges.h"
#include "mecefo_internal.h"

namespace mecefo {
namespace {

constexpr int kThreads = 256;
// Slices of a sequence of mean length: of 512 tokens or more, and about four workgroups a CU.  Preference / policy with slices of
// 512 / 1024 / 2048 tokens, us: 128 sequences of 4096 tokens 10.8, 12.9 / 12.1, 14.8 / 17.9, 22.1; 512 of 2048 14.9, 20.4 / 14.0, 19.2 /
// 18.8, 24.0; 8 of 1000 6.9, 8.7 / 8.3, 9.8 / 8.4, 9.8.
constexpr int kSliceTokens = 512;
constexpr int kMaxSlices = 256;
constexpr int kRowSlices = 16;       // from here on 16 lanes add up a sequence's slices, below a thread does
constexpr int kRowSeqs = 128;        // batches of so many slices have about 4 * kCUs / (kRowSlices - 1) sequences at most
// One workgroup and one launch: a wave to a sequence.  GPU time of one launch / two, us: preference 8 x 64 tokens 6.0 / 6.6, 8 x 250
// 7.5 / 6.6, 64 x 16 13.1 / 6.7, 512 x 8 72 / 7.7; policy 2 x 100 8.1 / 7.5.  Calls that a program makes one by one, the launches among
// them: preference 2 x 20 to 16 x 32 7.6 to 8.1 / 11.4, policy 8.0 to 10 / 11.5.
constexpr int kSmallTokens = 512, kSmallSeqs = 16;

constexpr int kClearTokens = 16384;

// Batches of more sequences have their counts and sums added up by a launch in between: every workgroup of the second launch needs
// the count over all, and reading all counts there is quadratic in the sequences.  Without / with that launch, means over tokens, over
// sequences, us: 1800 sequences of 8 tokens 18, 21 / 22, 22; 3000 25, 31 / 24, 25; 8192 60, 82 / 42, 43; 32768 358, 578 / 124, 132; with it
// 1048576 3790, 4040.
constexpr int kGatherFrom = 2048;
constexpr int kGathered = 256;       // workgroups of that launch at most

struct Part { double sum; double count; };

__device__ inline TokenRange sequence(const int64_t* offsets, int64_t tokens, int k) { return token_range(offsets[k], offsets[k + 1], tokens); }

// Calls f(token, loaded values) for the tokens t0, t0 + stride, ... of a range, kAhead of them loaded before the first is used:
// a few bytes a token, so the time is that of the loads' latency.
constexpr int kAhead = 4;
template <class Load, class Use>
__device__ inline void for_tokens(TokenRange r, int first, int stride, Load load, Use use) {
  for (int64_t t = r.lo + first; t < r.hi; t += (int64_t)kAhead * stride) {
    decltype(load(t)) v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = load(t + (int64_t)u * stride < r.hi ? t + (int64_t)u * stride : t);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (t + (int64_t)u * stride < r.hi) use(t + (int64_t)u * stride, v[u]);
  }
}

__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// Sums over the workgroup, in every thread.
template <int N>
__device__ inline void block_sums(double (&v)[N]) {
  __shared__ double red[16][N];
#pragma unroll
  for (int q = 0; q < N; ++q) v[q] = wave_sum(v[q]);
  __syncthreads();
  if ((threadIdx.x & 63) == 0)
    for (int q = 0; q < N; ++q) red[threadIdx.x >> 6][q] = v[q];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < N; ++q) {
    v[q] = red[0][q];
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v[q] += red[w][q];
  }
}
__device__ inline double block_sum(double x) {
  double v[1] = {x};
  block_sums(v);
  return v[0];
}

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

// The slices of one sequence added up by a wave or by 16 lanes, in all of them, or by a thread.
__device__ inline Part wave_slices(const Part* p, int n) {
  Part s = {0.0, 0.0};
  for (int j = threadIdx.x & 63; j < n; j += 64) { s.sum += p[j].sum; s.count += p[j].count; }
  return Part{wave_sum(s.sum), wave_sum(s.count)};
}
__device__ inline Part row_slices(const Part* p, int n) {
  Part s = {0.0, 0.0};
#pragma unroll 4
  for (int j = threadIdx.x & 15; j < n; j += 16) { const Part x = p[j]; s.sum += x.sum; s.count += x.count; }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) { s.sum += __shfl_xor(s.sum, o, 64); s.count += __shfl_xor(s.count, o, 64); }
  return s;
}
__device__ inline Part thread_slices(const Part* p, int n) {
  Part s = {0.0, 0.0};
#pragma unroll 4
  for (int j = 0; j < n; ++j) { const Part x = p[j]; s.sum += x.sum; s.count += x.count; }
  return s;
}
// Sum over a range of the counted tokens' log ratios, and how many there are, a thread's share.
struct Ratio { float logp, ref; uint8_t on; };
__device__ inline Part ratio_sum(const PrefArgs& a, TokenRange r, int first, int stride) {
  Part s = {0.0, 0.0};
  for_tokens(r, first, stride,
             [&](int64_t t) { return Ratio{a.logp[t], a.ref ? a.ref[t] : 0.f, a.mask ? a.mask[t] : (uint8_t)1}; },
             [&](int64_t, const Ratio& x) {
               s.sum += x.on ? (double)x.logp - (double)x.ref : 0.0;
               s.count += x.on ? 1.0 : 0.0;
             });
  return s;
}
// The gradients of a range: g(), which may take a while, is asked for once the first tokens' masks are on their way.
template <class G>
__device__ inline void write_gradients(const PrefArgs& a, TokenRange r, int first, int stride, G g) {
  const int64_t t0 = r.lo + first;
  uint8_t on[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) on[u] = a.mask && t0 + (int64_t)u * stride < r.hi ? a.mask[t0 + (int64_t)u * stride] : (uint8_t)1;
  const float v = g();
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (t0 + (int64_t)u * stride < r.hi) a.dlogp[t0 + (int64_t)u * stride] = on[u] ? v : 0.f;
  for_tokens(r, first + kAhead * stride, stride, [&](int64_t t) { return a.mask ? a.mask[t] : (uint8_t)1; },
             [&](int64_t t, uint8_t m) { a.dlogp[t] = m ? v : 0.f; });
}
// beta times the sum, or the mean, of the ratios of one sequence, and what one of its tokens contributes to that.
__device__ inline double reward(const PrefArgs& a, Part p, double* per_token) {
  *per_token = a.mean ? a.beta / (p.count > 1.0 ? p.count : 1.0) : a.beta;
  return p.sum * *per_token;
}
// A pair's loss and its slope in h, from one exponential: softplus(t) = max(t, 0) + log1p(exp(-|t|)).
struct PairLoss { double loss, slope; };
__device__ inline PairLoss pair_loss(const PrefArgs& a, double h) {
  const double e = exp(-fabs(h)), l = log1p(e), s = 1.0 / (1.0 + e), up = h >= 0 ? s : e * s, down = h >= 0 ? e * s : s;
  return PairLoss{(1.0 - a.smooth) * ((h < 0 ? -h : 0.0) + l) + a.smooth * ((h > 0 ? h : 0.0) + l), a.smooth * up - (1.0 - a.smooth) * down};
}

__global__ __launch_bounds__(kThreads) void preference_sums_kernel(const PrefArgs a) {
  const int k = blockIdx.x / a.slices, j = blockIdx.x - k * a.slices;
  const Part p = ratio_sum(a, token_slice(sequence(a.offsets, a.tokens, k), j, a.slices), threadIdx.x, kThreads);
  double v[2] = {p.sum, p.count};
  block_sums(v);
  if (threadIdx.x == 0) a.parts[blockIdx.x] = Part{v[0], v[1]};
}

// Zeros for the tokens in front of the first sequence and behind the last one, workgroup `at` of `of`.
__device__ inline void clear_outside(const int64_t* offsets, int64_t tokens, int n, float* dlogp, int at, int of) {
  const int64_t first = n > 0 ? sequence(offsets, tokens, 0).lo : tokens, last = n > 0 ? sequence(offsets, tokens, n - 1).hi : tokens;
  const int64_t t0 = (int64_t)at * blockDim.x + threadIdx.x, stride = (int64_t)of * blockDim.x;
  for (int64_t t = t0; t < first; t += stride) dlogp[t] = 0.f;
  for (int64_t t = last + t0; t < tokens; t += stride) dlogp[t] = 0.f;
}

// Workgroups 0 .. 2 * pairs * slices - 1: the gradients of a slice; the one behind them: the mean loss, every pair's margin and
// rewards; the last ones: the tokens of no sequence.  The one takes a thread to a pair (64 pairs of 4
// slices: the launch 28 us with a wave to a pair, 6 with a thread), and 16 lanes to a sequence first where it has many slices (32 pairs of 16
// slices: the call 28.6 us with a wave to a pair, 18.5).
__global__ __launch_bounds__(kThreads) void preference_grad_kernel(const PrefArgs a) {
  const int grads = 2 * a.pairs * a.slices;
  if ((int)blockIdx.x == grads) {
    double total = 0.0;
    auto pair = [&](int i, const Part& chosen, const Part& other) {
      double w;
      const double rc = reward(a, chosen, &w), rr = reward(a, other, &w), h = rc - rr - a.margin;
      total += pair_loss(a, h).loss;
      if (a.margins) a.margins[i] = (float)h;
      if (a.rewards) { a.rewards[2 * i] = (float)rc; a.rewards[2 * i + 1] = (float)rr; }
    };
    const Part* parts = a.parts;
    const int n = a.slices;
    if (n >= kRowSlices && 2 * a.pairs <= kRowSeqs) {
      __shared__ Part sums[kRowSeqs];
      for (int k = threadIdx.x >> 4; k < 2 * a.pairs; k += kThreads / 16) {
        const Part p = row_slices(parts + (int64_t)k * n, n);
        if ((threadIdx.x & 15) == 0) sums[k] = p;
      }
      __syncthreads();
      if ((int)threadIdx.x < a.pairs) pair(threadIdx.x, sums[2 * threadIdx.x], sums[2 * threadIdx.x + 1]);
    } else {
      for (int i = threadIdx.x; i < a.pairs; i += kThreads)
        pair(i, thread_slices(parts + (int64_t)(2 * i) * n, n), thread_slices(parts + (int64_t)(2 * i + 1) * n, n));
    }
    total = block_sum(total);
    if (threadIdx.x == 0) a.loss[0] = a.pairs > 0 ? (float)(total / a.pairs) : 0.f;
    return;
  }
  if ((int)blockIdx.x > grads) return clear_outside(a.offsets, a.tokens, 2 * a.pairs, a.dlogp, blockIdx.x - grads - 1, gridDim.x - grads - 1);
  const int k = blockIdx.x / a.slices, j = blockIdx.x - k * a.slices;
  const TokenRange r = token_slice(sequence(a.offsets, a.tokens, k), j, a.slices);
  write_gradients(a, r, threadIdx.x, kThreads, [&]() {
    double wc, wr;
    const int c = k & ~1;
    const Part pc = wave_slices(a.parts + (int64_t)c * a.slices, a.slices), pr = wave_slices(a.parts + (int64_t)(c + 1) * a.slices, a.slices);
    const double rc = reward(a, pc, &wc), rr = reward(a, pr, &wr);
    const double g = pair_loss(a, rc - rr - a.margin).slope * a.grad_scale / a.pairs;
    return (float)(k & 1 ? -g * wr : g * wc);
  });
}

// A small batch in one workgroup and one launch: a wave to a sequence, the sums in LDS.
__global__ __launch_bounds__(1024) void preference_small_kernel(const PrefArgs a) {
  __shared__ Part parts[kSmallSeqs];
  __shared__ float slope[kSmallSeqs];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int k = wave; k < 2 * a.pairs; k += 16) {
    const Part p = ratio_sum(a, sequence(a.offsets, a.tokens, k), lane, 64);
    const double sum = wave_sum(p.sum), count = wave_sum(p.count);
    if (lane == 0) parts[k] = Part{sum, count};
  }
  __syncthreads();
  double total = 0.0;
  for (int i = threadIdx.x; i < a.pairs; i += 1024) {
    double wc, wr;
    const double rc = reward(a, parts[2 * i], &wc), rr = reward(a, parts[2 * i + 1], &wr), h = rc - rr - a.margin;
    const PairLoss l = pair_loss(a, h);
    const double g = l.slope * a.grad_scale / a.pairs;
    slope[2 * i] = (float)(g * wc);
    slope[2 * i + 1] = (float)(-g * wr);
    total += l.loss;
    if (a.margins) a.margins[i] = (float)h;
    if (a.rewards) { a.rewards[2 * i] = (float)rc; a.rewards[2 * i + 1] = (float)rr; }
  }
  total = block_sum(total);      // and its barriers: the slopes are written
  if (threadIdx.x == 0) a.loss[0] = a.pairs > 0 ? (float)(total / a.pairs) : 0.f;
  for (int k = wave; k < 2 * a.pairs; k += 16) write_gradients(a, sequence(a.offsets, a.tokens, k), lane, 64, [&]() { return slope[k]; });
  clear_outside(a.offsets, a.tokens, 2 * a.pairs, a.dlogp, 0, 1);
}

struct PolicySums { double loss, kl, clipped; uint32_t count; };      // without the tokens' weights

struct PolicyArgs {
  const float *logp, *old, *ref, *advantage;
  const uint8_t* mask;
  const int64_t* offsets;
  float *loss, *kl, *clipped, *dlogp;
  double* sums;         // [3][sequences * slices]: loss, KL, clipped tokens
  uint32_t* counts;     // [sequences][slices]: counted tokens
  double* gathered;     // [4][groups]: of a range of sequences the count for the weights; loss, KL, clipped tokens without the common part of their weights
  int groups;           // 0: nothing is gathered
  int64_t tokens;
  int seqs, slices, by_sequence, per_token;
  double low, high, log_low, log_high;      // bounds of the ratio, and their logarithms
  float kl_coef, grad_scale;
};

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

struct PolicyToken { float logp, old, ref, A; uint8_t on; };
__device__ inline PolicyToken policy_token(const PolicyArgs& a, int64_t t, int k) {
  return PolicyToken{a.logp[t], a.old[t], a.ref ? a.ref[t] : 0.f, a.advantage[a.per_token ? t : k], a.mask ? a.mask[t] : (uint8_t)1};
}
// Which side of a bound the ratio lies on is decided by the difference itself, in 64 bits.
__device__ inline bool policy_over(const PolicyArgs& a, float A, double diff) {
  return (A > 0.f && diff > a.log_high) || (A < 0.f && diff < a.log_low);
}

// A counted token's terms where fp32 does not hold one of them: exp(88.8) is beyond it.  An exponential that fp32 holds is taken as
// the other tokens have it; the others stay below infinity, so that a ratio without an advantage and a KL term without a
// coefficient are zero at any distance.
struct PolicyTerms { double loss, kl, grad; };
__device__ inline PolicyTerms policy_far(const PolicyArgs& a, const PolicyToken& x) {
  auto power = [](double v) {      // a NaN stays one
    const float near = expf((float)v);
    const double far = near < INFINITY ? (double)near : exp(v);
    return far > 1.7976931348623157e308 ? 1.7976931348623157e308 : far;
  };
  const double diff = (double)x.logp - (double)x.old, A = x.A, q = a.ref ? (double)x.ref - (double)x.logp : 0.0;
  const bool over = policy_over(a, x.A, diff);
  const double rho = power(diff), kept = over ? (x.A > 0.f ? a.high : a.low) : rho;
  const float near = exp_excess((float)q);
  const double excess = near < INFINITY ? (double)near : power(q) - 1.0 - q;      // |q| is large
  return PolicyTerms{a.kl_coef * excess - kept * A, excess, a.grad_scale * ((over ? 0.0 : -rho * A) - a.kl_coef * (q + excess))};
}

// The tokens of a range: their gradients without the weight, and a thread's share of the sums.
__device__ inline PolicySums policy_tokens(const PolicyArgs& a, TokenRange r, int first, int stride, int k) {
  PolicySums s = {0.0, 0.0, 0.0, 0};
  bool far = false;      // of some tokens fp32 does not hold a term: they get a NaN, and their turn behind the loop
  for_tokens(r, first, stride, [&](int64_t t) { return policy_token(a, t, k); },
             [&](int64_t t, const PolicyToken& x) {
               float g = 0.f;
               if (x.on) {
                 const double diff = (double)x.logp - (double)x.old;
                 const bool over = policy_over(a, x.A, diff);
                 const float rho = expf((float)diff);
                 const double kept = over ? (x.A > 0.f ? a.high : a.low) : (double)rho;
                 const float q = a.ref ? (float)((double)x.ref - (double)x.logp) : 0.f, excess = exp_excess(q);
                 g = a.grad_scale * ((over ? 0.f : -rho * x.A) - a.kl_coef * (q + excess));      // exp(q) - 1
                 if (rho + excess + fabsf(g) < INFINITY) {
                   s.loss += (double)a.kl_coef * excess - kept * x.A;      // the clipped terms are all of one size: a rounding of it would add up
                   s.kl += (double)excess;
                 } else {
                   g = __builtin_nanf("");
                   far = true;
                 }
                 s.clipped += over ? 1.0 : 0.0;
                 s.count += 1;
               }
               a.dlogp[t] = g;
             });
  if (far)
#pragma unroll 1
    for (int64_t t = r.lo + first; t < r.hi; t += stride)
      if (isnan(a.dlogp[t])) {
        const PolicyTerms f = policy_far(a, policy_token(a, t, k));
        a.dlogp[t] = (float)f.grad;
        s.loss += f.loss;
        s.kl += f.kl;
      }
  return s;
}
// What the tokens' weights are made of: over all sequences their counted tokens, or how many have any (by_sequence).
__device__ inline double share(const PolicyArgs& a, double count) { return a.by_sequence ? (count > 0.0 ? 1.0 : 0.0) : count; }
// The weight of a counted token: 1 / all of them, or 1 / (those of its sequence x sequences that have any).
__device__ inline double token_weight(const PolicyArgs& a, double n, double own) {
  const double c = a.by_sequence ? n * own : n;
  return c > 0.0 ? 1.0 / c : 0.0;
}
// A gradient without the weight that is beyond fp32 may be back in it with the weight: it is formed again in 64 bits.
template <class W>
__device__ inline void scale_gradients(const PolicyArgs& a, TokenRange r, int first, int stride, int k, W weight) {
  const int64_t t0 = r.lo + first;
  float g[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) g[u] = t0 + (int64_t)u * stride < r.hi ? a.dlogp[t0 + (int64_t)u * stride] : 0.f;
  const double weight64 = weight();
  const float w = (float)weight64;
  bool far = false;
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (t0 + (int64_t)u * stride < r.hi) {
      far |= isinf(g[u]);
      a.dlogp[t0 + (int64_t)u * stride] = g[u] * w;
    }
  for_tokens(r, first + kAhead * stride, stride, [&](int64_t t) { return a.dlogp[t]; },
             [&](int64_t t, float x) {
               far |= isinf(x);
               a.dlogp[t] = x * w;
             });
  if (far)
#pragma unroll 1
    for (int64_t t = t0; t < r.hi; t += stride)
      if (isinf(a.dlogp[t])) a.dlogp[t] = (float)(policy_far(a, policy_token(a, t, k)).grad * weight64);
}
__device__ inline void policy_results(const PolicyArgs& a, double loss, double kl, double clipped) {
  a.loss[0] = (float)loss;
  if (a.kl) a.kl[0] = (float)kl;
  if (a.clipped) a.clipped[0] = (float)clipped;
}

// The first launch computes everything but the weight, which needs the count of all tokens, the second one scales: 8 bytes a
// token more than counting first and computing then, but the longer launch has nothing to wait for.  1048576 tokens: 19 us
// where a count, the gradients and a sum of the sums took 29, and 40 where the last workgroup of the gradients summed up
// (its device-scope ordering writes caches back).
__global__ __launch_bounds__(kThreads) void policy_tokens_kernel(const PolicyArgs a) {
  const int k = blockIdx.x / a.slices, j = blockIdx.x - k * a.slices;
  const PolicySums s = policy_tokens(a, token_slice(sequence(a.offsets, a.tokens, k), j, a.slices), threadIdx.x, kThreads, k);
  const int64_t n = (int64_t)a.seqs * a.slices;
  double t[4] = {s.loss, s.kl, s.clipped, (double)s.count};
  block_sums(t);
  if (threadIdx.x != 0) return;
  for (int q = 0; q < 3; ++q) a.sums[q * n + blockIdx.x] = t[q];
  a.counts[blockIdx.x] = (uint32_t)t[3];
}

// Between the two where there are many sequences, which are short then: a slice each.  A workgroup adds up a range of them, a thread to a sequence.
__global__ __launch_bounds__(kThreads) void policy_gather_kernel(const PolicyArgs a) {
  const int per = (a.seqs + a.groups - 1) / a.groups, lo = blockIdx.x * per, hi = min(lo + per, a.seqs);
  double t[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 2
  for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
    const double own = a.counts[i], w = a.by_sequence ? (own > 0.0 ? 1.0 / own : 0.0) : 1.0;
    t[0] += share(a, own);
    for (int m = 0; m < 3; ++m) t[m + 1] += a.sums[(int64_t)m * a.seqs + i] * w;
  }
  block_sums(t);
  if (threadIdx.x == 0)
    for (int m = 0; m < 4; ++m) a.gathered[m * a.groups + blockIdx.x] = t[m];
}

// Workgroup seqs * slices: the results; those behind it: the tokens of no sequence.  Sequences of many slices are added up by 16
// lanes each, where there are no more than four by a wave each (means over sequences, us, a wave each / this: 64 sequences of 16000 tokens 41.5 / 22.5, 16 of
// 60000 23.4 / 18.4, 2 of 200000 15.2 / 13.5).
__global__ __launch_bounds__(kThreads) void policy_scale_kernel(const PolicyArgs a) {
  const int grads = a.seqs * a.slices, k = blockIdx.x / a.slices, j = blockIdx.x - k * a.slices;
  if ((int)blockIdx.x > grads) return clear_outside(a.offsets, a.tokens, a.seqs, a.dlogp, blockIdx.x - grads - 1, gridDim.x - grads - 1);
  const bool total = (int)blockIdx.x == grads, rows = a.slices >= kRowSlices;
  auto lanes_count = [&](int i, auto of) {
    constexpr int lanes = decltype(of)::value;
    uint32_t c = 0;
#pragma unroll 4
    for (int q = threadIdx.x & (lanes - 1); q < a.slices; q += lanes) c += a.counts[i * a.slices + q];
#pragma unroll
    for (int o = lanes / 2; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
    return (double)c;
  };
  using Wave = std::integral_constant<int, 64>;
  using Row = std::integral_constant<int, 16>;      // lanes to a sequence of many slices, where there are more than four
  auto thread_count = [&](int i) {
    uint32_t c = 0;
#pragma unroll 4
    for (int q = 0; q < a.slices; ++q) c += a.counts[i * a.slices + q];
    return (double)c;
  };
  // all counted tokens, or the sequences that have any
  auto all = [&]() {
    double n = 0.0;
    if (a.groups > 0) {
      if ((int)threadIdx.x < a.groups) n = a.gathered[threadIdx.x];
    } else if (!a.by_sequence) {
      for (int i = threadIdx.x; i < grads; i += kThreads) n += a.counts[i];
    } else if (rows) {
      auto live = [&](auto of) {
        constexpr int L = decltype(of)::value;
        for (int i = threadIdx.x / L; i < a.seqs; i += kThreads / L) n += lanes_count(i, of) > 0.0 && threadIdx.x % L == 0 ? 1.0 : 0.0;
      };
      if (a.seqs <= 4) live(Wave{});
      else live(Row{});
    } else {
      for (int i = threadIdx.x; i < a.seqs; i += kThreads) n += thread_count(i) > 0.0 ? 1.0 : 0.0;
    }
    return block_sum(n);
  };
  if (!total) {
    const TokenRange r = token_slice(sequence(a.offsets, a.tokens, k), j, a.slices);
    return scale_gradients(a, r, threadIdx.x, kThreads, k, [&]() { return token_weight(a, all(), a.by_sequence ? lanes_count(k, Wave{}) : 0.0); });
  }
  const double n = all();
  double t[3] = {0.0, 0.0, 0.0};
  auto add = [&](int q, double w) {
    for (int m = 0; m < 3; ++m) t[m] += a.sums[(int64_t)m * grads + q] * w;
  };
  if (a.groups > 0) {
    const double w = token_weight(a, n, 1.0);
    if ((int)threadIdx.x < a.groups)
      for (int m = 0; m < 3; ++m) t[m] = a.gathered[(m + 1) * a.groups + threadIdx.x] * w;
  } else if (!a.by_sequence) {
    const double w = token_weight(a, n, 0.0);
#pragma unroll 2
    for (int q = threadIdx.x; q < grads; q += kThreads) add(q, w);
  } else if (rows) {
    auto weighted = [&](auto of) {
      constexpr int L = decltype(of)::value;
      for (int i = threadIdx.x / L; i < a.seqs; i += kThreads / L) {
        const double w = token_weight(a, n, lanes_count(i, of));
#pragma unroll 2
        for (int q = threadIdx.x % L; q < a.slices; q += L) add(i * a.slices + q, w);
      }
    };
    if (a.seqs <= 4) weighted(Wave{});
    else weighted(Row{});
  } else {
    for (int i = threadIdx.x; i < a.seqs; i += kThreads) {
      const double w = token_weight(a, n, thread_count(i));
#pragma unroll 2
      for (int q = 0; q < a.slices; ++q) add(i * a.slices + q, w);
    }
  }
  block_sums(t);
  if (threadIdx.x == 0) policy_results(a, t[0], t[1], t[2]);
}

// A small batch in one workgroup and one launch: a wave to a sequence.
__global__ __launch_bounds__(1024) void policy_small_kernel(const PolicyArgs a) {
  __shared__ PolicySums sums[kSmallSeqs];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  double n = 0.0;
  for (int k = wave; k < a.seqs; k += 16) {
    const PolicySums s = policy_tokens(a, sequence(a.offsets, a.tokens, k), lane, 64, k);
    const PolicySums t = {wave_sum(s.loss), wave_sum(s.kl), wave_sum(s.clipped), (uint32_t)wave_sum((double)s.count)};
    if (lane == 0) {
      sums[k] = t;
      n += share(a, t.count);
    }
  }
  n = block_sum(n);      // and its barriers: the sums are written
  double t[3] = {0.0, 0.0, 0.0};
  for (int k = wave; k < a.seqs; k += 16) {
    const double w = token_weight(a, n, sums[k].count);
    scale_gradients(a, sequence(a.offsets, a.tokens, k), lane, 64, k, [&]() { return w; });
    if (lane == 0) { t[0] += sums[k].loss * w; t[1] += sums[k].kl * w; t[2] += sums[k].clipped * w; }
  }
  clear_outside(a.offsets, a.tokens, a.seqs, a.dlogp, 0, 1);
  block_sums(t);
  if (threadIdx.x == 0) policy_results(a, t[0], t[1], t[2]);
}

// Whether a batch goes to one workgroup.
bool small(int64_t tokens, int64_t sequences) { return tokens <= kSmallTokens && sequences <= kSmallSeqs; }

int slices_of(int64_t tokens, int64_t sequences) {
  const int64_t mean = sequences > 0 ? tokens / sequences : 0;
  const int64_t least = tokens / (4 * kCUs), size = least > kSliceTokens ? least : kSliceTokens, n = (mean + size - 1) / size;
  return (int)(n < 1 ? 1 : n > kMaxSlices ? kMaxSlices : n);
}

// Workgroups that clear the tokens of no sequence: how many those are only the device knows.
int clears(int64_t tokens) { return (int)(tokens / kClearTokens) + 1; }

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
// What a call writes, the workspace among it, lies apart from everything else that it gets.
struct Span { const void* p; size_t bytes; const char* name; bool written; };
template <size_t N>
mecefo_status_t check_apart(const Span (&v)[N]) {
  for (size_t i = 0; i < N; ++i)
    for (size_t j = 0; j < N; ++j) {
      if (!v[i].written || i == j || !v[i].p || !v[j].p || !v[i].bytes || !v[j].bytes) continue;
      const uintptr_t x = (uintptr_t)v[i].p, y = (uintptr_t)v[j].p;
      if (x < y + v[j].bytes && y < x + v[i].bytes) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "%s overlaps %s", v[i].name, v[j].name);
    }
  return MECEFO_OK;
}
void* aligned(void* ws) { return (void*)(((uintptr_t)ws + 255) / 256 * 256); }

size_t preference_bytes(const mecefo_preference_desc_t* d) {
  return (size_t)2 * d->pairs * slices_of(d->tokens, (int64_t)d->pairs * 2) * sizeof(Part) + 256;
}
// Workgroups of the launch that gathers, 0 where there is none.  Sequences are one slice each there: with 4 * kCUs of them or more the
// mean is no longer than a slice.
int groups_of(int64_t sequences) {
  static_assert(kGatherFrom >= 4 * kCUs && kGathered <= kThreads, "");
  const int64_t n = (sequences + kThreads - 1) / kThreads;
  return sequences <= kGatherFrom ? 0 : (int)(n < kGathered ? n : kGathered);
}
size_t policy_bytes(const mecefo_policy_desc_t* d) {
  return (size_t)d->sequences * slices_of(d->tokens, d->sequences) * (3 * sizeof(double) + sizeof(uint32_t)) +
         4 * groups_of(d->sequences) * sizeof(double) + 256;
}

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
  const size_t tokens = (size_t)desc->tokens, pairs = (size_t)desc->pairs;
  const Span spans[] = {{loss, 4, "loss", true}, {margins, 4 * pairs, "margins", true}, {rewards, 8 * pairs, "rewards", true},
                        {dlogp, 4 * tokens, "dlogp", true}, {ws, preference_bytes(desc), "the workspace", true},
                        {logp, 4 * tokens, "logp", false}, {ref_logp, 4 * tokens, "ref_logp", false}, {mask, tokens, "mask", false},
                        {offsets, pairs > 0 ? 8 * (2 * pairs + 1) : 0, "offsets", false}};
  TRY(check_apart(spans));
  hipStream_t s = (hipStream_t)hip_stream;
  const int slices = slices_of(desc->tokens, (int64_t)desc->pairs * 2), grads = 2 * desc->pairs * slices;
  const PrefArgs a = {logp, ref_logp, mask, offsets, loss, margins, rewards, dlogp, (Part*)aligned(ws), desc->tokens, desc->pairs,
                      slices, desc->length_mean, desc->beta, desc->label_smoothing, desc->margin, desc->grad_scale};
  if (small(desc->tokens, (int64_t)desc->pairs * 2)) {
    hipLaunchKernelGGL(preference_small_kernel, dim3(1), dim3(1024), 0, s, a);
    LAUNCHED("preference_loss");
    return MECEFO_OK;
  }
  if (grads > 0) {
    hipLaunchKernelGGL(preference_sums_kernel, dim3(grads), dim3(kThreads), 0, s, a);
    LAUNCHED("preference_loss");
  }
  hipLaunchKernelGGL(preference_grad_kernel, dim3(grads + 1 + clears(desc->tokens)), dim3(kThreads), 0, s, a);
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
  if (any && !ref_logp && desc->kl_coef != 0.f) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "kl_coef needs ref_logp");
  TRY(check_ws(policy_bytes(desc), ws, ws_bytes));
  const size_t tokens = (size_t)desc->tokens, seqs = (size_t)desc->sequences;
  const Span spans[] = {{loss, 4, "loss", true}, {kl, 4, "kl", true}, {clipped, 4, "clipped", true}, {dlogp, 4 * tokens, "dlogp", true},
                        {ws, policy_bytes(desc), "the workspace", true}, {logp, 4 * tokens, "logp", false},
                        {old_logp, 4 * tokens, "old_logp", false}, {ref_logp, 4 * tokens, "ref_logp", false},
                        {advantage, 4 * (desc->advantage_per_token ? tokens : seqs), "advantage", false}, {mask, tokens, "mask", false},
                        {offsets, seqs > 0 ? 8 * (seqs + 1) : 0, "offsets", false}};
  TRY(check_apart(spans));
  hipStream_t s = (hipStream_t)hip_stream;
  const int slices = slices_of(desc->tokens, desc->sequences), grads = desc->sequences * slices;
  const int groups = groups_of(desc->sequences);
  double* const sums = (double*)aligned(ws) + 4 * groups;      // what is gathered lies in front of it
  const PolicyArgs a = {logp, old_logp, ref_logp, advantage, mask, offsets, loss, kl, clipped, dlogp, sums,
                        (uint32_t*)(sums + (int64_t)3 * grads), (double*)aligned(ws), groups, desc->tokens, desc->sequences, slices, desc->mean == MECEFO_MEAN_SEQUENCES, desc->advantage_per_token,
                        1.0 - (double)desc->clip_low, 1.0 + (double)desc->clip_high, log1p(-(double)desc->clip_low),
                        log1p((double)desc->clip_high), desc->kl_coef, desc->grad_scale};
  if (small(desc->tokens, desc->sequences)) {
    hipLaunchKernelGGL(policy_small_kernel, dim3(1), dim3(1024), 0, s, a);
    LAUNCHED("policy_loss");
    return MECEFO_OK;
  }
  if (grads > 0) {
    hipLaunchKernelGGL(policy_tokens_kernel, dim3(grads), dim3(kThreads), 0, s, a);
    LAUNCHED("policy_loss");
  }
  if (groups > 0) {
    hipLaunchKernelGGL(policy_gather_kernel, dim3(groups), dim3(kThreads), 0, s, a);
    LAUNCHED("policy_loss");
  }
  hipLaunchKernelGGL(policy_scale_kernel, dim3(grads + 1 + clears(desc->tokens)), dim3(kThreads), 0, s, a);
  LAUNCHED("policy_loss");
  return MECEFO_OK;
}

}  // extern "C"
