// Log-probabilities of given tokens under the LM head, and their gradient: what lies between the last block's output and the
// gradient that the stack takes back.
//   U = norm(X) gamma (or X),  z = logit_scale U W^T [b x V],  lse_i = log sum_v exp z_iv,  logp_i = z_i,label - lse_i
//   dz_iv = logit_scale dlogp_i (1[v = label_i] - exp(z_iv - lse_i)),  dU = dz W,  dW = dz^T U
// Everything that is large is a product on the GEMM core: 2 b d V operations forward, 6 b d V backward (z is formed again).
// bf16 roundings: dz, because dU and dW are bf16 products of it (two bf16 halves of dz would double them), 2.2e-3 on either against
// 1.7e-3 for the result's own rounding; with a gain U, an operand as well, and dU, which the norm's backward reads as the blocks' norms
// read theirs (in fp32 its bytes would double).  Of few tokens dU is added up from fp32 parts and rounded once.
#include <math.h>
#include <string.h>

#include "../../include/mecefo.h"
#include "gemm_bf16_launch.hip.h"
#include "gemm_common.hip.h"
#include "mecefo_internal.h"

namespace mecefo {
namespace {

__device__ inline bool counted(int64_t label, int vocab) { return label >= 0 && label < vocab; }

// A logit is rounded once: fused into z - m it would not be the one that m was taken from.
__device__ inline float logit(float z, float scale) {
#pragma clang fp contract(off)
  return z * scale;
}

// lse and logp of the rows of fp32 products z (before logit_scale), a workgroup per row, in one pass with a running maximum.
constexpr int kRowGroups = 1 << 21;      // at most: a launch of 2^32 threads leaves some of them out, without an error
__global__ __launch_bounds__(1024) void head_rows_kernel(const float* __restrict__ Z, int64_t ldz, int rows, int vocab, float scale,
                                                        const int64_t* __restrict__ labels, float* __restrict__ logp,
                                                        float* __restrict__ lse) {
  __shared__ float2 red[16];
  auto join = [](float2 x, float2 y) {      // a share without columns is (-inf, 0)
    const float m = fmaxf(x.x, y.x), k = m == -INFINITY ? 0.f : m;
    return float2{m, x.y * expf(x.x - k) + y.y * expf(y.x - k)};
  };
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const float* z = Z + row * ldz;
    float2 a = {-INFINITY, 0.f};
    for (int v0 = 4 * threadIdx.x; v0 < vocab; v0 += 4096) {      // rows are whole vectors of eight
      typedef __attribute__((ext_vector_type(4))) float f4;
      const f4 x = *(const f4*)(z + v0);
      float y[4], m = a.x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = v0 + e < vocab ? logit(x[e], scale) : -INFINITY;
        m = fmaxf(m, y[e]);
      }
      float s = a.x == -INFINITY ? 0.f : a.y * expf(a.x - m);
#pragma unroll
      for (int e = 0; e < 4; ++e) s += expf(y[e] - m);
      a = float2{m, s};
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) a = join(a, float2{__shfl_xor(a.x, o, 64), __shfl_xor(a.y, o, 64)});
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < 16; ++w) a = join(a, red[w]);
      const float l = a.x + logf(a.y);
      const int64_t label = labels[row];
      logp[row] = counted(label, vocab) ? logit(z[label], scale) - l : 0.f;
      if (lse) lse[row] = l;
    }
    if (row + gridDim.x < rows) __syncthreads();      // `red` is read
  }
}

// lse and logp from the parts that the products' epilogue leaves: (largest z', sum of 2^(z' - that)) of a row over part_cols
// columns, [parts][rows], z' = z log2(e), and z at the label.  ROWS neighbouring rows to a workgroup, 1024 / ROWS threads share out a row's
// parts: 16 rows read whole lines, where there are few rows 2 use more of the chip.  Forwards of d 128, vocabulary 32000, with 16 / with 2,
// us: 1 row 10.0 / 8.3, 77 rows 12.1 / 11.5, 256 13.9 / 14.3, 1024 26.6 / 28.8, 8192 155 / 172.
template <int ROWS>
__global__ __launch_bounds__(1024) void head_parts_kernel(const float2* __restrict__ part, int parts, int rows, int vocab,
                                                          const float* __restrict__ zl, const int64_t* __restrict__ labels,
                                                          float* __restrict__ logp, float* __restrict__ lse) {
  constexpr int G = 1024 / ROWS;
  __shared__ float2 red[16][ROWS];
  const int r = threadIdx.x % ROWS, g = threadIdx.x / ROWS, row = blockIdx.x * ROWS + r;
  auto join = [](float2 x, float2 y) {      // a share without parts is (-inf, 0)
    const float m = fmaxf(x.x, y.x), k = m == -INFINITY ? 0.f : m;
    return float2{m, x.y * __builtin_amdgcn_exp2f(x.x - k) + y.y * __builtin_amdgcn_exp2f(y.x - k)};
  };
  float2 a = {-INFINITY, 0.f};
  const int at = row < rows ? row : rows - 1;
#pragma unroll 4
  for (int k = g; k < parts; k += G) a = join(a, part[(int64_t)k * rows + at]);
#pragma unroll
  for (int o = ROWS; o < 64; o *= 2) a = join(a, float2{__shfl_xor(a.x, o, 64), __shfl_xor(a.y, o, 64)});
  if ((threadIdx.x & 63) < ROWS) red[threadIdx.x >> 6][r] = a;
  __syncthreads();
  if (threadIdx.x >= ROWS || row >= rows) return;
#pragma unroll
  for (int w = 1; w < 16; ++w) a = join(a, red[w][r]);
  const float l = a.x * kLn2 + logf(held_sum(a.y));
  logp[row] = counted(labels[row], vocab) ? zl[row] - l : 0.f;
  if (lse) lse[row] = l;
}

// out[row, 0 .. cols) = sum of the parts [k][row, col], in their order, V columns per thread.  list: the rows are *count in
// number, and row r goes to row list[r].  accumulate: added to what is there.
template <typename T, int V>
__global__ __launch_bounds__(256) void head_sum_kernel(const float* __restrict__ part, int parts, int64_t rows, int cols,
                                                       T* __restrict__ out, int64_t ldo, const int* __restrict__ list,
                                                       const int* __restrict__ count, int accumulate) {
  if (list) rows = *count;
  struct alignas(4 * V) In { float e[V]; };
  struct alignas(sizeof(T) * V) Out { T e[V]; };
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
  if (i >= rows * cols) return;
  const int64_t row = i / cols;
  In s = *(const In*)(part + i);
#pragma unroll 4
  for (int k = 1; k < parts; ++k) {
    const In x = *(const In*)(part + (int64_t)k * rows * cols + i);
#pragma unroll
    for (int e = 0; e < V; ++e) s.e[e] += x.e[e];
  }
  Out* to = (Out*)(out + (list ? (int64_t)list[row] : row) * ldo + (i - row * cols));
  Out o;
  if (accumulate) {
    o = *to;
#pragma unroll
    for (int e = 0; e < V; ++e) s.e[e] += (float)o.e[e];
  }
#pragma unroll
  for (int e = 0; e < V; ++e) o.e[e] = (T)s.e[e];
  *to = o;
}

// The rows that take part in the gradient, a label in the vocabulary and a dlogp that is not zero, in their order at the front
// of `list`, the others behind them; *count of the former.  One workgroup, eight rows per thread at a time.
__global__ __launch_bounds__(1024) void head_list_kernel(const int64_t* __restrict__ labels, const float* __restrict__ dlogp, int rows,
                                                         int vocab, int* __restrict__ list, int* __restrict__ count) {
  __shared__ int waves[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int done = 0;      // listed rows of the rounds before
  for (int base = 0; base < rows; base += 8192) {
    const int r0 = base + 8 * threadIdx.x;
    uint32_t on = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (r0 + k < rows) on |= (counted(labels[r0 + k], vocab) && dlogp[r0 + k] != 0.f ? 1u : 0u) << k;
    const int mine = __popc(on);
    int before = mine;      // inclusive, over the wave
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int x = __shfl_up(before, o, 64);
      before += lane >= o ? x : 0;
    }
    __syncthreads();        // the round before has read `waves`
    if (lane == 63) waves[wave] = before;
    __syncthreads();
    int at = done + before - mine, all = 0;
    for (int w = 0; w < 16; ++w) {
      at += w < wave ? waves[w] : 0;
      all += waves[w];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int row = r0 + k;
      if (row >= rows) break;
      if (on >> k & 1) list[at++] = row;
      else list[rows - 1 - (row - at)] = row;      // row - at rows in front of this one are not listed
    }
    done += all;
  }
  if (threadIdx.x == 0) *count = done;
}

// What the listed rows' gradients are made of, gathered, and zeros for the gradients of the others.  A wave per row.
struct HeadGather {
  const __bf16* U; int64_t ldu;
  const int64_t* labels; const float *lse, *dlogp;
  const int *list, *count;
  __bf16* Uc; int64_t* labels_c; float *lse_c, *dlogp_c;
  __bf16* dU; int64_t lddu;
  int rows, d;
};
__global__ __launch_bounds__(256) void head_gather_kernel(const HeadGather a) {
  struct alignas(16) V8 { __bf16 e[8]; };
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.rows) return;
  const int src = a.list[r];
  if (r >= *a.count) {
    for (int i = lane; i < a.d / 8; i += 64) *(V8*)(a.dU + (int64_t)src * a.lddu + 8 * i) = V8{};
    return;
  }
#pragma unroll 4
  for (int i = lane; i < a.d / 8; i += 64) *(V8*)(a.Uc + (int64_t)r * a.d + 8 * i) = *(const V8*)(a.U + (int64_t)src * a.ldu + 8 * i);
  if (lane == 0) {
    a.labels_c[r] = a.labels[src];
    a.lse_c[r] = a.lse[src];
    a.dlogp_c[r] = a.dlogp[src];
  }
}

__global__ __launch_bounds__(256) void head_zero_kernel(uint32_t* p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0;
}

inline int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

struct Head {
  const mecefo_head_desc_t* d;
  bool bf16;
  int esz, b, dm, vocab;
  int64_t ldz;
};

#define FAIL(st, ...) ((mecefo_status_t)fail((int)(st), __VA_ARGS__))
#define TRY(x) do { mecefo_status_t st__ = (x); if (st__ != MECEFO_OK) return st__; } while (0)
#define HIP_TRY(x) do { hipError_t e__ = (x); if (e__ != hipSuccess) return FAIL(MECEFO_ERR_LAUNCH, "%s: %s", #x, hipGetErrorString(e__)); } while (0)

// The products read their operands with 32-bit offsets: X, W and the backward's dz stay below 2 GiB; outputs are addressed with 64
// bits.  The bf16 forward stores no logits: its parts at their smallest tiles, 8 bytes to 32 columns, are what is bounded then.
mecefo_status_t check_desc(const mecefo_head_desc_t* d, bool backward, Head* h) {
  if (!d) return FAIL(MECEFO_ERR_INVALID_ARG, "descriptor is NULL");
  if (d->dtype != MECEFO_F32 && d->dtype != MECEFO_BF16) return FAIL(MECEFO_ERR_INVALID_ARG, "dtype must be MECEFO_F32 or MECEFO_BF16");
  if (d->grad_dtype != MECEFO_F32 && d->grad_dtype != d->dtype) return FAIL(MECEFO_ERR_UNSUPPORTED, "grad_dtype must be MECEFO_F32 or equal to dtype");
  if (d->tokens < 0 || d->d_model < 1 || d->vocab < 1) return FAIL(MECEFO_ERR_INVALID_ARG, "tokens >= 0, d_model >= 1, vocab >= 1 required");
  if (d->ld_act_d < d->d_model || d->ld_w < d->d_model) return FAIL(MECEFO_ERR_INVALID_ARG, "a row stride is smaller than the logical width");
  // times log2(e) it is still a number
  if (!(fabsf(d->logit_scale) <= 0x1p127f)) return FAIL(MECEFO_ERR_INVALID_ARG, "logit_scale must be a number of at most 2^127");
  h->d = d;
  h->bf16 = d->dtype == MECEFO_BF16;
  h->esz = h->bf16 ? 2 : 4;
  if (h->bf16 && d->d_model % 8) return FAIL(MECEFO_ERR_UNSUPPORTED, "bf16 path needs d_model to be a multiple of 8 (got %d)", d->d_model);
  if (h->bf16 && (d->ld_act_d % 8 || d->ld_w % 8)) return FAIL(MECEFO_ERR_INVALID_ARG, "bf16 path needs every row stride to be a multiple of 8 elements");
  const bool parts = h->bf16 && !backward;
  if (reaches_2gib(d->tokens, d->ld_act_d, h->esz) || reaches_2gib(d->vocab, d->ld_w, h->esz) ||
      reaches_2gib(d->tokens, parts ? ((int64_t)d->vocab + 31) / 32 : up(d->vocab, 8), parts ? 8 : h->esz))
    return FAIL(MECEFO_ERR_UNSUPPORTED, "a tensor reaches 2 GiB; split the token batch");
  if (d->tokens > kMaxWaveRows) return FAIL(MECEFO_ERR_UNSUPPORTED, "more than 2^26 - 64 tokens; split the token batch");
  h->b = (int)d->tokens;
  h->dm = d->d_model;
  h->vocab = d->vocab;
  h->ldz = up(d->vocab, 8);
  return MECEFO_OK;
}

mecefo_status_t check_ptr(const Head& h, const void* p, const char* name, bool required) {
  if (!p) return required ? FAIL(MECEFO_ERR_INVALID_ARG, "%s is NULL", name) : MECEFO_OK;
  if ((uintptr_t)p % (h.bf16 ? 16 : 4)) return FAIL(MECEFO_ERR_INVALID_ARG, "%s is not %d-byte aligned", name, h.bf16 ? 16 : 4);
  return MECEFO_OK;
}
mecefo_status_t check_small(const void* p, const char* name, int align, bool required) {
  if (!p) return required ? FAIL(MECEFO_ERR_INVALID_ARG, "%s is NULL", name) : MECEFO_OK;
  if ((uintptr_t)p % align) return FAIL(MECEFO_ERR_INVALID_ARG, "%s is not %d-byte aligned", name, align);
  return MECEFO_OK;
}
mecefo_status_t check_apart(const void* a, size_t na, const char* an, const void* b, size_t nb, const char* bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  if (a && b && na && nb && x < y + nb && y < x + na) return FAIL(MECEFO_ERR_INVALID_ARG, "%s overlaps %s", an, bn);
  return MECEFO_OK;
}

// Parts of dU at most: the contraction over the vocabulary is long and its output small where there are few tokens.
constexpr int kMaxParts = 16;
constexpr int64_t kPartRoom = 32 << 20;      // fp32 elements

// Whether the backward goes by a list of the rows that take part: a list, a copy of their U and products over them only.  Which
// rows these are is known on the device alone; two launches and the copy cost 10 to 20 us, which is 0.4 % of the largest calls.  All rows /
// the list, us, with none, a tenth and three tenths of the tokens out: [8192 x 4096], vocabulary 32000, 5240 / 5259, 5211 / 4966,
// 5151 / 4237; [2048 x 2048] 735 / 735, 730 / 701, 720 / 579; [1024 x 1024] (2e11 operations) 232 / 231, 219 / 222, 219 / 194; [512 x 2048]
// 227 / 236, 225 / 228, 223 / 213; [1024 x 512] (1e11) 140 / 150, 140 / 146, 140 / 133.  And only where
// dW has about a 256 x 256 tile for every CU: with fewer it is cut along the tokens, which a number of rows that the host does not know rules out.
// A tenth out, us: 16384 x 1024, V 4096 401 / 449; 65536 x 512, V 8192 1733 / 1991; 8192 x 1024, V 8192 392 / 411; 16384 x 2048, V 8192
// 1336 / 1289; 65536 x 1024, V 16000 5781 / 5701; 32768 x 512, V 32000 3582 / 3291.  In fp32 all rows.
bool by_list(const Head& h) {
  if (!h.bf16) return false;
  const int forced = options().head_rows.load(std::memory_order_relaxed);
  return forced ? forced == 2 : (int64_t)h.vocab * h.dm >= 16000000 && 6.0 * h.b * h.dm * h.vocab >= 2e11;
}

struct HeadWs {
  size_t U, rstd, Z, zl, dZ, dU, part, dgp, zero, list, count, Uc, labels, lse, dlogp, total;
  int64_t room;
  bool listed;      // read from the switch once per call
};
HeadWs layout(const Head& h, bool backward) {
  HeadWs w;
  size_t off = 0;
  auto take = [&](int64_t bytes) { size_t o = off; off += (size_t)up(bytes, 256); return o; };
  const int64_t act = (int64_t)h.b * h.dm;
  w.U = take(act * h.esz);
  w.rstd = take((int64_t)h.b * 4);
  w.Z = w.zl = w.dZ = w.dU = w.part = w.dgp = w.zero = w.list = w.count = w.Uc = w.labels = w.lse = w.dlogp = off;
  w.room = 0;
  w.listed = backward && by_list(h);
  if (!backward) {      // bf16: the parts of the log-sum-exps, over 32 columns where the tiles are the smallest; fp32: the products
    w.Z = take(h.bf16 ? ((int64_t)h.vocab + 31) / 32 * h.b * 8 : (int64_t)h.b * h.ldz * 4);
    w.zl = take((int64_t)h.b * 4);
  }
  if (backward) {
    w.dZ = take((int64_t)h.b * h.ldz * h.esz);
    w.dU = take(act * h.esz);
    w.room = act * kMaxParts < kPartRoom ? act * kMaxParts : kPartRoom;
    w.part = take(w.room * 4);
    w.dgp = take((int64_t)rmsnorm_bwd_blocks(h.b) * h.dm * 4);
    w.zero = take((int64_t)h.dm * h.esz);
    if (w.listed) {
      w.list = take((int64_t)h.b * 4);
      w.count = take(4);
      w.Uc = take(act * h.esz);
      w.labels = take((int64_t)h.b * 8);
      w.lse = take((int64_t)h.b * 4);
      w.dlogp = take((int64_t)h.b * 4);
    }
  }
  w.total = off + 256;
  return w;
}
mecefo_status_t carve(const Head& h, bool backward, void* ws, size_t ws_bytes, HeadWs* w, char** base) {
  *w = layout(h, backward);
  if (w->total > ws_bytes) return FAIL(MECEFO_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu needed", ws_bytes, w->total);
  if (!ws) return FAIL(MECEFO_ERR_INVALID_ARG, "workspace is NULL");
  *base = (char*)(((uintptr_t)ws + 255) / 256 * 256);
  return MECEFO_OK;
}

GemmLaunch product(const Head& h, bool akc, bool bkc, int epi, const void* A, int64_t lda, const void* B, int64_t ldb, void* C,
                   int64_t ldc, int M, int N, int K) {
  GemmLaunch g;
  memset(&g, 0, sizeof(g));
  g.a_kcontig = akc;
  g.b_kcontig = bkc;
  g.epi = epi;
  g.bf16 = h.bf16;
  g.nprob = 1;
  GemmProblem& p = g.p[0];
  p.A[0] = p.A[1] = A;
  p.B[0] = p.B[1] = B;
  p.C[0] = C;
  p.lda = lda; p.ldb = ldb; p.ldc = ldc;
  p.M = M; p.N = N; p.K = K; p.nseg = 1;
  return g;
}

// U, which is X where there is no gain.
mecefo_status_t head_norm(const Head& h, const HeadWs& w, char* base, const void* X, const void* gamma, const void** U, int64_t* ldu,
                          hipStream_t s) {
  *U = X;
  *ldu = h.d->ld_act_d;
  if (!gamma) return MECEFO_OK;
  HIP_TRY(launch_rmsnorm_fwd(h.bf16, X, h.d->ld_act_d, gamma, h.d->rms_eps, base + w.U, h.dm, (float*)(base + w.rstd), h.b, h.dm, s));
  *U = base + w.U;
  *ldu = h.dm;
  return MECEFO_OK;
}

hipError_t sum_parts(bool bf16, const void* part, int parts, int64_t rows, int cols, void* out, int64_t ldo, const int* list, const int* count,
                     int accumulate, hipStream_t s) {
  auto go = [&](auto type, auto v) {
    using T = decltype(type);
    constexpr int V = decltype(v)::value;
    hipLaunchKernelGGL((head_sum_kernel<T, V>), dim3((unsigned)((rows * cols / V + 255) / 256)), dim3(256), 0, s, (const float*)part, parts, rows, cols, (T*)out, ldo, list, count, accumulate);
  };
  if (bf16) go(__bf16{}, std::integral_constant<int, 4>{});      // rows are whole vectors of eight
  else if (cols % 4 == 0 && ldo % 4 == 0 && (uintptr_t)out % 16 == 0) go(float{}, std::integral_constant<int, 4>{});
  else go(float{}, std::integral_constant<int, 1>{});
  return hipGetLastError();
}

}  // namespace
}  // namespace mecefo

using namespace mecefo;

extern "C" {

mecefo_status_t mecefo_head_workspace_bytes(const mecefo_head_desc_t* desc, int backward, size_t* out_bytes) {
  Head h;
  TRY(check_desc(desc, backward != 0, &h));
  if (!out_bytes) return FAIL(MECEFO_ERR_INVALID_ARG, "out_bytes is NULL");
  *out_bytes = layout(h, backward != 0).total;
  return MECEFO_OK;
}

mecefo_status_t mecefo_head_logprob_fwd(const mecefo_head_desc_t* desc, const void* X, const void* gamma, const void* W,
                                        const int64_t* labels, float* logp, float* lse, void* ws, size_t ws_bytes,
                                        void* hip_stream) {
  Head h;
  TRY(check_desc(desc, false, &h));
  const bool any = h.b > 0;
  TRY(check_ptr(h, X, "X", any)); TRY(check_ptr(h, gamma, "gamma", false)); TRY(check_ptr(h, W, "W", true));
  TRY(check_small(labels, "labels", 8, any)); TRY(check_small(logp, "logp", 4, any)); TRY(check_small(lse, "lse", 4, false));
  HeadWs w;
  char* base;
  TRY(carve(h, false, ws, ws_bytes, &w, &base));
  if (!any) return MECEFO_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  const void* U;
  int64_t ldu;
  TRY(head_norm(h, w, base, X, gamma, &U, &ldu, s));
  GemmLaunch g = product(h, true, true, h.bf16 ? EPI_HEAD_LSE : EPI_STORE, U, ldu, W, desc->ld_w, base + w.Z,
                         h.bf16 ? h.b : h.ldz, h.b, h.vocab, h.dm);
  if (h.bf16) {
    g.p[0].C[1] = const_cast<int64_t*>(labels);
    g.p[0].C[2] = base + w.zl;
    g.p[0].scale = desc->logit_scale;
  }
  HIP_TRY(launch_gemm(g, s));
  if (h.bf16) {
    const float2* part = (const float2*)(base + w.Z);
    const float* zl = (const float*)(base + w.zl);
    const int parts = cdiv(h.vocab, g.part_cols);
    if (h.b >= 256) hipLaunchKernelGGL(head_parts_kernel<16>, dim3(cdiv(h.b, 16)), dim3(1024), 0, s, part, parts, h.b, h.vocab, zl, labels, logp, lse);
    else hipLaunchKernelGGL(head_parts_kernel<2>, dim3(cdiv(h.b, 2)), dim3(1024), 0, s, part, parts, h.b, h.vocab, zl, labels, logp, lse);
  } else
    hipLaunchKernelGGL(head_rows_kernel, dim3(h.b < kRowGroups ? h.b : kRowGroups), dim3(1024), 0, s, (const float*)(base + w.Z), h.ldz, h.b, h.vocab,
                       desc->logit_scale, labels, logp, lse);
  HIP_TRY(hipGetLastError());
  return MECEFO_OK;
}

mecefo_status_t mecefo_head_logprob_bwd(const mecefo_head_desc_t* desc, const void* X, const void* gamma, const void* W,
                                        const int64_t* labels, const float* lse, const float* dlogp, void* dX, void* dgamma,
                                        void* dW, int accumulate, void* ws, size_t ws_bytes, void* hip_stream) {
  Head h;
  TRY(check_desc(desc, true, &h));
  const bool any = h.b > 0, grad_f32 = desc->grad_dtype == MECEFO_F32;
  TRY(check_ptr(h, X, "X", any)); TRY(check_ptr(h, gamma, "gamma", false)); TRY(check_ptr(h, W, "W", true));
  TRY(check_small(labels, "labels", 8, any)); TRY(check_small(lse, "lse", 4, any)); TRY(check_small(dlogp, "dlogp", 4, any));
  TRY(check_ptr(h, dX, "dX", any)); TRY(check_ptr(h, dgamma, "dgamma", false)); TRY(check_ptr(h, dW, "dW", true));
  if (dgamma && !gamma) return FAIL(MECEFO_ERR_INVALID_ARG, "dgamma requested but gamma is NULL");
  const size_t act = any ? (size_t)((h.b - 1) * desc->ld_act_d + h.dm) * h.esz : 0, wt = (size_t)((h.vocab - 1) * desc->ld_w + h.dm);
  TRY(check_apart(dX, act, "dX", X, act, "X")); TRY(check_apart(dX, act, "dX", W, wt * h.esz, "W"));
  TRY(check_apart(dW, wt * (grad_f32 ? 4 : h.esz), "dW", W, wt * h.esz, "W")); TRY(check_apart(dW, wt * (grad_f32 ? 4 : h.esz), "dW", X, act, "X"));
  TRY(check_apart(dW, wt * (grad_f32 ? 4 : h.esz), "dW", dX, act, "dX"));
  HeadWs w;
  char* base;
  TRY(carve(h, true, ws, ws_bytes, &w, &base));
  hipStream_t s = (hipStream_t)hip_stream;
  const void* U = X;
  int64_t ldu = desc->ld_act_d;
  void* dZ = base + w.dZ;
  void* dU = gamma ? base + w.dU : dX;
  const int64_t lddu = gamma ? h.dm : desc->ld_act_d;
  const int* list = nullptr;
  int* count = nullptr;
  if (any) {
    TRY(head_norm(h, w, base, X, gamma, &U, &ldu, s));
    if (w.listed) {
      count = (int*)(base + w.count);
      hipLaunchKernelGGL(head_list_kernel, dim3(1), dim3(1024), 0, s, labels, dlogp, h.b, h.vocab, (int*)(base + w.list), count);
      HIP_TRY(hipGetLastError());
      list = (const int*)(base + w.list);
      const HeadGather a = {(const __bf16*)U, ldu, labels, lse, dlogp, list, count, (__bf16*)(base + w.Uc), (int64_t*)(base + w.labels),
                            (float*)(base + w.lse), (float*)(base + w.dlogp), (__bf16*)dU, lddu, h.b, h.dm};
      hipLaunchKernelGGL(head_gather_kernel, dim3(cdiv(h.b, 4)), dim3(256), 0, s, a);
      HIP_TRY(hipGetLastError());
      U = a.Uc; ldu = h.dm; labels = a.labels_c; lse = a.lse_c; dlogp = a.dlogp_c;
    }
    GemmLaunch g = product(h, true, true, EPI_HEAD_GRAD, U, ldu, W, desc->ld_w, dZ, h.ldz, h.b, h.vocab, h.dm);
    GemmProblem& p = g.p[0];
    p.C[1] = const_cast<int64_t*>(labels);
    p.C[2] = count;
    p.pad_cols = (int)h.ldz;
    p.rowvec = lse;
    p.addend = dlogp;
    p.scale = desc->logit_scale;
    HIP_TRY(launch_gemm(g, s));
  }
  {  // dW = dz^T U   [V x d], contraction over tokens, cut where there are many to a small dW (by the list their number is not known here)
    GemmLaunch g = product(h, false, false, EPI_STORE, dZ, h.ldz, U, ldu, base + w.part, h.dm, h.vocab, h.dm, h.b);
    if (any && !list) {
      const int64_t most = w.room / ((int64_t)h.vocab * h.dm);
      if (h.bf16) bf16_plan_splits(g, w.room);
      else f32_plan_splits(g, (int)(most < kMaxParts ? most : kMaxParts));
    }
    const int parts = g.p[0].splits;
    if (parts < 2) {
      g.epi = list ? EPI_HEAD_DW : EPI_GRAD;
      g.p[0].C[0] = dW;
      g.p[0].C[2] = count;
      g.p[0].ldc = desc->ld_w;
      g.out_f32 = grad_f32;
      g.accumulate = accumulate;
    }
    HIP_TRY(launch_gemm(g, s));
    if (parts > 1) HIP_TRY(sum_parts(!grad_f32, base + w.part, parts, h.vocab, h.dm, dW, desc->ld_w, nullptr, nullptr, accumulate, s));
  }
  int nblk = 0;
  float* dgp = (float*)(base + w.dgp);
  if (any) {  // dU = dz W   [b x d], contraction over the vocabulary
    GemmLaunch g = product(h, true, false, list ? EPI_HEAD_DU : EPI_STORE, dZ, h.ldz, W, desc->ld_w, dU, h.dm, h.b, h.dm, h.vocab);
    g.p[0].kpad_ok = 1;      // dz has zeros behind the vocabulary
    g.p[0].C[1] = const_cast<int*>(list);
    g.p[0].C[2] = count;
    if (h.bf16) bf16_plan_splits(g, w.room);
    else f32_plan_splits(g, (int)(w.room / ((int64_t)h.b * h.dm)));
    const int parts = g.p[0].splits;
    if (parts > 1) g.p[0].C[0] = base + w.part;
    else g.p[0].ldc = lddu;
    HIP_TRY(launch_gemm(g, s));
    if (parts > 1) HIP_TRY(sum_parts(h.bf16, base + w.part, parts, h.b, h.dm, dU, lddu, list, count, 0, s));
    if (gamma) {  // dX = normbwd(dU): the norm backward adds a residual gradient, here a row of zeros with stride 0
      const int words = (h.dm * h.esz + 3) / 4;
      hipLaunchKernelGGL(head_zero_kernel, dim3((words + 255) / 256), dim3(256), 0, s, (uint32_t*)(base + w.zero), words);
      HIP_TRY(hipGetLastError());
      const NormBwd n = {dU, h.dm, 0, 0, X, desc->ld_act_d, (const float*)(base + w.rstd), gamma, base + w.zero, 0, dX, desc->ld_act_d,
                         dgamma ? dgp : nullptr, (int64_t)rmsnorm_bwd_blocks(h.b) * h.dm, h.b, h.dm};
      HIP_TRY(launch_rmsnorm_bwd(h.bf16, n, &nblk, s));
    }
  }
  if (dgamma) HIP_TRY(launch_dgamma_reduce(dgp, nblk, h.dm, dgamma, grad_f32, h.bf16, accumulate, s));
  return MECEFO_OK;
}

}  // extern "C"
