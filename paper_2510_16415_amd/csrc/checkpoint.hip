// Activation checkpoints in 8 bits: a row is cut into groups of 32 columns, a group holds 32 signed bytes q and one byte e,
// and stands for the values q 2^(e - 127).  e is the exponent of the group's largest magnitude less 6, so that the largest
// byte lies in 64 .. 127, and q = x 2^(127 - e) rounded to the nearest whole number (halves to even), at most 127.
// A power of two and seven bits: every value is a bf16 number, so unpacking is exact in either storage type, and the
// scaling is exact in both directions, so the bytes do not depend on the order or the kind of the arithmetic.  Gaussian values are off
// by 0.83 % (norm); one fp32 scale per 128 columns, which takes the same bytes, 0.65 %, but there a loud column costs 127 others
// instead of the 31 next to it.  A group with an infinity or a NaN is NaN throughout.
#include "checkpoint.hip.h"
#include "gemm_common.hip.h"
#include "mecefo_internal.h"

namespace mecefo {
namespace {

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Vec { T e[VEC]; };

// Packing: 16 columns per lane, whose bytes are one 16-byte store; unpacking: 16 bytes of the values per lane, so that its
// stores cover whole lines.  [8192 x 4096] bf16, us: packing 17 / 22 (8 columns per lane), unpacking 25 (16 columns) / 20.
// kUnits such pieces per lane, 256 lanes apart, all loaded before the first is used.  ALIGNED: rows start on 16 bytes.
constexpr int kUnits = 2;
template <typename T> constexpr int kCols = 16 / sizeof(T);
constexpr int kPackCols = 16;

template <typename T, int N, bool ALIGNED>
__device__ inline void load_cols(const T* x, int n, float (&v)[N]) {
  constexpr int V = kCols<T>;
  if (ALIGNED && n >= N) {
#pragma unroll
    for (int h = 0; h < N / V; ++h) {
      const Vec<T, V> a = *(const Vec<T, V>*)(x + h * V);
#pragma unroll
      for (int k = 0; k < V; ++k) v[h * V + k] = (float)a.e[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = k < n ? (float)x[k] : 0.f;
  }
}
template <typename T, int N, bool ALIGNED>
__device__ inline void store_cols(T* x, int n, const float (&v)[N]) {
  if (ALIGNED && n >= N) {
    Vec<T, N> a;
#pragma unroll
    for (int k = 0; k < N; ++k) a.e[k] = (T)v[k];
    *(Vec<T, N>*)x = a;
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < n) x[k] = (T)v[k];
  }
}

// Row and first column of piece i; `per` pieces to a row, whole groups.  rows * per is below 2^31 (q is below 2 GiB).
template <int N> struct Piece { uint32_t row; int c; };
template <int N> __device__ inline Piece<N> piece(uint32_t i, uint32_t per) {
  const uint32_t row = i / per;
  return Piece<N>{row, (int)(i - row * per) * N};
}

template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void ckpt_pack_kernel(const T* __restrict__ X, int64_t ldx, uint32_t pieces, int cols, uint32_t per,
                                                        int8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ e, int64_t lde) {
  constexpr int N = kPackCols;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= pieces) return;      // whole groups: pieces is even
  const Piece<N> p = piece<N>(i, per);
  float v[N];
  load_cols<T, N, ALIGNED>(X + p.row * ldx + p.c, cols - p.c, v);
  const int ex = ckpt_exponent(ckpt_most(v));
  Vec<uint32_t, N / 4> b;
  ckpt_bytes(v, ex, b.e);
  *(Vec<uint32_t, N / 4>*)(q + p.row * ldq + p.c) = b;
  if (p.c % kCkptGroup == 0) e[p.row * lde + p.c / kCkptGroup] = (uint8_t)ex;
}

template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void ckpt_unpack_kernel(const int8_t* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ e,
                                                          int64_t lde, uint32_t pieces, int cols, uint32_t per, T* __restrict__ X,
                                                          int64_t ldx) {
  constexpr int N = kCols<T>;
  CkptBytes<N> b[kUnits];
  int ex[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const uint32_t i = (blockIdx.x * kUnits + u) * 256 + threadIdx.x;
    const Piece<N> p = piece<N>(i < pieces ? i : 0, per);
    b[u] = *(const CkptBytes<N>*)(q + p.row * ldq + p.c);
    ex[u] = e[p.row * lde + p.c / kCkptGroup];
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const uint32_t i = (blockIdx.x * kUnits + u) * 256 + threadIdx.x;
    if (i >= pieces) return;
    const Piece<N> p = piece<N>(i, per);
    float v[N];
    ckpt_unpack(b[u], ex[u], v);
    store_cols<T, N, ALIGNED>(X + p.row * ldx + p.c, cols - p.c, v);
  }
}

// U = norm(X) gamma and rstd, and X to a checkpoint on the way: a wave per row, the sums in the order of the norm kernels
// (VEC columns per lane and step), which the packing adds nothing to but its own bytes (a launch of its own reads X again:
// [2048 x 512] 4 us a layer).  Lanes behind the row take part in the groups with zeros.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void rmsnorm_pack_kernel(const T* __restrict__ X, int64_t ldx, const T* __restrict__ gamma, float eps,
                                                           T* __restrict__ U, float* __restrict__ rstd, int64_t rows, int d,
                                                           int8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ e, int64_t lde) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const T* x = X + row * ldx;
  const int nv = d / VEC, ng = (d + kCkptGroup - 1) / kCkptGroup * (kCkptGroup / VEC);
  float ss = 0.f;
  for (int i0 = 0; i0 < ng; i0 += 64) {
    const int i = i0 + lane;
    float v[VEC];
    const Vec<T, VEC> h = i < nv ? *(const Vec<T, VEC>*)(x + i * VEC) : Vec<T, VEC>{};
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = (float)h.e[k];
    if (i < nv) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) ss += v[k] * v[k];
    }
    const int ex = ckpt_exponent(ckpt_most(v));
    if (i < ng) {
      if constexpr (VEC % 4 == 0) {
        Vec<uint32_t, VEC / 4> b;
        ckpt_bytes(v, ex, b.e);
        *(Vec<uint32_t, VEC / 4>*)(q + row * ldq + i * VEC) = b;
      } else {
        q[row * ldq + i] = ckpt_byte(v[0], ex);
      }
      if (i % (kCkptGroup / VEC) == 0) e[row * lde + i / (kCkptGroup / VEC)] = (uint8_t)ex;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
  const float rs = 1.0f / sqrtf(ss / (float)d + eps);
  if (lane == 0) rstd[row] = rs;
#pragma unroll 4
  for (int i = lane; i < nv; i += 64) {
    const Vec<T, VEC> h = *(const Vec<T, VEC>*)(x + i * VEC), g = *(const Vec<T, VEC>*)(gamma + i * VEC);
    Vec<T, VEC> o;
#pragma unroll
    for (int k = 0; k < VEC; ++k) o.e[k] = (T)((float)h.e[k] * rs * (float)g.e[k]);
    *(Vec<T, VEC>*)(U + row * d + i * VEC) = o;
  }
}

// The norm recompute from a checkpoint: H (its values), U = norm(H) gamma and rstd, a wave per row, the sums in the order of
// the norm kernels that read H itself (VEC columns per lane and step), so that U is theirs bit for bit.  One launch and
// one read of the bytes where unpacking and norm are two, the second with a read of H.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void rmsnorm_ckpt_kernel(const int8_t* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ e,
                                                           int64_t lde, const T* __restrict__ gamma, float eps, T* __restrict__ H,
                                                           T* __restrict__ U, float* __restrict__ rstd, int64_t rows, int d) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int nv = d / VEC;
  float ss = 0.f;
#pragma unroll 4
  for (int i = lane; i < nv; i += 64) {
    float v[VEC];
    ckpt_unpack(*(const CkptBytes<VEC>*)(q + row * ldq + i * VEC), e[row * lde + i * VEC / kCkptGroup], v);
    Vec<T, VEC> h;
#pragma unroll
    for (int k = 0; k < VEC; ++k) { h.e[k] = (T)v[k]; ss += v[k] * v[k]; }
    *(Vec<T, VEC>*)(H + row * d + i * VEC) = h;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
  const float rs = 1.0f / sqrtf(ss / (float)d + eps);
  if (lane == 0) rstd[row] = rs;
#pragma unroll 4
  for (int i = lane; i < nv; i += 64) {
    float v[VEC];
    ckpt_unpack(*(const CkptBytes<VEC>*)(q + row * ldq + i * VEC), e[row * lde + i * VEC / kCkptGroup], v);
    const Vec<T, VEC> g = *(const Vec<T, VEC>*)(gamma + i * VEC);
    Vec<T, VEC> o;
#pragma unroll
    for (int k = 0; k < VEC; ++k) o.e[k] = (T)(v[k] * rs * (float)g.e[k]);
    *(Vec<T, VEC>*)(U + row * d + i * VEC) = o;
  }
}

// The SwiGLU backward from checkpoints of G and Z: dA (in DG) -> DG = dG, DZ = dZ, AA = silu(G) Z, zeros behind f.  16 bytes of
// each output per lane; ldf (a multiple of 8) is no more than the groups of a row hold.
template <typename T>
__global__ __launch_bounds__(256) void swiglu_bwd_ckpt_kernel(Ckpt G, Ckpt Z, T* DG, T* __restrict__ DZ, T* __restrict__ AA, int64_t ldf,
                                                              int64_t b, int f) {
  constexpr int N = kCols<T>;
  const int nv = (int)(ldf / N);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= b * nv) return;
  const int64_t r = i / nv;
  const int c = (int)(i - r * nv) * N;
  float g[N], z[N];
  const CkptBytes<N> bg = *(const CkptBytes<N>*)(G.q + r * G.ldq + c), bz = *(const CkptBytes<N>*)(Z.q + r * Z.ldq + c);
  const int eg = G.e[r * G.lde + c / kCkptGroup], ez = Z.e[r * Z.lde + c / kCkptGroup];
  const Vec<T, N> da = *(const Vec<T, N>*)(DG + r * ldf + c);
  ckpt_unpack(bg, eg, g);
  ckpt_unpack(bz, ez, z);
  Vec<T, N> odg, odz, oa;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const SwigluGrad o = swiglu_grad<sizeof(T) == 4>(g[k], z[k], (float)da.e[k]);
    const bool in = c + k < f;
    odg.e[k] = (T)(in ? o.dg : 0.f);
    odz.e[k] = (T)(in ? o.dz : 0.f);
    oa.e[k] = (T)(in ? o.a : 0.f);
  }
  *(Vec<T, N>*)(DG + r * ldf + c) = odg;
  *(Vec<T, N>*)(DZ + r * ldf + c) = odz;
  *(Vec<T, N>*)(AA + r * ldf + c) = oa;
}

inline unsigned blocks_for(int64_t n) { return (unsigned)((n + 255) / 256); }
inline bool rows_aligned(const void* p, int64_t ld, int esz) { return ((uintptr_t)p | (uintptr_t)(ld * esz)) % 16 == 0; }

}  // namespace

hipError_t launch_ckpt_pack(bool bf16, const void* X, int64_t ldx, int64_t rows, int cols, const Ckpt& k, hipStream_t s) {
  auto go = [&](auto type, auto al) {
    using T = decltype(type);
    const uint32_t per = (cols + kCkptGroup - 1) / kCkptGroup * (kCkptGroup / kPackCols), pieces = (uint32_t)rows * per;
    hipLaunchKernelGGL((ckpt_pack_kernel<T, decltype(al)::value>), dim3(blocks_for(pieces)), dim3(256), 0, s, (const T*)X, ldx, pieces, cols, per, k.q, k.ldq, k.e, k.lde);
  };
  if (bf16) go(__bf16{}, std::true_type{});
  else if (rows_aligned(X, ldx, 4)) go(float{}, std::true_type{});
  else go(float{}, std::false_type{});
  return hipGetLastError();
}

hipError_t launch_ckpt_unpack(bool bf16, const Ckpt& k, int64_t rows, int cols, void* X, int64_t ldx, hipStream_t s) {
  auto go = [&](auto type, auto al) {
    using T = decltype(type);
    const uint32_t per = (cols + kCkptGroup - 1) / kCkptGroup * (kCkptGroup / kCols<T>), pieces = (uint32_t)rows * per;
    hipLaunchKernelGGL((ckpt_unpack_kernel<T, decltype(al)::value>), dim3(blocks_for((pieces + kUnits - 1) / kUnits)), dim3(256), 0, s,
                       k.q, k.ldq, k.e, k.lde, pieces, cols, per, (T*)X, ldx);
  };
  if (bf16) go(__bf16{}, std::true_type{});
  else if (rows_aligned(X, ldx, 4)) go(float{}, std::true_type{});
  else go(float{}, std::false_type{});
  return hipGetLastError();
}

hipError_t launch_rmsnorm_pack(bool bf16, const void* X, int64_t ldx, const void* gamma, float eps, void* U, float* rstd, int64_t rows,
                               int d, const Ckpt& k, hipStream_t s) {
  const dim3 grid((unsigned)((rows + 3) / 4));
  if (bf16)
    hipLaunchKernelGGL((rmsnorm_pack_kernel<__bf16, 8>), grid, dim3(256), 0, s, (const __bf16*)X, ldx, (const __bf16*)gamma, eps, (__bf16*)U,
                       rstd, rows, d, k.q, k.ldq, k.e, k.lde);
  else
    hipLaunchKernelGGL((rmsnorm_pack_kernel<float, 1>), grid, dim3(256), 0, s, (const float*)X, ldx, (const float*)gamma, eps, (float*)U,
                       rstd, rows, d, k.q, k.ldq, k.e, k.lde);
  return hipGetLastError();
}

hipError_t launch_rmsnorm_ckpt(bool bf16, const Ckpt& k, const void* gamma, float eps, void* H, void* U, float* rstd, int64_t rows, int d,
                               hipStream_t s) {
  const dim3 grid((unsigned)((rows + 3) / 4));
  if (bf16)
    hipLaunchKernelGGL((rmsnorm_ckpt_kernel<__bf16, 8>), grid, dim3(256), 0, s, k.q, k.ldq, k.e, k.lde, (const __bf16*)gamma, eps, (__bf16*)H,
                       (__bf16*)U, rstd, rows, d);
  else
    hipLaunchKernelGGL((rmsnorm_ckpt_kernel<float, 1>), grid, dim3(256), 0, s, k.q, k.ldq, k.e, k.lde, (const float*)gamma, eps, (float*)H,
                       (float*)U, rstd, rows, d);
  return hipGetLastError();
}

hipError_t launch_swiglu_bwd_ckpt(bool bf16, const Ckpt& G, const Ckpt& Z, void* DG, void* DZ, void* AA, int64_t ldf, int64_t b, int f,
                                  hipStream_t s) {
  if (bf16)
    hipLaunchKernelGGL(swiglu_bwd_ckpt_kernel<__bf16>, dim3(blocks_for(b * (ldf / 8))), dim3(256), 0, s, G, Z, (__bf16*)DG, (__bf16*)DZ,
                       (__bf16*)AA, ldf, b, f);
  else
    hipLaunchKernelGGL(swiglu_bwd_ckpt_kernel<float>, dim3(blocks_for(b * (ldf / 4))), dim3(256), 0, s, G, Z, (float*)DG, (float*)DZ,
                       (float*)AA, ldf, b, f);
  return hipGetLastError();
}

bool reaches_2gib(int64_t rows, int64_t ld, int esz) {
  const int64_t most = (int64_t)1 << 31;
  return rows > 0 && (rows >= most || ld >= most || rows * ld >= most / esz);
}

int check_ckpt(const mecefo_ckpt_t* k, int64_t rows, int cols, const char* name, Ckpt* out) {
  if (!k) return fail(MECEFO_ERR_INVALID_ARG, "checkpoint %s is NULL", name);
  if (rows > 0 && (!k->q || !k->e)) return fail(MECEFO_ERR_INVALID_ARG, "checkpoint %s: q and e are required", name);
  if ((uintptr_t)k->q % 16 || k->ld_q % 16) return fail(MECEFO_ERR_INVALID_ARG, "checkpoint %s: q must be 16-byte aligned and ld_q a multiple of 16", name);
  const int64_t groups = ((int64_t)cols + 31) / 32;
  if (k->ld_q < 32 * groups || k->ld_e < groups)
    return fail(MECEFO_ERR_INVALID_ARG, "checkpoint %s: %d columns need ld_q >= %lld and ld_e >= %lld", name, cols, (long long)(32 * groups), (long long)groups);
  if (reaches_2gib(rows, k->ld_q, 1) || reaches_2gib(rows, k->ld_e, 1)) return fail(MECEFO_ERR_UNSUPPORTED, "checkpoint %s reaches 2 GiB", name);
  *out = Ckpt{(int8_t*)k->q, (uint8_t*)k->e, k->ld_q, k->ld_e};
  return MECEFO_OK;
}

namespace {
mecefo_status_t check_call(mecefo_dtype_t dtype, const void* X, int64_t rows, int cols, int64_t ldx, const mecefo_ckpt_t* ckpt, Ckpt* k) {
  if (dtype != MECEFO_F32 && dtype != MECEFO_BF16) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "dtype must be MECEFO_F32 or MECEFO_BF16");
  if (rows < 0 || cols < 1) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "rows >= 0 and cols >= 1 required");
  if (ldx < cols) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "a row stride is smaller than the logical width");
  const bool bf16 = dtype == MECEFO_BF16;
  if (bf16 && ldx % 8) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "bf16 path needs every row stride to be a multiple of 8 elements");
  if (rows > 0 && !X) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "X is NULL");
  if ((uintptr_t)X % (bf16 ? 16 : 4)) return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "X is not %d-byte aligned", bf16 ? 16 : 4);
  if (reaches_2gib(rows, ldx, bf16 ? 2 : 4)) return (mecefo_status_t)fail(MECEFO_ERR_UNSUPPORTED, "a tensor reaches 2 GiB; split the rows");
  const int ck = check_ckpt(ckpt, rows, cols, "ckpt", k);
  if (ck != MECEFO_OK) return (mecefo_status_t)ck;
  const uintptr_t x = (uintptr_t)X, q = (uintptr_t)k->q, e = (uintptr_t)k->e;
  // from the first element to the last: what lies behind a last row's columns may belong to another tensor
  const int64_t groups = ((int64_t)cols + 31) / 32;
  const uintptr_t nx = ((rows - 1) * ldx + cols) * (bf16 ? 2 : 4), nq = (rows - 1) * k->ldq + 32 * groups, ne = (rows - 1) * k->lde + groups;
  if (rows > 0 && ((x < q + nq && q < x + nx) || (x < e + ne && e < x + nx) || (q < e + ne && e < q + nq)))
    return (mecefo_status_t)fail(MECEFO_ERR_INVALID_ARG, "the tensor and the parts of its checkpoint overlap");
  return MECEFO_OK;
}
}  // namespace
}  // namespace mecefo

using namespace mecefo;

extern "C" {

mecefo_status_t mecefo_checkpoint_pack(mecefo_dtype_t dtype, const void* X, int64_t rows, int cols, int64_t ldx,
                                       const mecefo_ckpt_t* ckpt, void* hip_stream) {
  Ckpt k;
  const mecefo_status_t st = check_call(dtype, X, rows, cols, ldx, ckpt, &k);
  if (st != MECEFO_OK) return st;
  if (rows == 0) return MECEFO_OK;
  const hipError_t e = launch_ckpt_pack(dtype == MECEFO_BF16, X, ldx, rows, cols, k, (hipStream_t)hip_stream);
  if (e != hipSuccess) return (mecefo_status_t)fail(MECEFO_ERR_LAUNCH, "checkpoint_pack: %s", hipGetErrorString(e));
  return MECEFO_OK;
}

mecefo_status_t mecefo_checkpoint_unpack(mecefo_dtype_t dtype, const mecefo_ckpt_t* ckpt, int64_t rows, int cols, void* X,
                                         int64_t ldx, void* hip_stream) {
  Ckpt k;
  const mecefo_status_t st = check_call(dtype, X, rows, cols, ldx, ckpt, &k);
  if (st != MECEFO_OK) return st;
  if (rows == 0) return MECEFO_OK;
  const hipError_t e = launch_ckpt_unpack(dtype == MECEFO_BF16, k, rows, cols, X, ldx, (hipStream_t)hip_stream);
  if (e != hipSuccess) return (mecefo_status_t)fail(MECEFO_ERR_LAUNCH, "checkpoint_unpack: %s", hipGetErrorString(e));
  return MECEFO_OK;
}

}  // extern "C"
