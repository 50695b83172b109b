// Activation checkpoints in 8 bits: a row is cut into groups of 32 columns, a group holds 32 signed bytes q and one byte e,
// and stands for the values q 2^(e - 127).  e is the exponent of the group's largest magnitude less 6, so that the largest
// byte lies in 64 .. 127, and q = x 2^(127 - e) rounded to the nearest whole number (halves to even), at most 127.
// A power of two and seven bits: every value is a bf16 number, so unpacking is exact in either storage type, and the
// scaling is exact in both directions, so the bytes do not depend on the order or the kind of the arithmetic.  Against one
// fp32 scale per 128 columns (the same bytes per value) the step is up to twice as wide where the largest value lies just
// above a power of two, but a loud column only costs the 31 next to it.  A group with an infinity or a NaN is NaN throughout.
#include "checkpoint.hip.h"
#include "mecefo_internal.h"

namespace mecefo {
namespace {

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Vec { T e[VEC]; };

// 16 columns per lane, two lanes to a group.  ALIGNED: rows start on 16 bytes, so that whole lanes load vectors.
template <typename T, bool ALIGNED>
__device__ inline void load16(const T* x, int n, float (&v)[16]) {
  constexpr int PER = 16 / sizeof(T);
  if (ALIGNED && n >= 16) {
#pragma unroll
    for (int q = 0; q < 16 / PER; ++q) {
      const Vec<T, PER> a = *(const Vec<T, PER>*)(x + q * PER);
#pragma unroll
      for (int k = 0; k < PER; ++k) v[q * PER + k] = (float)a.e[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = k < n ? (float)x[k] : 0.f;
  }
}
template <typename T, bool ALIGNED>
__device__ inline void store16(T* x, int n, const float (&v)[16]) {
  constexpr int PER = 16 / sizeof(T);
  if (ALIGNED && n >= 16) {
#pragma unroll
    for (int q = 0; q < 16 / PER; ++q) {
      Vec<T, PER> a;
#pragma unroll
      for (int k = 0; k < PER; ++k) a.e[k] = (T)v[q * PER + k];
      *(Vec<T, PER>*)(x + q * PER) = a;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (k < n) x[k] = (T)v[k];
  }
}

template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void ckpt_pack_kernel(const T* __restrict__ X, int64_t ldx, int64_t rows, int cols, int per,
                                                        int8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ e, int64_t lde) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;      // per is even: the two lanes of a group share a row
  const int64_t row = i / per;
  if (row >= rows) return;
  const int c = (int)(i - row * per) * 16;
  float v[16];
  load16<T, ALIGNED>(X + row * ldx + c, cols - c, v);
  uint32_t bytes[4];
  const int ex = ckpt_pack16(v, bytes, 2);
  *(Vec<uint32_t, 4>*)(q + row * ldq + c) = Vec<uint32_t, 4>{{bytes[0], bytes[1], bytes[2], bytes[3]}};
  if ((c & 16) == 0) e[row * lde + (c >> 5)] = (uint8_t)ex;
}

template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void ckpt_unpack_kernel(const int8_t* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ e,
                                                          int64_t lde, int64_t rows, int cols, int per, T* __restrict__ X, int64_t ldx) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / per;
  if (row >= rows) return;
  const int c = (int)(i - row * per) * 16;
  const Vec<uint32_t, 4> b = *(const Vec<uint32_t, 4>*)(q + row * ldq + c);
  float v[16];
  ckpt_unpack16(b.e, e[row * lde + (c >> 5)], v);
  store16<T, ALIGNED>(X + row * ldx + c, cols - c, v);
}

inline unsigned blocks_for(int64_t n) { return (unsigned)((n + 255) / 256); }
inline int lanes_per_row(int cols) { return (cols + 31) / 32 * 2; }
inline bool rows_aligned(const void* p, int64_t ld, int esz) { return ((uintptr_t)p | (uintptr_t)(ld * esz)) % 16 == 0; }

}  // namespace

hipError_t launch_ckpt_pack(bool bf16, const void* X, int64_t ldx, int64_t rows, int cols, const Ckpt& k, hipStream_t s) {
  const int per = lanes_per_row(cols);
  const dim3 grid(blocks_for(rows * per));
  auto go = [&](auto type, auto al) {
    using T = decltype(type);
    hipLaunchKernelGGL((ckpt_pack_kernel<T, decltype(al)::value>), grid, dim3(256), 0, s, (const T*)X, ldx, rows, cols, per, k.q, k.ldq,
                       k.e, k.lde);
  };
  if (bf16) go(__bf16{}, std::true_type{});
  else if (rows_aligned(X, ldx, 4)) go(float{}, std::true_type{});
  else go(float{}, std::false_type{});
  return hipGetLastError();
}

hipError_t launch_ckpt_unpack(bool bf16, const Ckpt& k, int64_t rows, int cols, void* X, int64_t ldx, hipStream_t s) {
  const int per = lanes_per_row(cols);
  const dim3 grid(blocks_for(rows * per));
  auto go = [&](auto type, auto al) {
    using T = decltype(type);
    hipLaunchKernelGGL((ckpt_unpack_kernel<T, decltype(al)::value>), grid, dim3(256), 0, s, k.q, k.ldq, k.e, k.lde, rows, cols, per, (T*)X,
                       ldx);
  };
  if (bf16) go(__bf16{}, std::true_type{});
  else if (rows_aligned(X, ldx, 4)) go(float{}, std::true_type{});
  else go(float{}, std::false_type{});
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
  const uintptr_t nx = rows * ldx * (bf16 ? 2 : 4), nq = rows * k->ldq, ne = rows * k->lde;
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
