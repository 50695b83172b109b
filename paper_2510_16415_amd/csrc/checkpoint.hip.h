// Device side of the 8-bit checkpoints: the values of a group that a lane holds, to bytes and back.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/mecefo.h"
#include "mecefo_internal.h"

namespace mecefo {

// The descriptor as the kernels take it, after the checks of an entry point (a mecefo_status_t; the message names `name`).
int check_ckpt(const mecefo_ckpt_t* k, int64_t rows, int cols, const char* name, Ckpt* out);

constexpr int kCkptGroup = 32;
template <int N> struct alignas(N) CkptBytes { int8_t q[N]; };      // what a lane of N columns holds of q

// 2^(e - 127) for e = 1 .. 254, NaN for 255, 0 for 0 (which packing never writes).
__device__ inline float ckpt_power(int e) { return e == 255 ? __builtin_nanf("") : __builtin_bit_cast(float, (uint32_t)e << 23); }

// The group's byte e from the largest magnitude of its values, as bits: the sign cleared, an infinity or a NaN is larger than
// every number.  At least 1, so that 2^(127 - e) and the values are normal numbers.
__device__ inline int ckpt_exponent(uint32_t most) {
  const int high = (int)(most >> 23);
  return high == 255 ? 255 : (high > 7 ? high : 7) - 6;
}

// Largest magnitude, as bits, of N values, and over the group's 32 / N neighbouring lanes.
template <int N> __device__ inline uint32_t ckpt_most(const float (&v)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t a = __builtin_bit_cast(uint32_t, v[k]) & 0x7FFFFFFFu;
    most = a > most ? a : most;
  }
#pragma unroll
  for (int o = 1; o < kCkptGroup / N; o *= 2) {
    const uint32_t a = __shfl_xor(most, o, 64);
    most = a > most ? a : most;
  }
  return most;
}

// N values (a multiple of four) to bytes.  Clamped to 127 steps first, x / step + 1.5 * 2^23 in one exact product and one
// rounding of the sum: the nearest whole number, halves to even, in the low bits of the result.
template <int N>
__device__ inline void ckpt_bytes(const float (&v)[N], int ex, uint32_t (&words)[N / 4]) {
  const int e = ex == 255 ? 127 : ex;
  const float inv = __builtin_bit_cast(float, (uint32_t)(254 - e) << 23), most = 127.f * __builtin_bit_cast(float, (uint32_t)e << 23);
#pragma unroll
  for (int w = 0; w < N / 4; ++w) {
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      b[k] = __builtin_bit_cast(uint32_t, __builtin_fmaf(__builtin_amdgcn_fmed3f(v[4 * w + k], -most, most), inv, 12582912.f));
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000C0Cu);
    words[w] = ex == 255 ? 0u : lo | hi;
  }
}

__device__ inline int8_t ckpt_byte(float v, int ex) {
  const int e = ex == 255 ? 127 : ex;
  const float inv = __builtin_bit_cast(float, (uint32_t)(254 - e) << 23), most = 127.f * __builtin_bit_cast(float, (uint32_t)e << 23);
  const float r = __builtin_fmaf(__builtin_amdgcn_fmed3f(v, -most, most), inv, 12582912.f);
  return ex == 255 ? (int8_t)0 : (int8_t)__builtin_bit_cast(uint32_t, r);
}

template <int N>
__device__ inline void ckpt_unpack(const CkptBytes<N>& b, int e, float (&v)[N]) {
  const float p = ckpt_power(e);
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = (float)b.q[k] * p;
}

}  // namespace mecefo
