// Device side of the 8-bit checkpoints: sixteen values of a group to bytes and back.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/mecefo.h"
#include "mecefo_internal.h"

namespace mecefo {

// The descriptor as the kernels take it, after the checks of an entry point (a mecefo_status_t; the message names `name`).
int check_ckpt(const mecefo_ckpt_t* k, int64_t rows, int cols, const char* name, Ckpt* out);

// 2^(e - 127) for e = 1 .. 254, NaN for 255, 0 for 0 (which packing never writes).
__device__ inline float ckpt_power(int e) { return e == 255 ? __builtin_nanf("") : __builtin_bit_cast(float, (uint32_t)e << 23); }

// The group's byte e from the largest magnitude of its values, as bits: the sign cleared, an infinity or a NaN is larger than
// every number.  At least 1, so that 2^(127 - e) and the values are normal numbers.
__device__ inline int ckpt_exponent(uint32_t most) {
  const int high = (int)(most >> 23);
  return high == 255 ? 255 : (high > 7 ? high : 7) - 6;
}

__device__ inline uint32_t ckpt_byte(float x, float inv) {
  const float r = __builtin_rintf(x * inv);
  return (uint32_t)(int)fminf(fmaxf(r, -127.f), 127.f) & 0xFFu;
}

// Sixteen values to bytes; a group is shared by `lanes` neighbouring lanes (2: all of them take part).
__device__ inline int ckpt_pack16(const float (&v)[16], uint32_t (&bytes)[4], int lanes) {
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const uint32_t a = __builtin_bit_cast(uint32_t, v[k]) & 0x7FFFFFFFu;
    most = a > most ? a : most;
  }
  for (int o = 1; o < lanes; o *= 2) {
    const uint32_t a = __shfl_xor(most, o, 64);
    most = a > most ? a : most;
  }
  const int ex = ckpt_exponent(most);
  const float inv = ex == 255 ? 0.f : __builtin_bit_cast(float, (uint32_t)(254 - ex) << 23);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t b = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) b |= (ex == 255 ? 0u : ckpt_byte(v[4 * w + k], inv)) << (8 * k);
    bytes[w] = b;
  }
  return ex;
}

__device__ inline void ckpt_unpack16(const uint32_t (&bytes)[4], int e, float (&v)[16]) {
  const float p = ckpt_power(e);
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = (float)(int8_t)(bytes[k >> 2] >> (8 * (k & 3))) * p;
}

}  // namespace mecefo
