// Where the tokens of a sequence and of its slices lie.  Host and device: plain arithmetic.
#pragma once
#include <stdint.h>

#ifdef __HIP__
#define MECEFO_RANGE __host__ __device__ inline
#else
#define MECEFO_RANGE inline
#endif

namespace mecefo {

struct TokenRange { int64_t lo, hi; };

// Sequence [a, b) of `tokens` tokens: always inside [0, tokens], also where the offsets are not, or decrease.
MECEFO_RANGE TokenRange token_range(int64_t a, int64_t b, int64_t tokens) {
  TokenRange r;
  r.lo = a < 0 ? 0 : (a > tokens ? tokens : a);
  r.hi = b < r.lo ? r.lo : (b > tokens ? tokens : b);
  return r;
}

// Slice j of n: whole multiples of 64 tokens but for the last one that has any.  tokens < 2^29.
MECEFO_RANGE TokenRange token_slice(TokenRange r, int j, int n) {
  const uint32_t len = (uint32_t)(r.hi - r.lo);
  const int64_t step = (int64_t)((len + 64u * n - 1) / (64u * n)) * 64, lo = r.lo + step * j, hi = lo + step;
  return TokenRange{lo < r.hi ? lo : r.hi, hi < r.hi ? hi : r.hi};
}

}  // namespace mecefo
