// Whole-number arithmetic of the attention's units of work (gift_kv.hip): exact for every count that a call can have.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gift {

// a / b: the usual small a by way of floats, which takes a fraction of the steps of a 32-bit division.  Exact: below 2^23
// the product is off by less than the distance of a quotient from the next.
__host__ __device__ inline uint32_t quotient(uint32_t a, uint32_t b) {
  if (a >= 1u << 23) return a / b;
#if defined(__HIP_DEVICE_COMPILE__)
  const float q = (float)a * __builtin_amdgcn_rcpf((float)b);
#else
  const float q = (float)a * (1.f / (float)b);
#endif
  uint32_t n = (uint32_t)q;
  const int32_t left = (int32_t)(a - n * b);
  return left < 0 ? n - 1 : (uint32_t)left >= b ? n + 1 : n;
}

// a / b for a < 2^63, with the reciprocal of b: the product is off by a 2^51st of the quotient at most, which is less than 1
// as long as the quotient is below 2^51, and some steps beyond.
__host__ __device__ inline uint64_t quotient(uint64_t a, uint64_t b, double reciprocal) {
  uint64_t q = (uint64_t)((double)a * reciprocal);
  while ((int64_t)(a - q * b) < 0) q--;
  while (a - q * b >= b) q++;
  return q;
}

// A unit of a request: of which of its columns, and which round of that.  A request of many rows over a long cache has
// more than 2^32 of them (2^20 rows of 64 heads over 2^21 tokens).
struct Unit {
  uint32_t column, round;
};

__host__ __device__ inline Unit unit_of(uint64_t at, uint32_t rounds) {
  const uint32_t column =
      at >> 32 ? (uint32_t)quotient(at, rounds, 1.0 / (double)rounds) : quotient((uint32_t)at, rounds);
  return Unit{column, (uint32_t)(at - (uint64_t)column * rounds)};
}

}  // namespace gift
