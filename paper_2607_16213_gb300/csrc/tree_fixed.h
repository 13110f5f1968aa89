// Probabilities as 64-bit fixed point: plain C++, so that it can be tested without a device.
#pragma once

#include <cstdint>
#include <cstring>

#ifdef __CUDACC__
#define SELKV_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define SELKV_HOST_DEVICE inline
#endif

namespace selkv {

// A probability in units of 2^-62 (cut off); one that is none, of 2 or more, negative or NaN, counts as 0.
SELKV_HOST_DEVICE unsigned long long to_fix(float p, bool& bad) {
  const bool ok = p >= 0.f && p < 2.f;
  bad = bad || !ok;
  uint32_t u;
#ifdef __CUDA_ARCH__
  u = __float_as_uint(p);
#else
  std::memcpy(&u, &p, sizeof(u));
#endif
  u = ok ? u & 0x7fffffffu : 0u;  // (-0 is a zero: its sign would shift the mantissa out of the word)
  // the mantissa in its place, by shifts (the conversion instruction runs at a quarter of their rate)
  const int shift = (int)(u >> 23) - 88;
  const unsigned long long m = (u & 0x7fffffu) | 0x800000u;
  return shift >= 0 ? m << shift : shift > -32 ? (unsigned long long)((uint32_t)m >> -shift) : 0ull;
}

}  // namespace selkv
