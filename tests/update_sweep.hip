// Compares the square root, the reciprocal and the quotient of csrc/update_math.h with the correctly rounded ones, bit for bit: the first two for every
// significand (the root for both parities of the exponent), the quotient for 2^28 pairs.  Prints how many differ.
#include <cstdio>

#include "../paper_2602_02192_amd/csrc/update_math.h"

__global__ void roots(unsigned long long *off) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;   // 2^24 values from 1 to 4
  for (int e = -90; e <= 86; e += 44) {
    const float x = ldexpf(__uint_as_float(0x3f800000u + i), e);
    if (__float_as_uint(echo::moderate_sqrt(x)) != __float_as_uint((float)sqrt((double)x))) atomicAdd(off, 1ull);
  }
}
__global__ void reciprocals(unsigned long long *off) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;   // 2^23 values from 1 to 2
  for (int e = -60; e <= 60; e += 30) {
    const float x = ldexpf(__uint_as_float(0x3f800000u + i), e);
    if (__float_as_uint(echo::moderate_reciprocal(x)) != __float_as_uint((float)(1.0 / (double)x))) atomicAdd(off, 1ull);
  }
}
// (53 bits are enough that rounding the f64 root, reciprocal or quotient of f32 values once more gives the correctly rounded f32: S. Figueroa, 1995.)
__global__ void quotients(unsigned long long *off) {
  uint64_t s = (uint64_t)(blockIdx.x * 256 + threadIdx.x) * 0x9E3779B97F4A7C15ull + 77;
  for (int k = 0; k < 256; ++k) {
    s ^= s << 13; s ^= s >> 7; s ^= s << 17;
    const float n = ldexpf(__uint_as_float(0x3f800000u + ((uint32_t)s & 0x7fffff)), (int)(s >> 23 & 127) - 64);
    const float d = ldexpf(__uint_as_float(0x3f800000u + ((uint32_t)(s >> 32) & 0x7fffff)), (int)(s >> 56 & 63) - 40);
    if (__float_as_uint(echo::moderate_quotient(n, d)) != __float_as_uint((float)((double)n / (double)d))) atomicAdd(off, 1ull);
  }
}

int main() {
  unsigned long long *off, found[3];
  if (hipMalloc((void **)&off, sizeof found) != hipSuccess || hipMemset(off, 0, sizeof found) != hipSuccess) return 2;
  roots<<<(1 << 24) / 256, 256>>>(off);
  reciprocals<<<(1 << 23) / 256, 256>>>(off + 1);
  quotients<<<4096, 256>>>(off + 2);
  if (hipMemcpy(found, off, sizeof found, hipMemcpyDeviceToHost) != hipSuccess) return 2;
  printf("roots %llu reciprocals %llu quotients %llu\n", found[0], found[1], found[2]);
  return found[0] || found[1] || found[2];
}
