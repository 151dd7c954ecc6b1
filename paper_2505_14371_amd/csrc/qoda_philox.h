// The counter-based generator of the quantizer and of dropout.
#pragma once

#include <hip/hip_runtime.h>

namespace qoda {

// Philox4x32-10 (Salmon et al., SC'11).
__device__ __forceinline__ void philox4x32_10(unsigned int c0, unsigned int c1, unsigned int c2, unsigned int c3,
                                               unsigned int k0, unsigned int k1, unsigned int out[4]) {
  constexpr unsigned long long M0 = 0xD2511F53ull, M1 = 0xCD9E8D57ull;
  constexpr unsigned int W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    if (r > 0) { k0 += W0; k1 += W1; }
    const unsigned long long p0 = M0 * (unsigned long long)c0;
    const unsigned long long p1 = M1 * (unsigned long long)c2;
    const unsigned int n0 = __builtin_amdgcn_bitop3_b32((unsigned int)(p1 >> 32), c1, k0, 0x96);   // 3-input xor
    const unsigned int n1 = (unsigned int)p1;
    const unsigned int n2 = __builtin_amdgcn_bitop3_b32((unsigned int)(p0 >> 32), c3, k1, 0x96);
    const unsigned int n3 = (unsigned int)p0;
    c0 = n0; c1 = n1; c2 = n2; c3 = n3;
  }
  out[0] = c0; out[1] = c1; out[2] = c2; out[3] = c3;
}

}  // namespace qoda
