// Division of a position by a page size that is known on the host, as plain arithmetic (no CUDA, so that it can be
// compiled and checked on the host).
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define UAD_FD __host__ __device__ __forceinline__
#else
#define UAD_FD inline
#endif

namespace uad {

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31 with a multiplication: with s = ceil(log2 d) and
// m = floor(2^32 (2^s - d) / d) + 1, n / d = (hi32(m n) + n) >> s (Granlund and Montgomery, Division by invariant
// integers using multiplication, 1994). hi32(m n) <= n < 2^31, so the sum does not leave 32 bits.
struct FastDiv {
  uint32_t d = 1, m = 1, s = 0;
  FastDiv() = default;
  explicit FastDiv(uint32_t div) : d(div) {
    while (s < 31 && (1u << s) < d) ++s;
    m = (uint32_t)(((uint64_t)((1ull << s) - d) << 32) / d) + 1;
  }
  UAD_FD uint32_t div(uint32_t n) const { return ((uint32_t)(((uint64_t)m * n) >> 32) + n) >> s; }
};

}  // namespace uad
