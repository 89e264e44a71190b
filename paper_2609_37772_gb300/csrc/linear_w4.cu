// The projection of few tokens with 4-bit weights.
#include <cmath>
#include <cstring>

#include "../../include/uad.h"
#include "kv_pages.cuh"
#include "uad_internal.cuh"

using namespace uad;

namespace {

struct W4Args {
  const __nv_bfloat16* x;
  const uint8_t* q;
  const __nv_bfloat16* scale;
  const uint8_t* zero;
  const float* bias;
  float* out;
  int M, N, K, group;
};

// One warp an output: its lanes take bytes of the row in turn.
__global__ void __launch_bounds__(256) w4_kernel(const W4Args a) {
  pdl_wait();
  pdl_trigger();
  const int n = blockIdx.x * 8 + (threadIdx.x >> 5), m = blockIdx.y, lane = threadIdx.x & 31;
  if (n >= a.N) return;
  const int groups = a.K / a.group;
  float sum = 0.f;
  for (int g = 0; g < groups; ++g) {
    const int64_t e = (int64_t)n * groups + g;
    const int z = a.zero ? a.zero[e] & 15 : 8;
    float part = 0.f;
    for (int i = lane; i < a.group / 2; i += 32) {
      const int k = g * a.group + 2 * i;
      const int w = a.q[((int64_t)n * a.K + k) >> 1];
      part += __bfloat162float(a.x[(int64_t)m * a.K + k]) * (float)((w & 15) - z);
      part += __bfloat162float(a.x[(int64_t)m * a.K + k + 1]) * (float)((w >> 4) - z);
    }
    sum += part * __bfloat162float(a.scale[e]);
  }
  for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
  if (lane == 0) a.out[(int64_t)m * a.N + n] = sum + (a.bias ? a.bias[n] : 0.f);
}

// fp32 -> bf16 bits, nearest, ties to even, for finite values.
uint16_t bf16_bits(float f) {
  uint32_t u;
  memcpy(&u, &f, 4);
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}
float bf16_value(uint16_t h) {
  const uint32_t u = (uint32_t)h << 16;
  float f;
  memcpy(&f, &u, 4);
  return f;
}

}  // namespace

extern "C" {

int uad_linear_w4(const void* x, const uint8_t* q, const uint16_t* scale, const uint8_t* zero, const float* bias, float* out,
                  int32_t M, int32_t N, int32_t K, int32_t group, void* stream) {
  if (!x || !q || !scale || !out || M < 1 || N < 1 || K < 1) return UAD_EINVAL;
  if ((group != 32 && group != 64 && group != 128) || K % group || (int64_t)N * K >= (1ll << 40)) return UAD_EINVAL;
  if (reinterpret_cast<uintptr_t>(x) % 16 || reinterpret_cast<uintptr_t>(q) % 16 || reinterpret_cast<uintptr_t>(scale) % 2 ||
      reinterpret_cast<uintptr_t>(bias) % 4 || reinterpret_cast<uintptr_t>(out) % 4)
    return UAD_EINVAL;
  if (M > UAD_W4_MAX_ROWS) return UAD_ETOOBIG;
  if (!on_current_device(q)) return UAD_EINVAL;
  const W4Args a{static_cast<const __nv_bfloat16*>(x), q, reinterpret_cast<const __nv_bfloat16*>(scale), zero, bias, out, M, N, K, group};
  const cudaError_t e = launch_k(w4_kernel, dim3((N + 7) / 8, M), 256, 0, static_cast<cudaStream_t>(stream), a);
  return e == cudaSuccess ? UAD_OK : UAD_ECUDA;
}

int uad_quantize_w4(const float* w, int32_t K, int32_t N, int32_t group, uint8_t* q, uint16_t* scale, uint8_t* zero) {
  if (!w || !q || !scale || N < 1 || K < 1 || (group != 32 && group != 64 && group != 128) || K % group) return UAD_EINVAL;
  const int groups = K / group;
  for (size_t i = 0; i < (size_t)K * N; ++i)
    if (!std::isfinite(w[i])) return UAD_EINVAL;
  for (int n = 0; n < N; ++n)
    for (int g = 0; g < groups; ++g) {
      float lo = 0.f, hi = 0.f;
      for (int k = g * group; k < (g + 1) * group; ++k) {
        const float v = w[(size_t)k * N + n];
        lo = std::fmin(lo, v);
        hi = std::fmax(hi, v);
      }
      const size_t e = (size_t)n * groups + g;
      const float range = zero ? (hi / 15.f - lo / 15.f) : std::fmax(hi, -lo) / 7.f;
      const uint16_t bits = bf16_bits(range);
      const float s = bf16_value(bits);
      const bool usable = s > 0.f && std::isfinite(s);   // all zeros, or a range that bf16 does not hold
      scale[e] = usable ? bits : 0;
      int z = 8;
      if (zero) {
        z = usable ? (int)std::fmin(15.f, std::fmax(0.f, std::nearbyint(-lo / s))) : 0;
        zero[e] = (uint8_t)z;
      }
      const float least = zero ? 0.f : 1.f;   // symmetric: -7..7
      for (int k = g * group; k < (g + 1) * group; k += 2) {
        uint8_t byte = 0;
        for (int i = 0; i < 2; ++i) {
          const float v = usable ? std::nearbyint(w[(size_t)(k + i) * N + n] / s) + z : (float)z;
          byte |= (uint8_t)((int)std::fmin(15.f, std::fmax(least, v)) << (4 * i));
        }
        q[((size_t)n * K + k) / 2] = byte;
      }
    }
  return UAD_OK;
}

}  // extern "C"
