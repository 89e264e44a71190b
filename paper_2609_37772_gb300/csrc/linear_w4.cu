// The projection of few tokens with 4-bit weights.
#include <cmath>
#include <cstring>

#include "../../include/uad.h"
#include "kv_pages.cuh"
#include "once_per_device.h"
#include "ptx.cuh"
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

// mma.sync m16n8k16 with 16 weight rows as A and 8 tokens as B. A warp walks its rows in chunks of 128 k (64 bytes a row),
// which it copies ahead into a ring of its own (cp.async; rows 80 bytes apart, so that eight rows' words lie in different
// banks). Step i of a chunk is k = 32 i .. 32 i + 31, of which lane (g, t) has the word of k = 32 i + 8 t .. + 7 of rows g and g + 8:
// the contraction's order is free, so a pair is (k, k + 4), whose bits one mask takes out of the word, and a step lies in
// one group. 0x4300 | q is the bf16 128 + q; minus 128 + zero leaves q - zero, exactly. Tokens are read as they lie, 16 bytes
// a lane, and put in the same order.
constexpr int kChunk = 128, kRowPitch = 80, kW4Warps = 8;

__device__ __forceinline__ void w4_mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t sub2(uint32_t x, uint32_t y) {
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&y));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t lds4(uint32_t s) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(s) : "memory");
  return v;
}

// Copies in flight a warp: about 10 KB.
template <int RT>
constexpr int w4_slots() { return RT == 1 ? 8 : RT == 2 ? 4 : 3; }
template <int RT>
constexpr size_t w4_smem() { return (size_t)kW4Warps * w4_slots<RT>() * RT * 16 * kRowPitch; }

template <int NT, int RT, int G>   // 8 NT tokens, 16 RT rows a warp, group
__global__ void __launch_bounds__(32 * kW4Warps, RT * NT > 3 ? 1 : 2) w4_kernel(const W4Args a, int wn) {
  constexpr int SLOTS = w4_slots<RT>(), SLOT = RT * 16 * kRowPitch, PG = kChunk / G;
  static_assert(RT * NT * 512 <= SLOTS * SLOT, "the warps' sums fit the ring");
  extern __shared__ __align__(16) unsigned char smem[];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int wk = kW4Warps / wn, kw = warp / wn;   // warps that share rows, and which of them this is
  const int n0 = (blockIdx.x * wn + warp % wn) * RT * 16;
  const int groups = a.K / G, chunks = (a.K + kChunk - 1) / kChunk, mine = n0 < a.N ? (chunks - kw + wk - 1) / wk : 0;
  const uint32_t ring = ptx::su32(smem) + warp * SLOTS * SLOT;

  // 16 bytes a lane: 4 lanes a row's 64 bytes, 8 rows at a time
  const uint8_t* src = a.q + (((int64_t)n0 + g) * a.K >> 1) + 16 * t;
  const int64_t step8 = (int64_t)a.K * 4;   // 8 rows on
  const auto copy = [&](int i, int slot) {
    if (i < mine) {
      const int k = (kw + i * wk) * kChunk;
#pragma unroll
      for (int r = 0; r < 2 * RT; ++r) {
        const bool ok = n0 + 8 * r + g < a.N && k + 32 * t < a.K;
        const uint8_t* p = ok ? src + r * step8 + (k >> 1) : a.q;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ring + slot * SLOT + (8 * r + g) * kRowPitch + 16 * t), "l"(p), "r"(ok ? 16 : 0)
                     : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < SLOTS - 1; ++i) copy(i, i);

  float acc[RT][NT][4] = {};
  // scales and zero points of a chunk's groups, loaded a chunk ahead
  uint16_t sc[RT][2][PG], sn[RT][2][PG];
  uint8_t zc[RT][2][PG], zn[RT][2][PG];
  const auto load_groups = [&](int i) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < PG; ++j) {
          const int gr = (kw + i * wk) * PG + j, n = n0 + 16 * r + 8 * h + g;
          const bool ok = i < mine && gr < groups && n < a.N;
          const int64_t e = (int64_t)n * groups + gr;
          sn[r][h][j] = ok ? reinterpret_cast<const uint16_t*>(a.scale)[e] : (uint16_t)0;
          zn[r][h][j] = ok && a.zero ? a.zero[e] : (uint8_t)8;
        }
  };
  load_groups(0);
  int slot = 0;
  for (int i = 0; i < mine; ++i) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < PG; ++j) sc[r][h][j] = sn[r][h][j], zc[r][h][j] = zn[r][h][j];
    load_groups(i + 1);
    const int k0 = (kw + i * wk) * kChunk + 8 * t;
    asm volatile("cp.async.wait_group %0;" ::"n"(SLOTS - 2) : "memory");
    __syncwarp();   // all lanes' copies are there, and what the next copy overwrites has been read
    copy(i + SLOTS - 1, slot == 0 ? SLOTS - 1 : slot - 1);
    const uint32_t ws = ring + slot * SLOT + g * kRowPitch + 4 * t;
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
    float part[RT][NT][4];
    uint32_t z[RT][2];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      constexpr int kStepsOfGroup = G / 32;
      if (s % kStepsOfGroup == 0) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            z[r][h] = 0x43004300u | (zc[r][h][s / kStepsOfGroup] & 15u) * 0x10001u;
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[r][n][e] = 0.f;
        }
      }
      uint32_t xb[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (8 * n + g < a.M && k0 + 32 * s < a.K) v = __ldg(reinterpret_cast<const uint4*>(a.x + (int64_t)(8 * n + g) * a.K + k0 + 32 * s));
        xb[n][0] = __byte_perm(v.x, v.z, 0x5410);
        xb[n][1] = __byte_perm(v.x, v.z, 0x7632);
        xb[n][2] = __byte_perm(v.y, v.w, 0x5410);
        xb[n][3] = __byte_perm(v.y, v.w, 0x7632);
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint32_t w0 = lds4(ws + (16 * r) * kRowPitch + 16 * s), w1 = lds4(ws + (16 * r + 8) * kRowPitch + 16 * s);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          uint32_t f[4];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            f[2 * u] = sub2((w0 >> (4 * (2 * y + u)) & 0x000f000fu) | 0x43004300u, z[r][0]);
            f[2 * u + 1] = sub2((w1 >> (4 * (2 * y + u)) & 0x000f000fu) | 0x43004300u, z[r][1]);
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) w4_mma(part[r][n], f, xb[n][2 * y], xb[n][2 * y + 1]);
        }
      }
      if ((s + 1) % kStepsOfGroup == 0) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float s0 = __uint_as_float((uint32_t)sc[r][0][s / kStepsOfGroup] << 16), s1 = __uint_as_float((uint32_t)sc[r][1][s / kStepsOfGroup] << 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            acc[r][n][0] += part[r][n][0] * s0;
            acc[r][n][1] += part[r][n][1] * s0;
            acc[r][n][2] += part[r][n][2] * s1;
            acc[r][n][3] += part[r][n][3] * s1;
          }
        }
      }
    }
  }

  // the sums of the warps that share rows: [warp][token][row]
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);
  constexpr int ROWS = 16 * RT, TOK = 8 * NT;
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sums[(warp * TOK + 8 * n + 2 * t + (e & 1)) * ROWS + 16 * r + 8 * (e >> 1) + g] = acc[r][n][e];
  __syncthreads();
  for (int i = threadIdx.x; i < a.M * wn * ROWS; i += 32 * kW4Warps) {
    const int m = i / (wn * ROWS), r = i % (wn * ROWS), n = blockIdx.x * wn * ROWS + r;
    if (n >= a.N) continue;
    float v = 0.f;
    for (int w = 0; w < wk; ++w) v += sums[((w * wn + r / ROWS) * TOK + m) * ROWS + r % ROWS];
    a.out[(int64_t)m * a.N + n] = v + (a.bias ? a.bias[n] : 0.f);
  }
}

template <int NT, int RT, int G>
cudaError_t launch_w4(const W4Args& a, int wn, cudaStream_t s) {
  static OncePerDevice once;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  constexpr int smem = (int)w4_smem<RT>();
  e = (cudaError_t)once.run(dev, [&] { return (int)cudaFuncSetAttribute(w4_kernel<NT, RT, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); });
  if (e != cudaSuccess) return e;
  const int rows = 16 * RT * wn;
  return launch_k(w4_kernel<NT, RT, G>, dim3((unsigned)(((int64_t)a.N + rows - 1) / rows)), 32 * kW4Warps, smem, s, a, wn);
}

template <int G>
cudaError_t launch_group(const W4Args& a, cudaStream_t s) {
  const int tiles = (a.N + 15) / 16;   // of 16 rows
  const int tokens = (a.M + 7) / 8;
  if (tokens == 1) return tiles >= 152 * 8 ? launch_w4<1, 2, G>(a, 2, s) : launch_w4<1, 1, G>(a, 1, s);
  if (tokens == 2) return tiles >= 152 * 8 ? launch_w4<2, 2, G>(a, 2, s) : launch_w4<2, 1, G>(a, 1, s);
  if (tokens <= 4) return tiles >= 152 * 4 ? launch_w4<4, 2, G>(a, 2, s) : launch_w4<4, 1, G>(a, 1, s);
  if (tokens <= 6) return tiles >= 152 * 4 ? launch_w4<6, 2, G>(a, 2, s) : launch_w4<6, 1, G>(a, 1, s);
  return tiles >= 152 * 4 ? launch_w4<8, 2, G>(a, 2, s) : launch_w4<8, 1, G>(a, 1, s);
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
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = group == 32 ? launch_group<32>(a, s) : group == 64 ? launch_group<64>(a, s) : launch_group<128>(a, s);
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
