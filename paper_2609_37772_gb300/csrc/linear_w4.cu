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

constexpr int kChunk = 128, kW4Warps = 8, kSms = 152;

__device__ __forceinline__ uint32_t lds4(uint32_t s) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(s) : "memory");
  return v;
}

// Nibbles 0 and 4 of w as bf16: 128 + q. (x & mask) | constant in one instruction, which the compiler makes two of.
__device__ __forceinline__ uint32_t nibbles(uint32_t w) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(0x000f000fu), "r"(0x43004300u));
  return r;
}
__device__ __forceinline__ void mma_bf16_16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16_first(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t sub2(uint32_t x, uint32_t y) {
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&y));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// ---- up to 8 tokens: a stream of weights --------------------------------------------------------------------------------
//
// What bounds a few tokens, once the weights arrive at full bandwidth (14 cycles of an SM's quarter for 256 weights), is
// taking the nibbles apart: three shifts, four masks and four subtractions for the eight of a word, which make exact bf16 of
// q - zero (0x4300 | q is 128 + q; less 128 + zero). The tokens stay as they are, but for their order. A group's products are exact and
// summed in fp32, and the sum is then scaled. Products of q itself would save the subtractions, but sums of q x cancel against zero
// times the tokens' sum: a large token whose weights are all zero would take the small ones' bits.
// 1 token: 2048 x 32768 in groups of 128 13.3 us (2.65 TB/s), 4096 x 4096 6.3, 1024 x 2560 3.1; 8 of 2048 x 32768 14.4.
//
// A tile of 16 rows is walked by wk of a CTA's warps, which take its chunks in turn and add up in shared memory: one, where
// there are tiles enough for every warp, which saves the adding. A warp's copies run on from tile to tile. Where
// there are fewer tiles than CTAs, or the tokens do not fit, a cluster shares K.
//
// In a chunk of 128 k, group j is words 4 GS j .. of a row's 16, of which lane t has GS neighbours, read at once (GS = G / 32 steps of an
// MMA's 32 k): the order of k inside a group is free. Rows are so far apart in shared memory that this has no bank conflicts.
constexpr int kFewSlots = 5;          // chunks of a warp in the ring, four of them on their way: 64 KB an SM
constexpr int kFewX = 40 * 1024;      // bytes of tokens that a CTA should hold at most: two CTAs an SM
template <int G>
__host__ __device__ constexpr int few_pitch() { return G == 128 ? 64 : G == 64 ? 96 : 80; }
struct FewArgs {
  W4Args a;
  int split;        // CTAs of a cluster that share K
  int split_k;      // k of each, a multiple of kChunk
  int wk;           // warps of a tile: 1, 2, 4 or 8 (8 with a split)
  int per_cta;      // tiles that a CTA takes at a time, at most kW4Warps / wk
  FastDiv pieces;   // by the eights of k that a CTA holds
};
// A row's scales and zeros in a chunk, as the words they are loaded in.
template <int N>
struct Groups;
template <>
struct Groups<1> { uint16_t s; uint8_t z; };
template <>
struct Groups<2> { uint32_t s; uint16_t z; };
template <>
struct Groups<4> { uint64_t s; uint32_t z; };
constexpr int kAhead = 3;             // chunks that scales and zeros are loaded ahead
// Shared memory: 16 zeros; the warps' rings; their sums [2][warp][token][16]; the cluster's [2][rank][token][16]; the
// tokens [step][token][t] of 16 bytes. k: a multiple of kChunk.
template <int G>
__host__ __device__ inline size_t few_smem(int rows, int k) {
  return 16 + (size_t)kW4Warps * kFewSlots * 16 * few_pitch<G>() + (size_t)2 * kW4Warps * rows * 64 + (size_t)2 * 8 * rows * 64 +
         (size_t)rows * k * 2;
}

template <int G, bool VEC>   // VEC: a chunk's scales, and its zeros, are read as one word
__global__ void __launch_bounds__(32 * kW4Warps, 2) w4_few_kernel(const FewArgs f) {
  constexpr int PITCH = few_pitch<G>(), SLOT = 16 * PITCH, PG = kChunk / G, GS = G / 32;   // groups of a chunk, steps of a group
  extern __shared__ __align__(16) unsigned char smem[];
  pdl_wait();
  pdl_trigger();
  if (f.split > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // started: others may write here
  const W4Args& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int part = f.split > 1 ? blockIdx.x % f.split : 0, wk_bits = __ffs(f.wk) - 1, kw = warp & (f.wk - 1), of_cta = warp >> wk_bits;
  const int cta = f.split > 1 ? blockIdx.x / f.split : blockIdx.x, ctas = f.split > 1 ? gridDim.x / f.split : gridDim.x;
  const int tiles = (a.N + 15) / 16, groups = a.K / G, stride = ctas * f.per_cta;
  const int kb = part * f.split_k, ke = min(a.K, kb + f.split_k);
  int tile = cta * f.per_cta + of_cta, rounds = (tiles - cta * f.per_cta + stride - 1) / stride;   // of the CTA
  // this warp's chunks of a tile, and how many are left to copy and to find the scales of
  const int chunks = (ke - kb + kChunk - 1) / kChunk, mine = chunks > kw ? (chunks - kw + f.wk - 1) >> wk_bits : 0;
  const int own = of_cta < f.per_cta && tile < tiles && mine > 0 ? rounds - (tile + (rounds - 1) * stride >= tiles) : 0;   // rounds with work
  const uint32_t ring = ptx::su32(smem) + 16 + warp * kFewSlots * SLOT;
  float* red = reinterpret_cast<float*>(smem + 16 + kW4Warps * kFewSlots * SLOT);
  float* recv = red + 2 * kW4Warps * a.M * 16;
  unsigned char* xp = reinterpret_cast<unsigned char*>(recv + 2 * 8 * a.M * 16);
  const uint32_t xs = ptx::su32(xp);
  if (threadIdx.x < 4) reinterpret_cast<uint32_t*>(smem)[threadIdx.x] = 0;

  // Weights: 16 bytes a lane, 4 lanes a row's 64, rows g and g + 8 of the tile (past the last row: the last). What is past K is read
  // from the row's start, and the tokens are 0 there.
  int c_left = own * mine, c_tile = tile, c_i = 0, c_k = kb + kw * kChunk + 32 * t;
  const uint8_t *r0 = nullptr, *r1 = nullptr;
  const uint32_t to = ring + g * PITCH + 16 * t;
  const auto copy = [&](int slot) {
    if (c_left > 0) {
      if (c_i == 0) {
        r0 = a.q + ((int64_t)min(c_tile * 16 + g, a.N - 1) * a.K >> 1);
        r1 = a.q + ((int64_t)min(c_tile * 16 + 8 + g, a.N - 1) * a.K >> 1);
      }
      const int at = (c_k < ke ? c_k : kb + 32 * t < ke ? kb + 32 * t : kb) >> 1;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + slot * SLOT), "l"(r0 + at) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + slot * SLOT + 8 * PITCH), "l"(r1 + at) : "memory");
      --c_left;
      c_k += f.wk * kChunk;
      if (++c_i == mine) c_i = 0, c_k = kb + kw * kChunk + 32 * t, c_tile += stride;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kFewSlots - 1; ++i) copy(i);
  // scales and zeros
  int g_left = own * mine, g_tile = tile, g_i = 0, g_at = (kb + kw * kChunk) / G;
  const uint16_t *s0p = nullptr, *s1p = nullptr;
  const uint8_t *z0p = nullptr, *z1p = nullptr;
  Groups<PG> gs[kAhead + 1][2];
  using ScaleWord = decltype(gs[0][0].s);
  using ZeroWord = decltype(gs[0][0].z);
  uint16_t raw_s[2][PG];   // where they are not one word (K % 128 != 0, other addresses): as they come, put together a chunk later
  uint8_t raw_z[2][PG];
  const auto load = [&](Groups<PG>* dst) {
    if (g_left > 0) {
      if (g_i == 0) {
        const int64_t n0 = (int64_t)min(g_tile * 16 + g, a.N - 1) * groups, n1 = (int64_t)min(g_tile * 16 + 8 + g, a.N - 1) * groups;
        s0p = reinterpret_cast<const uint16_t*>(a.scale) + n0; s1p = reinterpret_cast<const uint16_t*>(a.scale) + n1;
        z0p = a.zero + n0; z1p = a.zero + n1;
      }
      if constexpr (VEC) {
        dst[0].z = dst[1].z = (ZeroWord)0x08080808u;
        dst[0].s = *reinterpret_cast<const ScaleWord*>(s0p + g_at);
        dst[1].s = *reinterpret_cast<const ScaleWord*>(s1p + g_at);
        if (a.zero) {
          dst[0].z = *reinterpret_cast<const ZeroWord*>(z0p + g_at);
          dst[1].z = *reinterpret_cast<const ZeroWord*>(z1p + g_at);
        }
      } else {
#pragma unroll
        for (int j = 0; j < PG; ++j) {   // past K: any group of the row, the tokens are 0 there
          const int at = min(g_at + j, groups - 1);
          raw_s[0][j] = s0p[at];
          raw_s[1][j] = s1p[at];
          raw_z[0][j] = raw_z[1][j] = 8;
          if (a.zero) raw_z[0][j] = z0p[at], raw_z[1][j] = z1p[at];
        }
      }
      --g_left;
      g_at += f.wk * PG;
      if (++g_i == mine) g_i = 0, g_at = (kb + kw * kChunk) / G, g_tile += stride;
    }
  };
  const auto put = [&](Groups<PG>* dst) {
    if constexpr (!VEC) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint64_t sv = 0;
        uint32_t zv = 0;
#pragma unroll
        for (int j = 0; j < PG; ++j) sv |= (uint64_t)raw_s[h][j] << (16 * j), zv |= (uint32_t)raw_z[h][j] << (8 * j);
        dst[h].s = (ScaleWord)sv;
        dst[h].z = (ZeroWord)zv;
      }
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    load(gs[i]);
    if (i + 1 < kAhead) put(gs[i]);
  }
  // Tokens: eight values a thread, put into the nibbles' order (k and k + 4 are a pair); 0 past K.
  const int work = a.M * (f.split_k / 8);
  for (int i0 = 0; i0 < work; i0 += 4 * 32 * kW4Warps) {
    uint4 vs[4];
    int ms[4], ps[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * 32 * kW4Warps + threadIdx.x;
      ms[u] = (int)f.pieces.div(i);
      ps[u] = i - ms[u] * (int)f.pieces.d;
      vs[u] = make_uint4(0, 0, 0, 0);
      if (i < work && kb + 8 * ps[u] < ke) vs[u] = *reinterpret_cast<const uint4*>(a.x + (int64_t)ms[u] * a.K + kb + 8 * ps[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i0 + u * 32 * kW4Warps + (int)threadIdx.x >= work) break;
      const int m = ms[u], p = ps[u], j = p / (4 * GS), tt = p / GS & 3, v = p & (GS - 1);   // group, lane and step of the group
      *reinterpret_cast<uint4*>(xp + (((j * GS + v) * a.M + m) * 4 + tt) * 16) =
          make_uint4(__byte_perm(vs[u].x, vs[u].z, 0x5410), __byte_perm(vs[u].x, vs[u].z, 0x7632), __byte_perm(vs[u].y, vs[u].w, 0x5410),
                     __byte_perm(vs[u].y, vs[u].w, 0x7632));
    }
  }
  __syncthreads();
  if (f.split > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");

  int slot = 0, buf = 0, i = 0;
  float acc[4] = {};
  uint32_t x_step = g < a.M ? a.M * 64 : 0, x_at = g < a.M ? xs + lane * 16 + kw * 4 * x_step : ptx::su32(smem);   // a lane without a token reads zeros
  // One chunk, with its scales, and those to be loaded. The loop below is unrolled over gs: moving a word that is on its way
  // waits for it.
  const auto chunk = [&](const Groups<PG>* now, Groups<PG>* before, Groups<PG>* later) {
    put(before);
    load(later);
    asm volatile("cp.async.wait_group %0;" ::"n"(kFewSlots - 2) : "memory");
    __syncwarp();   // all lanes' copies are there, and what the next copy overwrites has been read
    copy(slot == 0 ? kFewSlots - 1 : slot - 1);
    const uint32_t ws = ring + slot * SLOT + g * PITCH + 4 * GS * t;
    slot = slot + 1 == kFewSlots ? 0 : slot + 1;
#pragma unroll
    for (int j = 0; j < PG; ++j) {
      uint32_t w[2][GS];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t at = ws + 8 * h * PITCH + 16 * GS * j;
        if constexpr (GS == 4) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[h][0]), "=r"(w[h][1]), "=r"(w[h][2]), "=r"(w[h][3]) : "r"(at) : "memory");
        else if constexpr (GS == 2) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[h][0]), "=r"(w[h][1]) : "r"(at) : "memory");
        else w[h][0] = lds4(at);
      }
      float sum[4];
      const uint32_t z0 = 0x43004300u | ((uint32_t)now[0].z >> (8 * j) & 15u) * 0x10001u, z1 = 0x43004300u | ((uint32_t)now[1].z >> (8 * j) & 15u) * 0x10001u;
#pragma unroll
      for (int v = 0; v < GS; ++v) {
        uint32_t a0[2][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          a0[u >> 1][2 * (u & 1)] = sub2(nibbles(w[0][v] >> (4 * u)), z0);
          a0[u >> 1][2 * (u & 1) + 1] = sub2(nibbles(w[1][v] >> (4 * u)), z1);
        }
        uint4 b;
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(x_at + (j * GS + v) * x_step) : "memory");
        if (v == 0) mma_bf16_first(sum, a0[0], b.x, b.y);
        else mma_bf16_16816(sum, a0[0], b.x, b.y);
        mma_bf16_16816(sum, a0[1], b.z, b.w);
      }
      const float s0 = __uint_as_float((uint32_t)(now[0].s >> (16 * j)) << 16), s1 = __uint_as_float((uint32_t)(now[1].s >> (16 * j)) << 16);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] = fmaf(sum[c], c < 2 ? s0 : s1, acc[c]);
    }
    x_at += 4 * f.wk * x_step;
  };
  const auto end_tile = [&]() {
    if (f.wk == 1) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = tile * 16 + 8 * h + g;
        const float bias = a.bias && row < a.N ? a.bias[row] : 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int m = 2 * t + e;
          if (m < a.M && row < a.N) a.out[(int64_t)m * a.N + row] = acc[2 * h + e] + bias;
        }
      }
    } else {
      float* mine_red = red + (buf * kW4Warps + warp) * a.M * 16;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = 2 * t + (e & 1);
        if (m < a.M) mine_red[m * 16 + 8 * (e >> 1) + g] = acc[e];
      }
      __syncthreads();   // the buffer before this one is read by nobody any more
      for (int j = threadIdx.x; j < a.M * 16 * f.per_cta; j += 32 * kW4Warps) {
        const int c = f.per_cta > 1 ? j / (a.M * 16) : 0, r = j - c * (a.M * 16), n = (tile - of_cta + c) * 16 + (r & 15), m = r >> 4;
        float v = 0.f;
        for (int w = 0; w < f.wk; ++w) v += red[(buf * kW4Warps + c * f.wk + w) * a.M * 16 + r];
        if (f.split > 1) {   // to the cluster's first CTA
          uint32_t dst;
          asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(dst) : "r"(ptx::su32(recv + (buf * 8 + part) * a.M * 16 + r)));
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst), "f"(v) : "memory");
        } else if (n < a.N) {
          a.out[(int64_t)m * a.N + n] = v + (a.bias ? a.bias[n] : 0.f);
        }
      }
      if (f.split > 1) {   // everybody's sums are there after the barrier; the next tile's go to the other buffer
        asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (part == 0)
          for (int j = threadIdx.x; j < a.M * 16; j += 32 * kW4Warps) {
            const int n = tile * 16 + (j & 15), m = j >> 4;
            float v = 0.f;
            for (int c = 0; c < f.split; ++c) v += recv[(buf * 8 + c) * a.M * 16 + j];
            if (n < a.N) a.out[(int64_t)m * a.N + n] = v + (a.bias ? a.bias[n] : 0.f);
          }
      }
      buf ^= 1;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = 0.f;
    x_at -= 4 * f.wk * mine * x_step;
    tile += stride;
    i = 0;
    --rounds;
  };
  int left = own * mine;
  while (left > 0) {
#pragma unroll
    for (int u = 0; u <= kAhead; ++u)
      if (left > 0) {
        chunk(gs[u], gs[(u + kAhead - 1) % (kAhead + 1)], gs[(u + kAhead) % (kAhead + 1)]);
        --left;
        if (++i == mine) end_tile();
      }
  }
  if (f.wk > 1) {
    x_step = 0;
    while (rounds > 0) end_tile();   // a warp without a tile in the last round, or without chunks, still meets the others
  }
}

template <int NT, int G>
cudaError_t launch_many(const W4Args& a, cudaStream_t s);

template <int G, bool VEC>
cudaError_t launch_few(const W4Args& a, cudaStream_t s) {
  static OncePerDevice once;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = (cudaError_t)once.run(dev, [&] { return (int)cudaFuncSetAttribute(w4_few_kernel<G, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024); });
  if (e != cudaSuccess) return e;
  FewArgs f{a, 1, 0, 0, 0, FastDiv(1)};
  const int tiles = (a.N + 15) / 16, chunks = (a.K + kChunk - 1) / kChunk;
  while (f.split < 8 && (tiles * f.split * 2 <= 2 * kSms || (int64_t)a.M * 2 * ((chunks + f.split - 1) / f.split) * kChunk > kFewX) && chunks >= 2 * kW4Warps * f.split) f.split *= 2;
  f.split_k = (chunks + f.split - 1) / f.split * kChunk;
  f.pieces = FastDiv((uint32_t)(f.split_k / 8));
  const size_t smem = few_smem<G>(a.M, f.split_k);
  const int ctas = (smem <= 113 * 1024 ? 2 : 1) * kSms;
  // warps of a tile: the least of rounds times (chunks of a warp, and as much as a chunk for the adding)
  f.wk = kW4Warps;
  if (f.split == 1) {
    int64_t best = INT64_MAX;
    for (int wk = 1; wk <= kW4Warps; wk *= 2) {
      const int64_t rounds = ((int64_t)tiles * wk + (int64_t)ctas * kW4Warps - 1) / ((int64_t)ctas * kW4Warps);
      const int64_t cost = rounds * ((chunks + wk - 1) / wk + (wk > 1));
      if (cost < best) best = cost, f.wk = wk;
    }
  }
  // Three tokens and more go faster by tiles of 32 rows where a tile's chunks are shared out, unless they are few (8 tokens of
  // 4096 x 4096 in groups of 128 7.3 us against 8.9, 4 of 14336 x 4096 15.3 against 23.6; but 3.3 against 2.7 for 4 of 768 x 2304, and
  // 15.0 against 14.4 for 2048 x 32768 in groups of 64, where every warp has tiles of its own). Where the tokens of a CTA do not fit,
  // all do.
  if ((a.M > 2 && f.wk > 1 && chunks > 8) || smem > 227 * 1024) return launch_many<1, G>(a, s);
  const int64_t clusters = ctas / f.split, rounds = ((int64_t)tiles * f.wk + clusters * kW4Warps - 1) / (clusters * kW4Warps);
  f.per_cta = (int)((tiles + clusters * rounds - 1) / (clusters * rounds));   // even rounds
  const int64_t n = (tiles + f.per_cta - 1) / f.per_cta;
  return launch_cluster(w4_few_kernel<G, VEC>, dim3((unsigned)((n < clusters ? n : clusters) * f.split)), dim3(32 * kW4Warps), smem, f.split, s, f);
}

// ---- up to 64 tokens: mma.sync ------------------------------------------------------------------------------------------
//
// Here mma.sync (8 cycles of an SM's quarter for 256 weights by 8 tokens) takes as long as the weights or longer, so the
// weights become exact bf16 (0x4300 | q is 128 + q; less 128 + zero), which needs nothing of the tokens but their order. A warp
// has 32 rows, whose tokens it reads once from shared memory; the four warps of a quarter of the CTA's rows share out K,
// chunk by chunk, and those of the same chunks share the tokens' copies. k, k + 4 make a pair of each word and of the tokens.
// What bounds it is issuing: with 40 tokens some 830 instructions a warp and chunk, 80 of them MMAs, at 0.45 a cycle. 16, 24 and 32
// tokens: 4096 x 14337 in groups of 64 16.6, 18.5 and 21.9 us (30 MB: 1.8, 1.6 and 1.4 TB/s), 2048 x 32768 17, 23 and 32 us.
constexpr int kManyPitch = 80;   // bytes between weight rows: no bank conflicts for words of eight rows
template <int NT>
constexpr int many_groups() { return NT <= 2 ? 4 : NT <= 5 ? 3 : 2; }   // most 32-row groups of a CTA: registers
template <int NT>
__host__ __device__ constexpr size_t many_smem(int wn, int stages) {
  // tokens [stage][quarter of K][token][256 bytes], weights [stage][warp][32 rows], scales and zeros [2][warp][4 groups][32 rows]
  return stages * ((size_t)4 * 8 * NT * 256 + (size_t)4 * wn * 32 * kManyPitch) + (size_t)2 * 4 * wn * 4 * 32 * 4;
}

template <int NT, int G>   // 8 NT tokens, group
__global__ void __launch_bounds__(128 * many_groups<NT>(), 1) w4_many_kernel(const W4Args a, int wn, int split, int stages) {
  constexpr int PG = kChunk / G, GS = G / 32, XQ = 8 * NT * 256;
  extern __shared__ __align__(16) unsigned char smem[];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, rg = warp >> 2, kq = (warp + rg) & 3;
  const int part = split > 1 ? blockIdx.x % split : 0, cta = split > 1 ? blockIdx.x / split : blockIdx.x;
  const int n0 = (cta * wn + rg) * 32, groups = a.K / G, chunks = (a.K + kChunk - 1) / kChunk;
  const int c0 = part * 4 + kq, next = 4 * split;   // this warp's first chunk, and how far it is to its next
  const int iters = chunks > c0 ? (chunks - c0 + next - 1) / next : 0;   // the same for the warps that share tokens
  const uint32_t base = ptx::su32(smem), wbase = base + stages * 4 * XQ;
  const int wstage = 4 * wn * 32 * kManyPitch;
  uint32_t* sg = reinterpret_cast<uint32_t*>(smem + stages * (4 * XQ + wstage)) + warp * 4 * 32;   // + buffer * 4 wn * 128

  // 16-byte pieces: tokens by the threads of this quarter of K, a token's pieces with bit 2 flipped for odd tokens (no bank
  // conflicts for two tokens' 64 bytes); weights by the warp; 0 past the last token, row and k.
  const int tid = rg * 32 + lane;
  const uint8_t* wrow[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) wrow[r] = a.q + ((int64_t)min(n0 + 8 * r + g, a.N - 1) * a.K >> 1);
  const auto copy = [&](int i, int st) {
    if (i < iters) {
      const int k0 = (c0 + next * i) * kChunk, k = k0 + 8 * (tid & 15);
      // 2 wn tokens at a time: an even number, so a thread's are all even or all odd
      uint32_t xd = base + (st * 4 + kq) * XQ + (tid >> 4) * 256 + (((tid & 15) ^ (tid >> 4 & 1) * 4) << 4);
      const __nv_bfloat16* src = a.x + (int64_t)(tid >> 4) * a.K + k;
      const int last = k < a.K ? a.M : 0;
      for (int m = tid >> 4; m < 8 * NT; m += 2 * wn) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(xd), "l"(m < last ? src : a.x), "r"(m < last ? 16 : 0) : "memory");
        xd += 2 * wn * 256;
        src += (int64_t)2 * wn * a.K;
      }
      const int at = k0 + 32 * t < a.K ? (k0 + 32 * t) >> 1 : 0;   // past K anything: the tokens are 0
#pragma unroll
      for (int r = 0; r < 4; ++r)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(wbase + st * wstage + (warp * 32 + 8 * r + g) * kManyPitch + 16 * t), "l"(wrow[r] + at) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // Scales and zeros of the warp's rows, PG neighbours of a row by as many lanes, held while a chunk is computed and then put to
  // where all lanes find them
  uint16_t raw_s[PG];
  uint8_t raw_z[PG];
  const auto load = [&](int i) {   // N K / G < 2^31
    if (i >= iters) return;
    const int gr = min((c0 + next * i) * PG + lane % PG, groups - 1);
#pragma unroll
    for (int j = 0; j < PG; ++j) {
      const int e = min(n0 + j * (32 / PG) + lane / PG, a.N - 1) * groups + gr;
      raw_s[j] = reinterpret_cast<const uint16_t*>(a.scale)[e];
      raw_z[j] = a.zero ? a.zero[e] : (uint8_t)8;
    }
  };
  const auto put = [&](int i) {
    if (i >= iters) return;
#pragma unroll
    for (int j = 0; j < PG; ++j) sg[(i & 1) * 4 * wn * 128 + (lane % PG) * 32 + j * (32 / PG) + lane / PG] = (uint32_t)raw_s[j] << 16 | (raw_z[j] & 15u);
  };
  for (int i = 0; i < stages - 1; ++i) copy(i, i);
  load(0);
  put(0);
  load(1);
  float acc[2][NT][4] = {};
  for (int i = 0, st = 0; i < iters; ++i) {
    if (stages == 4) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (stages == 3) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
    ptx::named_sync(1 + kq, 32 * wn);   // the tokens that others copied are there, and the chunk before has been read by all
    copy(i + stages - 1, st ? st - 1 : stages - 1);
    // token 8 n + g, piece 4 s + t, with bit 2 flipped for odd tokens
    const uint32_t xg = base + (st * 4 + kq) * XQ + g * 256 + t * 16, odd = g & 1, ws = wbase + st * wstage + (warp * 32 + g) * kManyPitch + 4 * t;
    const uint32_t* sgi = sg + (i & 1) * 4 * wn * 128;
#pragma unroll
    for (int j = 0; j < PG; ++j) {
      float sum[2][NT][4];
      uint32_t sz[2][2], z[2][2];
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          sz[r][h] = sgi[j * 32 + 16 * r + 8 * h + g];
          z[r][h] = 0x43004300u | (sz[r][h] & 15u) * 0x10001u;
        }
#pragma unroll
      for (int v = 0; v < GS; ++v) {
        const int s = j * GS + v;
        uint32_t xb[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          uint32_t x[4];
          asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                       : "r"(xg + n * 2048 + (s ^ odd) * 64) : "memory");
          xb[n][0] = __byte_perm(x[0], x[2], 0x5410);
          xb[n][1] = __byte_perm(x[0], x[2], 0x7632);
          xb[n][2] = __byte_perm(x[1], x[3], 0x5410);
          xb[n][3] = __byte_perm(x[1], x[3], 0x7632);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t w0 = lds4(ws + (16 * r) * kManyPitch + 16 * s), w1 = lds4(ws + (16 * r + 8) * kManyPitch + 16 * s);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            uint32_t f[4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              f[2 * u] = sub2(nibbles(w0 >> (4 * (2 * y + u))), z[r][0]);
              f[2 * u + 1] = sub2(nibbles(w1 >> (4 * (2 * y + u))), z[r][1]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              if (v == 0 && y == 0) mma_bf16_first(sum[r][n], f, xb[n][0], xb[n][1]);
              else mma_bf16_16816(sum[r][n], f, xb[n][2 * y], xb[n][2 * y + 1]);
            }
          }
        }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float s0 = __uint_as_float(sz[r][0] & 0xffff0000u), s1 = __uint_as_float(sz[r][1] & 0xffff0000u);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          acc[r][n][0] += sum[r][n][0] * s0;
          acc[r][n][1] += sum[r][n][1] * s0;
          acc[r][n][2] += sum[r][n][2] * s1;
          acc[r][n][3] += sum[r][n][3] * s1;
        }
      }
    }
    put(i + 1);
    load(i + 2);
    if (++st == stages) st = 0;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  // the sums of the quarters of K: [quarter][row of the CTA][token], rows 8 NT + 2 floats apart
  float* sums = reinterpret_cast<float*>(smem);
  constexpr int SP = 8 * NT + 2;
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<float2*>(sums + (size_t)(kq * wn * 32 + rg * 32 + 16 * r + 8 * h + g) * SP + 8 * n + 2 * t) = make_float2(acc[r][n][2 * h], acc[r][n][2 * h + 1]);
  __syncthreads();
  const int rows = wn * 32;
  if (split > 1) {   // each CTA's sums go to the cluster's first: [part][token][row], behind its own
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");   // its copies are done
    float* recv = sums + (size_t)4 * rows * SP;
    for (int m = warp; m < a.M; m += 4 * wn)
      for (int r = lane; r < rows; r += 32) {
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) v += sums[(size_t)(q * rows + r) * SP + m];
        uint32_t dst;
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(dst) : "r"(ptx::su32(recv + (part * a.M + m) * rows + r)));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst), "f"(v) : "memory");
      }
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (part) return;
    for (int m = warp; m < a.M; m += 4 * wn)
      for (int r = lane; r < rows; r += 32) {
        const int n = cta * rows + r;
        if (n >= a.N) continue;
        float v = 0.f;
        for (int c = 0; c < split; ++c) v += recv[(c * a.M + m) * rows + r];
        a.out[(int64_t)m * a.N + n] = v + (a.bias ? a.bias[n] : 0.f);
      }
    return;
  }
  for (int m = warp; m < a.M; m += 4 * wn)
    for (int r = lane; r < rows; r += 32) {
      const int n = cta * rows + r;
      if (n >= a.N) continue;
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) v += sums[(size_t)(q * rows + r) * SP + m];
      a.out[(int64_t)m * a.N + n] = v + (a.bias ? a.bias[n] : 0.f);
    }
}

template <int NT, int G>
cudaError_t launch_many(const W4Args& a, cudaStream_t s) {
  static OncePerDevice once;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = (cudaError_t)once.run(dev, [&] { return (int)cudaFuncSetAttribute(w4_many_kernel<NT, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024); });
  if (e != cudaSuccess) return e;
  // The rows a CTA that leave the fullest SM the fewest, the more the better; with SMs left over, a cluster shares K as far as
  // every warp keeps a chunk, and up to 16 tokens, four chunks, two CTAs an SM (5 tokens of 8192 x 2048 in groups of 32 7.1 us
  // against 8.7, of 2048 x 2560 4.7 against 4.1; 24 of 4096 x 4096 12.9 against 10.0).
  int wn = 1, split = 1;
  const int64_t sets = ((int64_t)a.N + 31) / 32;
  int64_t best = INT64_MAX;
  for (int w = many_groups<NT>(); w >= 1; --w) {
    const int64_t rows = ((sets + w - 1) / w + kSms - 1) / kSms * w;   // of the fullest SM
    if (rows < best) best = rows, wn = w;
  }
  const int64_t ctas = ((int64_t)a.N + 32 * wn - 1) / (32 * wn);
  const int chunks = (a.K + kChunk - 1) / kChunk;
  const auto more = [&] {
    const int64_t n = ctas * split * 2;
    return (n <= kSms && chunks > 4 * split) || (NT <= 2 && n <= 2 * kSms && chunks >= 32 * split);
  };
  while (wn == 1 && split < 8 && more()) split *= 2;
  // A CTA that is alone on its SM, or one of two in clusters, copies up to three chunks ahead; else the next CTA's work hides the
  // copies, and smaller ones let more of them in (24 tokens: 14336 x 4096 24 us against 29, but 2048 x 32768 39 against 23; 5 tokens of
  // 8192 x 2048 8.2 us both from a graph, and 8.8 against 10.2 without one, where the next call's CTAs would come in earlier).
  // Clusters of 8 need two CTAs an SM, or four, to find their places.
  const int64_t n = ctas * split;
  int stages = n <= kSms || (split > 1 && split < 8 && n <= 2 * kSms) ? 4 : 2;
  while (stages > 2 && many_smem<NT>(wn, stages) > (n <= kSms && split < 8 ? 227 : 112) * 1024) --stages;
  return launch_cluster(w4_many_kernel<NT, G>, dim3((unsigned)(ctas * split)), dim3(128 * wn), many_smem<NT>(wn, stages), split, s, a, wn, split, stages);
}

// ---- up to 64 tokens: tcgen05 ------------------------------------------------------------------------------------------
//
// A CTA of four warps has 128 rows and a share of K. A thread takes a row's nibbles apart, 128 k (64) at a time, as exact bf16
// (0x4300 | q is 128 + q; less 128 + zero) and puts them into tensor memory as the MMA's first operand; the tokens, in the
// nibbles' order (k, k + 4 are neighbours), are the second, in shared memory. A group's products are summed by themselves
// and read back: a thread has a row of them, and multiplies them by the group's scale. While the MMAs of one step run, the
// nibbles of the next are taken apart.
//
// A step is a chain (weights, nibbles, tensor memory, the sums before, a barrier, MMAs) of a microsecond, in which a CTA's four
// warps issue about 450 instructions each; what hides it is three CTAs an SM. MMAs are a fifth of it. With 40 and 64 tokens,
// 2048 x 32768 takes 25 and 27 us (the kernel above: 38 and 52), 14336 x 4096 25 and 31 (33 and 42), in groups of 32 4096 x 32768
// 55 and 58 (78 and 97); 4096 x 14336, which is an even share for the kernel above, 25 and 31 (22 and 44).
constexpr int kTcPitch = 80, kTcW = 3;   // bytes between weight rows: no bank conflicts for eight rows' 16 bytes; chunks in the ring
constexpr int kTcBlock = 8, kTcSg = 9;   // groups whose scales are loaded together; words between rows of them
template <int NB, int G>
struct TcShape {
  static constexpr int KS = G == 128 ? 128 : 64;                // k of a step
  static constexpr int GS = KS > G ? KS / G : 1;                // groups that end with a step
  static constexpr int COLS = KS / 2 + GS * NB <= 128 ? 128 : 256;   // tensor memory: a step's weights, the sums
  static constexpr int CTAS = COLS > 128 ? 2 : 3;                // of an SM
  static constexpr int R = NB >= 48 && KS == 128 ? 2 : 3;                    // steps of tokens in the ring
  static constexpr int XB = NB * 128, X = KS / 64 * XB;         // bytes of 64 k of the tokens, of a step's
  static constexpr int W0 = R * X, SG0 = W0 + kTcW * 128 * kTcPitch, BAR0 = SG0 + 2 * 128 * kTcSg * 4;
  static constexpr int SMEM = BAR0 + 16 + 1024;                 // and the alignment of the tokens
};

// MMAs that have been issued: a microsecond; false after a quarter of a second or so.
__device__ __forceinline__ bool wait_mma(uint64_t* bar, uint32_t parity) {
  for (uint32_t i = 0; i < (1u << 20); ++i)
    if (ptx::mbar_test(bar, parity)) return true;
  return false;
}

template <int NB, int G>   // tokens that the MMA has, group
__global__ void __launch_bounds__(128, TcShape<NB, G>::CTAS) w4_tc_kernel(const W4Args a, int split) {
  using S = TcShape<NB, G>;
  constexpr int KS = S::KS, GS = S::GS, R = S::R, NX = NB / 16, HB = KS / 64;   // 16-byte pieces of a thread of 64 k of the tokens
  constexpr int SB = kTcBlock * G / KS;                                       // steps of a block of scales
  extern __shared__ __align__(16) unsigned char smem_raw[];
  const uint32_t base = (ptx::su32(smem_raw) + 1023u) & ~1023u;
  unsigned char* smem = smem_raw + (base - ptx::su32(smem_raw));
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + S::BAR0);
  uint32_t* slot = reinterpret_cast<uint32_t*>(smem + S::BAR0 + 8);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ptx::su32(slot)), "r"(S::COLS));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (tid == 32) {
    ptx::mbar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const int part = split > 1 ? blockIdx.x % split : 0, cta = split > 1 ? blockIdx.x / split : blockIdx.x;
  const int n0 = cta * 128, groups = a.K / G, all = (a.K + kChunk - 1) / kChunk, per = (all + split - 1) / split;
  const int c0 = part * per, chunks = max(0, min(all - c0, per)), steps = chunks * (kChunk / KS);

  // weights: a lane has 16 of the 64 bytes of 8 rows apart; past K anything, the tokens are 0 there
  const int wr = lane >> 2, wt = lane & 3;
  const uint32_t wring = base + S::W0 + warp * 32 * kTcPitch;
  const uint8_t* wrow[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) wrow[r] = a.q + ((int64_t)min(n0 + warp * 32 + 8 * r + wr, a.N - 1) * a.K >> 1);
  int wk = c0 * kChunk + 32 * wt, wslot = 0, wleft = chunks;
  const auto copy_w = [&] {
    if (wleft > 0) {
      const int at = wk < a.K ? wk >> 1 : 0;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(wring + wslot * 128 * kTcPitch + (8 * r + wr) * kTcPitch + 16 * wt), "l"(wrow[r] + at) : "memory");
      wk += kChunk;
      --wleft;
      if (++wslot == kTcW) wslot = 0;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // tokens: 16-byte pieces, eight of a token's 64 k; past the last token and K zeros. A thread puts its own into the nibbles' order
  const int xm = tid >> 3, xp = tid & 7;
  const uint32_t xto = base + xm * 128 + (((tid ^ xm) & 7) << 4);   // 16 tokens further: 2048 bytes
  const __nv_bfloat16* xsrc = a.x + (int64_t)min(xm, a.M - 1) * a.K + c0 * kChunk + 8 * xp;
  int xk = c0 * kChunk + 8 * xp, xslot = 0, xleft = steps;
  const auto copy_x = [&] {
    if (xleft > 0) {
#pragma unroll
      for (int h = 0; h < HB; ++h)
#pragma unroll
        for (int i = 0; i < NX; ++i) {
          const bool in = xm + 16 * i < a.M && xk + 64 * h < a.K;
          const __nv_bfloat16* src = in ? xsrc + (int64_t)16 * i * a.K + 64 * h : a.x;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(xto + xslot * S::X + h * S::XB + i * 2048), "l"(src), "r"(in ? 16 : 0) : "memory");
        }
      xsrc += KS;
      xk += KS;
      --xleft;
      if (++xslot == R) xslot = 0;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const auto order_x = [&](int at) {
#pragma unroll
    for (int j = 0; j < HB * NX; ++j) {
      const uint32_t p = xto + at * S::X + j / NX * S::XB + j % NX * 2048;
      uint32_t x[4];
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(p) : "memory");
      asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(p), "r"(__byte_perm(x[0], x[2], 0x5410)), "r"(__byte_perm(x[0], x[2], 0x7632)),
                   "r"(__byte_perm(x[1], x[3], 0x5410)), "r"(__byte_perm(x[1], x[3], 0x7632)) : "memory");
    }
  };
  // scales and zeros: blocks of eight groups, whose 128 rows the threads load so that eight lanes have neighbours
  uint16_t raw_s[8];
  uint8_t raw_z[8];
  const auto load_sg = [&](int b) {   // block b of this CTA; N K / G < 2^31
    const int gr = min(c0 * (kChunk / G) + b * kTcBlock + xp, groups - 1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = min(n0 + 16 * i + xm, a.N - 1) * groups + gr;
      raw_s[i] = reinterpret_cast<const uint16_t*>(a.scale)[e];
      raw_z[i] = a.zero ? a.zero[e] : (uint8_t)8;
    }
  };
  const auto put_sg = [&](int b) {
    uint32_t* to = reinterpret_cast<uint32_t*>(smem + S::SG0) + (b & 1) * 128 * kTcSg + xp;
    const bool in = c0 * (kChunk / G) + b * kTcBlock + xp < groups;   // past K: 0
#pragma unroll
    for (int i = 0; i < 8; ++i) to[(16 * i + xm) * kTcSg] = in ? (uint32_t)raw_s[i] << 16 | (raw_z[i] & 15u) : 0u;
  };
  // In the ring's order: the tokens of a step, then weights; two steps ahead, tokens one where the ring has two.
  if (R == 3) copy_x();
  copy_w();
  copy_x();
  copy_w();
  load_sg(0);
  put_sg(0);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  pdl_trigger();   // not before this CTA's tensor memory is its own: the next kernel may take what is left before it waits
  const uint32_t tmem = *slot, mine = tmem + ((uint32_t)warp << 21);   // this warp's lanes
  const uint64_t xd = ptx::sw128_desc(base);

  float acc[NB], scale[GS];
  bool ok = true;
#pragma unroll
  for (int i = 0; i < NB; ++i) acc[i] = 0.f;
#pragma unroll
  for (int j = 0; j < GS; ++j) scale[j] = 0.f;
  const auto wait = [&](int s) {   // for the MMAs of step s
    ok = ok && wait_mma(bar, s & 1);
    ptx::tc_fence_after();
    __syncwarp();
  };
  const auto read = [&] {   // the sums of the groups that ended, times their scales
#pragma unroll
    for (int j = 0; j < GS; ++j) {
      const uint32_t d = mine + KS / 2 + j * NB;
      float v[NB];
#pragma unroll
      for (int i = 0; i + 32 <= NB; i += 32) ptx::tmem_ld32_nowait(d + i, reinterpret_cast<uint32_t*>(v) + i);
      if constexpr (NB % 32 != 0) ptx::tmem_ld16(d + NB - 16, v + NB - 16);
      else ptx::tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[i] += v[i] * scale[j];
    }
  };
  int st = 0, xs = 0, b = 0, in_block = 0;   // the weights' and the tokens' slots, the block of scales and the step of it
  for (int s = 0; s < steps; ++s) {
    const int h = KS == 64 ? s & 1 : 0;   // half of the chunk
    if (in_block == 0) load_sg(b + 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(2) : "memory");
    __syncwarp();   // the other lanes' weights
    uint32_t f[KS / 2], sz[GS];
    const uint32_t at = wring + st * 128 * kTcPitch + lane * kTcPitch + 32 * h;
    const uint32_t* sg = reinterpret_cast<const uint32_t*>(smem + S::SG0) + (b & 1) * 128 * kTcSg + tid * kTcSg + in_block * KS / G;
#pragma unroll
    for (int j = 0; j < GS; ++j) sz[j] = sg[j];
#pragma unroll
    for (int i = 0; i < KS / 32; ++i) {
      uint32_t w[4];
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at + 16 * i) : "memory");
      const uint32_t z = 0x43004300u | (sz[i * 32 / G] & 15u) * 0x10001u;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) f[16 * i + 4 * j + u] = sub2(nibbles(w[j] >> (4 * u)), z);
    }
    if (R == 2) asm volatile("cp.async.wait_group %0;" ::"n"(1) : "memory");
    order_x(xs);
    ptx::fence_async_smem();
    if (in_block == SB - 1) put_sg(b + 1);
    if (s > 0) wait(s - 1);
#pragma unroll
    for (int i = 0; i < KS / 32; ++i) ptx::tmem_st16_nowait(mine + 16 * i, f + 16 * i);
    if (s > 0) read();
#pragma unroll
    for (int j = 0; j < GS; ++j) scale[j] = __uint_as_float(sz[j] & 0xffff0000u);
    ptx::tmem_wait_st();
    ptx::tc_fence_before();
    __syncthreads();
    if (tid == 0) {
      ptx::tc_fence_after();
#pragma unroll
      for (int i = 0; i < KS / 16; ++i)
        ptx::mma_bf16_ts(tmem + KS / 2 + (G < KS ? i * 16 / G * NB : 0), tmem + 8 * i,
                         xd + (uint64_t)(xs * (S::X >> 4) + i / 4 * (S::XB >> 4) + i % 4 * 2), ptx::idesc_m128(NB), i * 16 % G != 0);
      ptx::mma_commit(bar);
    }
    __syncwarp();
    copy_x();
    if (KS == 128 || h == 1) {
      copy_w();
      if (++st == kTcW) st = 0;
    }
    if (++xs == R) xs = 0;
    if (++in_block == SB) in_block = 0, ++b;
  }
  if (steps > 0) {
    wait(steps - 1);
    read();
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::COLS));
  const int n = n0 + tid;
  const float poison = ok ? 0.f : __int_as_float(0x7fc00000);   // MMAs that have not ended: nothing that looks like a result
  if (split == 1) {
    const float add = (a.bias && n < a.N ? a.bias[n] : 0.f) + poison;
    float* o = a.out + n;
#pragma unroll
    for (int m = 0; m < NB; ++m) {
      if (m < a.M && n < a.N) *o = acc[m] + add;
      o += a.N;
    }
    return;
  }
  // A cluster's shares of K: each CTA adds up as many tokens, in shared memory: [part][token][row]. Tensor memory was given back
  // before the first wait for another CTA, so that CTAs that wait for some never wait for each other.
  const int tokens = (a.M + split - 1) / split;
  float* recv = reinterpret_cast<float*>(smem);
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");   // nobody's smem is in use
  int to = -1, left = 0;
  uint32_t dst = 0;
#pragma unroll
  for (int m = 0; m < NB; ++m)
    if (m < a.M) {
      if (left == 0) {
        left = tokens;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(ptx::su32(recv + part * tokens * 128 + tid)), "r"(++to));
      }
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst), "f"(acc[m] + poison) : "memory");
      dst += 512;
      --left;
    }
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
  const float bias = a.bias && n < a.N ? a.bias[n] : 0.f;
  for (int i = 0, m = part * tokens; i < tokens && m < a.M; ++i, ++m) {
    float v = 0.f;
    for (int c = 0; c < split; ++c) v += recv[(c * tokens + i) * 128 + tid];
    if (n < a.N) a.out[(int64_t)m * a.N + n] = v + bias;
  }
}

template <int NB, int G>
cudaError_t launch_tc(const W4Args& a, cudaStream_t s) {
  using S = TcShape<NB, G>;
  static OncePerDevice once;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = (cudaError_t)once.run(dev, [] { return (int)cudaFuncSetAttribute(w4_tc_kernel<NB, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM); });
  if (e != cudaSuccess) return e;
  const int64_t tiles = ((int64_t)a.N + 127) / 128;
  const int chunks = (a.K + kChunk - 1) / kChunk;
  // A cluster shares K as far as four fifths of the CTAs that fit: with more, clusters of some sizes do not find their places at
  // once (113 tiles of 4096 k, 40 tokens: 27 us with 3, 33.5 with 4, 30.5 with 2)
  int split = 1;
  while (split < 8 && split < chunks && tiles * (split + 1) <= 120 * S::CTAS) ++split;
  return launch_cluster(w4_tc_kernel<NB, G>, dim3((unsigned)(tiles * split)), dim3(128), (size_t)S::SMEM, split, s, a, split);
}

template <int G>
cudaError_t launch_group(const W4Args& a, cudaStream_t s) {
  const int tokens = (a.M + 7) / 8;
  if constexpr (G > 32) if (tokens == 1) {   // groups of 32: 1 token of 3648 x 14402 18.1 us from the stream against 14.8, of 4096 x 4096 7.0 against 7.7
    constexpr int PG = kChunk / G;   // groups of a chunk
    if (PG == 1 || (a.K % kChunk == 0 && reinterpret_cast<uintptr_t>(a.scale) % (2 * PG) == 0 && reinterpret_cast<uintptr_t>(a.zero) % PG == 0))
      return launch_few<G, true>(a, s);
    if constexpr (PG > 1) return launch_few<G, false>(a, s);
  }
  // tcgen05 from 33 tokens and 2^24 weights on: 4096 x 4096 takes 12 and 15 us with 40 and 64 tokens against 13 and 17, 1024 x 4096
  // 8 and 12 against 6 and 8; with 24 tokens it takes as long as with 40.
  if (tokens > 4 && (int64_t)a.N * a.K >= 1 << 24) return tokens <= 6 ? launch_tc<48, G>(a, s) : launch_tc<64, G>(a, s);
  switch (tokens) {
    case 1: return launch_many<1, G>(a, s);
    case 2: return launch_many<2, G>(a, s);
    case 3: return launch_many<3, G>(a, s);
    case 4: return launch_many<4, G>(a, s);
    case 5: return launch_many<5, G>(a, s);
    case 6: return launch_many<6, G>(a, s);
    default: return launch_many<8, G>(a, s);
  }
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
  if ((group != 32 && group != 64 && group != 128) || K % group || K > 1 << 30 || (int64_t)N * K > (1ll << 35)) return UAD_EINVAL;
  if (reinterpret_cast<uintptr_t>(x) % 16 || reinterpret_cast<uintptr_t>(q) % 16 || reinterpret_cast<uintptr_t>(scale) % 2 ||
      reinterpret_cast<uintptr_t>(bias) % 4 || reinterpret_cast<uintptr_t>(out) % 4)
    return UAD_EINVAL;
  if (M > UAD_W4_MAX_ROWS) return UAD_ETOOBIG;
  if (!on_current_device(q)) return UAD_EINVAL;
  const W4Args a{static_cast<const __nv_bfloat16*>(x), q, reinterpret_cast<const __nv_bfloat16*>(scale), zero, bias, out, M, N, K, group};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = group == 32 ? launch_group<32>(a, s) : group == 64 ? launch_group<64>(a, s) : launch_group<128>(a, s);
  return launched(e);
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
