// Attention over a paged cache: the kernels of bf16 and fp32 caches and their launches. SINKS: a window leaves the first tokens visible.
#pragma once
#include "paged_attn.cuh"

namespace uad {
namespace {

// ---- bf16 -------------------------------------------------------------------------------------------------------
//
// mma.sync m16n8k16: a warp takes a slice of 16 or 32 keys at a time by itself, with no barrier in the loop, out of a ring of
// its own in shared memory that it fills with cp.async (rows 16 bytes further apart than they are long: ldmatrix reads eight of
// them without a conflict). S = Q K^T has 16 query rows as A and 8 keys as B; O^T = V^T P^T has V^T as A (16 dims by 16 keys,
// transposed by ldmatrix) and P^T as B, which is S's own register layout: 8 query rows are one tile there, so the few
// rows of a decoding step waste nothing where most of the work is. P goes in as two bf16 (the cut value and the
// rest): a second MMA where the pipe idles, for an error of 2^-16 and not 2^-9. The tensor cores' own form (tcgen05)
// would need 128 rows where there are 8 to 32.
// One new token: 64 x 4000 keys of 32 heads over 8 of 128 take 170 us (1050 MB, 6.2 TB/s, memory bound), of 8 over 1 of 256 48 us
// (5.5 TB/s), 2 sequences of up to 131071 of the former 116 us (5.8 TB/s). With more rows the latency of a slice bounds: 64 x 4000
// keys and four tokens of 8 over 1 of 256 75 us, where two blocks of 16 rows read them (96 MMAs a slice and block).

__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldm4(uint32_t* r, uint32_t s) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(s) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t* r, uint32_t s) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(s) : "memory");
}
__device__ __forceinline__ uint32_t lds2(uint32_t s) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(s) : "memory");
  return v;
}
// Two bf16: ones in the halves that are infinite or NaN.
__device__ __forceinline__ uint32_t nonfinite2(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// Keys of a slice, in sixteens: two where registers and shared memory bear it, for more independent work in a warp.
template <int DH, int NR>
constexpr int slice_steps() { return DH == 256 || NR == 4 ? 1 : 2; }
template <int DH, int NR>   // K and V slices in turn
constexpr int ring_slots() { return DH == 256 ? 3 : DH == 128 ? (NR == 4 ? 4 : 2) : NR == 4 ? 6 : 2; }
template <int DH>
constexpr int row_pitch() { return 2 * DH + 16; }
template <int DH, int NR>
constexpr int tc_ring() { return kWarps * ring_slots<DH, NR>() * slice_steps<DH, NR>() * 16 * row_pitch<DH>(); }
template <int DH, int NR>
constexpr size_t tc_smem(int heads) { return (size_t)tc_ring<DH, NR>() + receive_extra<DH, 8 * NR>(tc_ring<DH, NR>()) + sizeof(EndShared<8 * NR>) + heads * 8 * NR * row_pitch<DH>(); }
template <int DH, int NR>
constexpr int tc_ctas() { return NR == 4 || DH == 256 ? 2 : DH == 64 && NR == 1 ? 4 : 3; }

template <int DH, int NR, bool SINKS>   // head dim; 8 NR query rows
__global__ void __launch_bounds__(kThreads, tc_ctas<DH, NR>()) paged_attn_tc_kernel(const PagedAttnArgs a) {
  constexpr int KT = slice_steps<DH, NR>(), KEYS = 16 * KT, SLOTS = ring_slots<DH, NR>(), AHEAD = (SLOTS + 1) / 2;
  constexpr int MT = (NR + 1) / 2, PITCH = row_pitch<DH>(), SLOT = KEYS * PITCH, STEPS = DH / 16;
  constexpr int RING = tc_ring<DH, NR>(), EXTRA = receive_extra<DH, 8 * NR>(RING);
  using S = Sums<DH, 8 * NR>;
  static_assert(kWarps * S::kBytes <= RING, "the warps' sums fit the ring");
  static_assert(AHEAD * KEYS <= 64, "the bits of the keys ahead");
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t base = su32(smem);
  EndShared<8 * NR>* end = reinterpret_cast<EndShared<8 * NR>*>(smem + RING + EXTRA);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t sq = base + RING + EXTRA + sizeof(EndShared<8 * NR>) + (a.warp_heads ? warp * 8 * NR * PITCH : 0);   // queries [row][dim]
  pdl_wait();
  pdl_trigger();
  Piece c;
  Found first[AHEAD + 1], found;
  if (!find_piece<AHEAD + 1, SINKS>(a, 8 * NR, KEYS, &c, first) || no_keys(a, c)) return;
  for (int i = a.warp_heads ? lane : threadIdx.x; i < 8 * NR * (DH / 8); i += a.warp_heads ? 32 : kThreads) {
    const int r = i / (DH / 8), x = i % (DH / 8);
    const bool ok = r < c.rows;
    cp16_or_zero(sq + r * PITCH + x * 16, static_cast<const __nv_bfloat16*>(a.q) + (ok ? row_at(a, c, r, a.q_stride, DH) + 8 * x : 0), ok);
  }
  const uint32_t ring = base + warp * (SLOTS * SLOT);
  const int slices = (c.k1 - c.k0 + KEYS - 1) / KEYS, mine = (slices - c.kw + c.wk - 1) / c.wk;
  const auto slice_key = [&](int i) { return c.k0 + (i * c.wk + c.kw) * KEYS; };

  // Copies: eight lanes 128 bytes of a key, four keys at a time. Lane l (and, of 16 keys, l + 16) has looked up key l; at: where
  // this lane's keys are, for the keys and then the values.
  uint64_t seen = 0;   // KEYS bits a slice, the next one lowest
  int64_t at[KEYS / 4];
  int slot = 0;
  const uint32_t to = ring + (lane >> 3) * PITCH + (lane & 7) * 16;
  const auto copy = [&](int i, const void* pool) {
    if (i < mine) {
#pragma unroll
      for (int h = 0; h < KEYS / 4; ++h) {
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(pool) + (at[h] < 0 ? 0 : at[h]) + 8 * (lane & 7);
#pragma unroll
        for (int x = 0; x < DH / 64; ++x) cp16_or_zero(to + slot * SLOT + 4 * h * PITCH + x * 128, src + 64 * x, at[h] >= 0);
      }
    }
    cp_commit();
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
  };
  const auto copy_k = [&](int i, int ahead, const Found& fnd) {
    const int64_t e = i < mine ? key_at(a, c, fnd) : -1;
    seen |= (uint64_t)(__ballot_sync(0xffffffffu, e >= 0) & (0xffffffffu >> (32 - KEYS))) << (KEYS * ahead);
#pragma unroll
    for (int h = 0; h < KEYS / 4; ++h) at[h] = __shfl_sync(0xffffffffu, e, 4 * h + (lane >> 3));
    copy(i, a.p.k);
  };
  const auto next_k = [&](int i) {
    copy_k(i, AHEAD - 1, found);
    if (i + 1 < mine) found = find_key<SINKS>(a, blockIdx.z, c.shift, slice_key(i + 1) + (lane & (KEYS - 1)));
  };
  const auto copy_v = [&](int i) { copy(i, a.p.v); };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    if (i & 1) copy_v(i / 2);
    else copy_k(i / 2, i / 2, first[i / 2]);
  }
  found = first[AHEAD];
  float o[STEPS][NR][4] = {}, m[2 * MT], l[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) m[i] = -INFINITY, l[i] = 0.f;
  cp_wait<SLOTS - 1>();
  __syncthreads();   // the queries are there
  // one tile of rows stays in registers
  uint32_t q[NR == 1 ? STEPS : 1][4];
  const uint32_t qa = sq + ((lane & 7) + (NR > 1 ? 8 * (lane >> 3 & 1) : 0)) * PITCH + (NR > 1 ? lane >> 4 : lane >> 3 & 1) * 16;
  if constexpr (NR == 1) {
#pragma unroll
    for (int x = 0; x < STEPS; x += 2) {
      uint32_t r[4];   // dims 16 x .. + 31 of rows 0..7
      ldm4(r, sq + (lane & 7) * PITCH + (lane >> 3) * 16 + x * 32);
      q[x][0] = r[0]; q[x][2] = r[1]; q[x + 1][0] = r[2]; q[x + 1][2] = r[3];
      q[x][1] = q[x][3] = q[x + 1][1] = q[x + 1][3] = 0;
    }
  }
  const uint32_t ka = ring + (lane & 7) * PITCH + (lane >> 3) * 16;                                    // 8 keys, 32 dims
  const uint32_t va = ring + ((lane & 7) + 8 * (lane >> 4)) * PITCH + (lane >> 3 & 1) * 16;            // 16 keys, 16 dims
  int use = 0;       // slot of the slice at hand
  for (int i = 0; i < mine; ++i) {
    cp_wait<SLOTS - 1>();
    __syncwarp();
    float s[MT][2 * KT][4] = {};
#pragma unroll
    for (int x = 0; x < STEPS; x += 2) {
      uint32_t kk[2 * KT][4];
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n) ldm4(kk[n], ka + use * SLOT + n * 8 * PITCH + x * 32);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          uint32_t qq[4];
          if constexpr (NR > 1) ldm4(qq, qa + mt * 16 * PITCH + (x + y) * 32);
#pragma unroll
          for (int n = 0; n < 2 * KT; ++n) mma16816(s[mt][n], NR > 1 ? qq : q[NR == 1 ? x + y : 0], kk[n][2 * y], kk[n][2 * y + 1]);
        }
    }
    use = use + 1 == SLOTS ? 0 : use + 1;
    const uint32_t bits = (uint32_t)seen & (0xffffffffu >> (32 - KEYS));
    seen >>= KEYS;
    __syncwarp();   // read by all: the slot may be filled again
    if constexpr (SLOTS & 1) copy_v(i + AHEAD - 1);
    else next_k(i + AHEAD);

    // scores, base 2; hidden keys
    const int key = slice_key(i);
    const bool mixed = (a.causal && key + KEYS - 1 > c.first_pos) || (a.window > 0 && key <= c.last_pos - a.window);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = s[mt][n][e] * a.scale_log2;
          s[mt][n][e] = v < kLeast ? kLeast : v;
        }
    if (mixed || bits != (0xffffffffu >> (32 - KEYS))) {
#pragma unroll
      for (int j = 0; j < (NR > 1 ? 2 * MT : 1); ++j) {   // rows g + 8 j
        int from = 0, end_key = c.k1;
        if (mixed) {
          const int pos = c.s.len - c.s.n - c.shift + (int)a.by_group.div(c.r0 + 8 * j + g);
          if (a.causal) end_key = pos + 1;
          if (a.window > 0) from = pos - a.window + 1;
        }
#pragma unroll
        for (int n = 0; n < 2 * KT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int k = 8 * n + 2 * t + e;
            if (!(bits >> k & 1) || (key + k < from && (!SINKS || key + k >= a.sinks)) || key + k >= end_key) s[j >> 1][n][2 * (j & 1) + e] = -INFINITY;
          }
      }
    }
    // running maxima: kept until a score passes them by 2^8, which fp32 sums and bf16 weights bear
    float f[2 * MT];
    bool grew = false;
#pragma unroll
    for (int j = 0; j < (NR > 1 ? 2 * MT : 1); ++j) {
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n) top = fmaxf(top, fmaxf(s[j >> 1][n][2 * (j & 1)], s[j >> 1][n][2 * (j & 1) + 1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      f[j] = 1.f;
      if (top > m[j] + 8.f) {
        f[j] = ex2_approx(m[j] - top);
        m[j] = top;
        grew = true;
      }
      const float mm = m[j] == -INFINITY ? 0.f : m[j];
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n) {
        float* v = s[j >> 1][n] + 2 * (j & 1);
        v[0] = ex2_approx(v[0] - mm);
        v[1] = ex2_approx(v[1] - mm);
        sum += v[0] + v[1];
      }
      l[j] = l[j] * f[j] + sum;
    }
    if (i > 0 && __any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const float f0 = __shfl_sync(0xffffffffu, f[n], 8 * t), f1 = __shfl_sync(0xffffffffu, f[n], 8 * t + 4);
#pragma unroll
        for (int y = 0; y < STEPS; ++y) {
          o[y][n][0] *= f0;
          o[y][n][1] *= f1;
          o[y][n][2] *= f0;
          o[y][n][3] *= f1;
        }
      }
    }
    // weights as two bf16: cut to the upper half, and the rest (above 0 wherever the weight is, so that a weight times an
    // infinite value is no NaN)
    uint32_t hi[NR][2 * KT], lo[NR][2 * KT];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int k = 0; k < 2 * KT; ++k) {
        const float p0 = s[n >> 1][k][2 * (n & 1)], p1 = s[n >> 1][k][2 * (n & 1) + 1];
        const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
        hi[n][k] = __byte_perm(u0, u1, 0x7632);
        lo[n][k] = pack_bf16(fmaxf(p0 - __uint_as_float(u0 & 0xffff0000u), fminf(p0, 1e-30f)),
                             fmaxf(p1 - __uint_as_float(u1 & 0xffff0000u), fminf(p1, 1e-30f)));
      }

    cp_wait<SLOTS - 1>();
    __syncwarp();
    const uint32_t vs = va + use * SLOT;
    // Where rows see different keys, a value that one of them does not see must not reach it, not even as 0 times NaN:
    // infinite and NaN values of such a slice are left out here and added row by row below.
    bool odd = false;
    if (mixed) {
      const __nv_bfloat162 none = __floats2bfloat162_rn(0.f, 0.f);
      __nv_bfloat162 any = none;
#pragma unroll 4
      for (int x = 0; x < STEPS * KT; ++x) {
        uint32_t u[4];
        ldm4t(u, vs + (x % KT) * 16 * PITCH + x / KT * 32);
#pragma unroll
        for (int j = 0; j < 4; ++j) any = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&u[j]), none, any);   // 0 times it: 0 or NaN
      }
      odd = __any_sync(0xffffffffu, !(__low2float(any) == 0.f && __high2float(any) == 0.f));
    }
    // the products of several dims, then those of the rest: a product that adds to the one before waits for it
    constexpr int XS = NR == 1 ? 4 : NR == 2 ? 2 : 1;
#pragma unroll
    for (int x = 0; x < STEPS; x += XS)
#pragma unroll
      for (int u = 0; u < KT; ++u) {
        uint32_t v[XS][4];
#pragma unroll
        for (int y = 0; y < XS; ++y) {
          ldm4t(v[y], vs + u * 16 * PITCH + (x + y) * 32);
          if (odd) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[y][j] &= ~nonfinite2(v[y][j]);
          }
        }
#pragma unroll
        for (int y = 0; y < XS; ++y)
#pragma unroll
          for (int n = 0; n < NR; ++n) mma16816(o[x + y][n], v[y], hi[n][2 * u], hi[n][2 * u + 1]);
#pragma unroll
        for (int y = 0; y < XS; ++y)
#pragma unroll
          for (int n = 0; n < NR; ++n) mma16816(o[x + y][n], v[y], lo[n][2 * u], lo[n][2 * u + 1]);
      }
    if (odd) {
#pragma unroll
      for (int h = 0; h < 2 * KT; ++h) {   // eight keys
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
          const uint32_t from = ring + use * SLOT + (8 * h + k) * PITCH + 2 * g;
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const float p = k & 1 ? s[n >> 1][h][2 * (n & 1) + 1] : s[n >> 1][h][2 * (n & 1)];
            const float p0 = __shfl_sync(0xffffffffu, p, 8 * t + (k >> 1)), p1 = __shfl_sync(0xffffffffu, p, 8 * t + 4 + (k >> 1));
#pragma unroll
            for (int x = 0; x < STEPS; ++x)
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const uint32_t w = lds2(from + x * 32 + y * 16);
                if ((w & 0x7f80u) != 0x7f80u) continue;
                const float val = __uint_as_float(w << 16);
                if (p0 != 0.f) o[x][n][2 * y] += p0 * val;
                if (p1 != 0.f) o[x][n][2 * y + 1] += p1 * val;
              }
          }
        }
      }
    }
    use = use + 1 == SLOTS ? 0 : use + 1;
    __syncwarp();   // read by all: the slot may be filled again
    if constexpr (SLOTS & 1) next_k(i + AHEAD);
    else copy_v(i + AHEAD);
  }

  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    l[j] += __shfl_xor_sync(0xffffffffu, l[j], 1);
    l[j] += __shfl_xor_sync(0xffffffffu, l[j], 2);
  }
  // the warps' sums, scaled to common maxima, to where the ring was
  if (t == 0) {
#pragma unroll
    for (int j = 0; j < NR; ++j) end->m[warp][8 * j + g] = m[j], end->l[warp][8 * j + g] = l[j];
  }
  __syncthreads();
  if (a.clustered) cluster_arrive();   // the ring is free: others may send their shares
  if (!a.warp_heads) common_rows(end);
  float* so = reinterpret_cast<float*>(smem) + warp * (S::kBytes / 4);
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int r = 8 * n + 2 * t;
    const float f0 = a.warp_heads ? 1.f : weight(end->m[warp][r], common_max(end, r));
    const float f1 = a.warp_heads ? 1.f : weight(end->m[warp][r + 1], common_max(end, r + 1));
    float* dst = so + r * S::kPitch + g;
#pragma unroll
    for (int x = 0; x < STEPS; ++x) {
      dst[16 * x] = o[x][n][0] * f0;
      dst[16 * x + S::kPitch] = o[x][n][1] * f1;
      dst[16 * x + 8] = o[x][n][2] * f0;
      dst[16 * x + 8 + S::kPitch] = o[x][n][3] * f1;
    }
  }
  if (a.warp_heads) {   // the warp's rows are its own
    __syncwarp();
    for (int gr = 0; gr < S::kGroups; ++gr) {
      const int r = S::row(gr, lane), d = S::dim(gr, lane);
      if (r < c.rows) put_row<BF16>(a, c, r, d, *reinterpret_cast<const float4*>(so + r * S::kPitch + d), end->m[warp][r], end->l[warp][r], true);
    }
    return;
  }
  __syncthreads();
  finish<BF16, DH, 8 * NR>(a, c, reinterpret_cast<const float*>(smem), end, reinterpret_cast<float4*>(smem + (EXTRA ? RING : kWarps * S::kBytes)));
}

// ---- fp32 ---------------------------------------------------------------------------------------------------------
//
// CUDA cores, packed FMAs. A warp takes a slice of keys by itself: lane (kq, dq) sums the products of KEYS / 4 keys and 8 rows
// over the dims 32 c + 4 dq .. + 3, the eight dq meet in a butterfly that leaves lane (kq, dq) row dq; then every lane has
// DH / 32 dims of all rows. Keys, values and queries come from shared memory (fp32 keys and values are half of what the
// memory of the SM can deliver at 8 rows; the FMAs take as long). One new token: 64 x 4000 keys of 8 heads over 1 of 256 100 us
// (525 MB, 5.3 TB/s), 64 x 8000 of 4 over 2 of 64 119 us (4.4 TB/s).

template <int DH>
constexpr int f32_slice() { return DH == 256 ? 8 : 16; }
template <int DH>
constexpr int f32_slots() { return DH == 64 ? 4 : 3; }
template <int DH>
constexpr int f32_ring() { return kWarps * f32_slots<DH>() * f32_slice<DH>() * DH * 4; }
template <int DH>
constexpr size_t f32_smem() { return (size_t)f32_ring<DH>() + receive_extra<DH, 8>(f32_ring<DH>()) + sizeof(EndShared<8>) + 8 * DH * 4 + kWarps * f32_slice<DH>() * 8 * 4; }

__device__ __forceinline__ void fma2(float2& d, float2 x, float2 y) {
  asm("{\n .reg .b64 a, b, c;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%0, %1};\n fma.rn.f32x2 c, a, b, c;\n mov.b64 {%0, %1}, c;\n}\n"
      : "+f"(d.x), "+f"(d.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
}
__device__ __forceinline__ float4 lds_f4(uint32_t s) {
  const uint4 v = lds16(s);
  return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}

template <int DH, int CTAS, bool SINKS>   // CTAs of an SM
__global__ void __launch_bounds__(kThreads, CTAS) paged_attn_f32_kernel(const PagedAttnArgs a) {
  constexpr int KEYS = f32_slice<DH>(), SLOTS = f32_slots<DH>(), AHEAD = (SLOTS + 1) / 2, SLOT = KEYS * DH * 4, KJ = KEYS / 4, E = DH / 32;
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int RING = f32_ring<DH>(), EXTRA = receive_extra<DH, 8>(RING), END = RING + EXTRA + (int)sizeof(EndShared<8>);
  const uint32_t base = su32(smem), sq = base + END;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, kq = lane >> 3, dq = lane & 7;
  float* sp = reinterpret_cast<float*>(smem + END + 8 * DH * 4) + warp * KEYS * 8;   // weights [key][row]
  EndShared<8>* end = reinterpret_cast<EndShared<8>*>(smem + RING + EXTRA);
  pdl_wait();
  pdl_trigger();
  Piece c;
  Found first[AHEAD + 1], found;
  if (!find_piece<AHEAD + 1, SINKS>(a, 8, KEYS, &c, first) || no_keys(a, c)) return;
  for (int i = threadIdx.x; i < 8 * DH / 4; i += kThreads) {   // [row][dim]
    const int r = i / (DH / 4);
    const bool ok = r < c.rows;
    cp16_or_zero(sq + i * 16, static_cast<const float*>(a.q) + (ok ? row_at(a, c, r, a.q_stride, DH) + i % (DH / 4) * 4 : 0), ok);
  }
  const uint32_t ring = base + warp * (SLOTS * SLOT);
  const int slices = (c.k1 - c.k0 + KEYS - 1) / KEYS, mine = (slices - c.kw + c.wk - 1) / c.wk;
  const auto slice_key = [&](int i) { return c.k0 + (i * c.wk + c.kw) * KEYS; };
  uint64_t seen = 0;
  int64_t cur = -1;
  int slot = 0;
  const auto copy = [&](int i, const void* pool) {
    if (i < mine) {
#pragma unroll
      for (int x = 0; x < KEYS * DH / 128; ++x) {
        const int piece = x * 32 + lane, key = piece / (DH / 4);
        const int64_t e = __shfl_sync(0xffffffffu, cur, key);
        cp16_or_zero(ring + slot * SLOT + piece * 16, static_cast<const float*>(pool) + (e < 0 ? 0 : e) + piece % (DH / 4) * 4, e >= 0);
      }
    }
    cp_commit();
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
  };
  const auto copy_k = [&](int i, int at, const Found& fnd) {
    cur = i < mine ? key_at(a, c, fnd) : -1;
    seen |= (uint64_t)(__ballot_sync(0xffffffffu, cur >= 0) & ((1u << KEYS) - 1)) << (16 * at);
    copy(i, a.p.k);
  };
  const auto next_k = [&](int i) {
    copy_k(i, AHEAD - 1, found);
    if (i + 1 < mine) found = find_key<SINKS>(a, blockIdx.z, c.shift, slice_key(i + 1) + lane % KEYS);
  };
  const auto copy_v = [&](int i) { copy(i, a.p.v); };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    if (i & 1) copy_v(i / 2);
    else copy_k(i / 2, i / 2, first[i / 2]);
  }
  found = first[AHEAD];
  float2 o[8][E / 2];
#pragma unroll
  for (int r = 0; r < 8; ++r)
#pragma unroll
    for (int e = 0; e < E / 2; ++e) o[r][e] = make_float2(0.f, 0.f);
  float m = -INFINITY, l = 0.f;   // of row dq
  cp_wait<SLOTS - 1>();
  __syncthreads();
  int use = 0;
  for (int i = 0; i < mine; ++i) {
    cp_wait<SLOTS - 1>();
    __syncwarp();
    float2 s2[KJ][8];
#pragma unroll
    for (int j = 0; j < KJ; ++j)
#pragma unroll
      for (int r = 0; r < 8; ++r) s2[j][r] = make_float2(0.f, 0.f);
    const uint32_t ks = ring + use * SLOT + kq * KJ * DH * 4 + dq * 16;
#pragma unroll
    for (int x = 0; x < E; ++x) {
      float4 k[KJ];
#pragma unroll
      for (int j = 0; j < KJ; ++j) k[j] = lds_f4(ks + j * DH * 4 + x * 128);
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float4 q = lds_f4(sq + r * DH * 4 + x * 128 + dq * 16);
#pragma unroll
        for (int j = 0; j < KJ; ++j) {
          fma2(s2[j][r], make_float2(k[j].x, k[j].y), make_float2(q.x, q.y));
          fma2(s2[j][r], make_float2(k[j].z, k[j].w), make_float2(q.z, q.w));
        }
      }
    }
    use = use + 1 == SLOTS ? 0 : use + 1;
    const uint32_t bits = (uint32_t)seen & 0xffffu;
    seen >>= 16;
    __syncwarp();   // read by all: the slot may be filled again
    if constexpr (SLOTS & 1) copy_v(i + AHEAD - 1);
    else next_k(i + AHEAD);

    // the butterfly: of 8, 4, 2 rows a lane keeps half and gives the others to its partner
    float s[KJ];
    const int key = slice_key(i);
    const bool mixed = (a.causal && key + KEYS - 1 > c.first_pos) || (a.window > 0 && key <= c.last_pos - a.window);
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      float v[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] = s2[j][r].x + s2[j][r].y;
#pragma unroll
      for (int w = 4; w > 0; w >>= 1)
#pragma unroll
        for (int r = 0; r < w; ++r) {
          const bool up = dq & w;
          const float mine_ = up ? v[r + w] : v[r], other = up ? v[r] : v[r + w];
          v[r] = mine_ + __shfl_xor_sync(0xffffffffu, other, w);
        }
      const float z = v[0] * a.scale_log2;
      s[j] = z < kLeast ? kLeast : z;
      const int k = kq * KJ + j;
      if (!(bits >> k & 1) || (mixed && !row_sees<SINKS>(a, c, dq, key + k))) s[j] = -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int j = 1; j < KJ; ++j) top = fmaxf(top, s[j]);
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
    float f = 1.f;
    const bool grew = top > m + 8.f;
    if (grew) {
      f = exp2f(m - top);
      m = top;
    }
    const float mm = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      const float p = exp2f(s[j] - mm);
      sum += p;
      sp[(kq * KJ + j) * 8 + dq] = p;
    }
    l = l * f + sum;
    if (i > 0 && __any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float fr = __shfl_sync(0xffffffffu, f, r);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) o[r][e].x *= fr, o[r][e].y *= fr;
      }
    }
    cp_wait<SLOTS - 1>();
    __syncwarp();   // values and weights of all lanes
    const uint32_t vs = ring + use * SLOT;
#pragma unroll 4
    for (int k = 0; k < KEYS; ++k) {
      float2 v[E / 2];
      if constexpr (E == 2) {
        asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v[0].x), "=f"(v[0].y) : "r"(vs + k * DH * 4 + lane * 8) : "memory");
      } else {
#pragma unroll
        for (int x = 0; x < E / 4; ++x) {
          const float4 y = lds_f4(vs + k * DH * 4 + x * 512 + lane * 16);
          v[2 * x] = make_float2(y.x, y.y);
          v[2 * x + 1] = make_float2(y.z, y.w);
        }
      }
      const float4 p0 = *reinterpret_cast<const float4*>(sp + k * 8), p1 = *reinterpret_cast<const float4*>(sp + k * 8 + 4);
      const float p[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        if (mixed && p[r] == 0.f) continue;   // a value that this row does not see, whatever it holds
#pragma unroll
        for (int e = 0; e < E / 2; ++e) fma2(o[r][e], make_float2(p[r], p[r]), v[e]);
      }
    }
    use = use + 1 == SLOTS ? 0 : use + 1;
    __syncwarp();   // read by all: the slot and the weights may be written again
    if constexpr (SLOTS & 1) next_k(i + AHEAD);
    else copy_v(i + AHEAD);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  l += __shfl_xor_sync(0xffffffffu, l, 8);
  l += __shfl_xor_sync(0xffffffffu, l, 16);
  if (kq == 0) end->m[warp][dq] = m, end->l[warp][dq] = l;
  __syncthreads();
  if (a.clustered) cluster_arrive();   // the ring is free: others may send their shares
  common_rows(end);
  const float scale = weight(m, common_max(end, dq));
  using S = Sums<DH, 8>;
  static_assert(kWarps * S::kBytes <= RING, "the warps' sums fit the ring");
  float* so = reinterpret_cast<float*>(smem) + warp * (S::kBytes / 4);
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const float f = __shfl_sync(0xffffffffu, scale, r);
    float* row = so + r * S::kPitch;
    if constexpr (E == 2) {
      *reinterpret_cast<float2*>(row + 2 * lane) = make_float2(o[r][0].x * f, o[r][0].y * f);
    } else {
#pragma unroll
      for (int x = 0; x < E / 4; ++x)
        *reinterpret_cast<float4*>(row + 128 * x + 4 * lane) = make_float4(o[r][2 * x].x * f, o[r][2 * x].y * f, o[r][2 * x + 1].x * f, o[r][2 * x + 1].y * f);
    }
  }
  __syncthreads();
  finish<F32, DH, 8>(a, c, reinterpret_cast<const float*>(smem), end, reinterpret_cast<float4*>(smem + (EXTRA ? RING : kWarps * S::kBytes)));
}

template <int DH, int NR, bool SINKS>
cudaError_t launch_tc(const PagedAttnArgs& a, cudaStream_t s) {
  static OncePerDevice once;
  return launch_attn(once, paged_attn_tc_kernel<DH, NR, SINKS>, tc_smem<DH, NR>(a.warp_heads ? kWarps : 1), tc_smem<DH, NR>(kWarps), a, a, s);
}
template <int DH, int CTAS, bool SINKS>
cudaError_t launch_f32(const PagedAttnArgs& a, cudaStream_t s) {
  static OncePerDevice once;
  return launch_attn(once, paged_attn_f32_kernel<DH, CTAS, SINKS>, f32_smem<DH>(), f32_smem<DH>(), a, a, s);
}

template <int DH, bool SINKS>
cudaError_t launch_dh(const PagedAttnArgs& a, cudaStream_t s) {
  cudaError_t e;
  if (a.p.dtype == F32) {
    if constexpr (DH == 64) e = a.f32_ctas == 3 ? launch_f32<DH, 3, SINKS>(a, s) : launch_f32<DH, 2, SINKS>(a, s);
    else e = launch_f32<DH, 2, SINKS>(a, s);
  } else if (a.row_tiles == 1) {
    e = launch_tc<DH, 1, SINKS>(a, s);
  } else {
    if constexpr (DH == 256) e = launch_tc<DH, 2, SINKS>(a, s);   // 16 rows at most
    else e = a.row_tiles == 2 ? launch_tc<DH, 2, SINKS>(a, s) : launch_tc<DH, 4, SINKS>(a, s);
  }
  if (e != cudaSuccess || a.pieces == 1 || a.clustered) return e;
  const dim3 grid((unsigned)a.n_heads * a.p.max_new, DH / 64, a.p.n_seqs);
  return a.p.dtype == F32 ? launch_k(paged_join_kernel<F32, DH>, grid, kThreads, 0, s, a) : launch_k(paged_join_kernel<BF16, DH>, grid, kThreads, 0, s, a);
}

}  // namespace
}  // namespace uad
