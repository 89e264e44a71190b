// Attention of few new tokens over a paged cache that is held in 8 bits.
//
// out = sum_j p_j sv_j c_j with p = softmax(scale sk_j q c'_j): codes c', c of e4m3 and a scale of keys and one of values for each
// block of tokens and head. Half the bytes of a bf16 cache for the same products, so that the instructions of a key count: the tensor
// cores multiply f16 (e4m3 is emulated in mma.sync here), which every code is exactly, two codes an instruction. A warp takes a
// slice of 16 or 32 keys at a time out of a ring of its own, as with bf16 caches, but
// - keys: the 16 bytes of a row that ldmatrix hands out are 16 dims, four to a lane. Which of an MMA's dims they are called does not matter
//   as long as the queries agree: a lane's four bytes are its two registers of B, and the queries lie in shared memory in that order;
// - values: ldmatrix transposes pairs of bytes, so a lane gets two dims of two keys. A byte permutation makes them two dims' pairs of
//   keys: the rows g and g + 8 of A, which stand for the dims 2 g and 2 g + 1;
// - queries: f16 after a power of two that takes each row's largest value to 2^13..2^14: bf16 has fewer bits, and what falls below
//   f16's least is 2^-38 of the largest;
// - scales come through the ring beside the codes. A key's multiplies its scores; a value's multiplies the weights, which are f16
//   of 2^11 p sv / r: r is a power of two, the largest sv so far, as m is the largest score so far. Rounding weights to f16 is an
//   error of 2^-12 at most, an eighth of what the output's own rounding to bf16 is, and 2^-36 of the largest weight for small ones.
#include "kv_pages8.cuh"
#include "paged_attn.cuh"

namespace uad {
namespace {

struct PagedAttn8Args {
  PagedAttnArgs a;
  Scales sc;
};

constexpr float kLag = 4.f;            // how far (base 2) scores may pass their running maximum before it follows: 2^15 holds their weights
constexpr int kWeightBits = 11;        // weights are 2^kWeightBits at the running maximum
constexpr float kLeastScale = 7.888609052210118e-31f;   // 2^-100

__device__ __forceinline__ void mma16816h(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldm4(uint32_t* r, uint32_t s) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(s) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t* r, uint32_t s) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(s) : "memory");
}
__device__ __forceinline__ float2 lds_f2(uint32_t s) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(s) : "memory");
  return v;
}
__device__ __forceinline__ float lds_f(uint32_t s) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(s) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds_u16(uint32_t s) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(s) : "memory");
  return v;
}
__device__ __forceinline__ void sts_u32(uint32_t s, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(s), "r"(v) : "memory"); }
// 4 bytes to shared memory, zeros where ok is false.
__device__ __forceinline__ void cp4_or_zero(uint32_t s, const void* g, bool ok) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(s), "l"(g), "r"(ok ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Four codes: 0x80 in the bytes that are NaN; 0xff there.
__device__ __forceinline__ uint32_t nan_bits(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (nan_bits(w) >> 7) * 0xffu; }

template <int DH, int NR>
constexpr int slice_steps() { return NR == 4 || (DH == 256 && NR == 2) ? 1 : 2; }   // keys of a slice, in sixteens
template <int DH, int NR>   // K and V slices in turn
constexpr int ring_slots() { return DH == 256 ? (NR == 1 ? 3 : 6) : NR == 4 ? 8 : 4; }
template <int DH>
constexpr int row_pitch() { return DH + 16; }        // eight rows of ldmatrix without a bank conflict
template <int DH>
constexpr int query_pitch() { return 2 * DH + 16; }
template <int DH, int NR>
constexpr int slot_bytes() { return slice_steps<DH, NR>() * 16 * (row_pitch<DH>() + 4); }   // codes, then scales
template <int DH, int NR>
constexpr int ring8() { return kWarps * ring_slots<DH, NR>() * slot_bytes<DH, NR>(); }
// a set of queries: rows, then what their scores are multiplied by
template <int DH, int NR>
constexpr int query_bytes() { return 8 * NR * (query_pitch<DH>() + 4); }
template <int DH, int NR>
constexpr size_t smem8(int heads) {
  return (size_t)ring8<DH, NR>() + receive_extra<DH, 8 * NR>(ring8<DH, NR>()) + sizeof(EndShared<8 * NR>) + heads * query_bytes<DH, NR>();
}
template <int DH, int NR>
constexpr int ctas8() { return NR == 4 || DH == 256 ? 2 : DH == 64 && NR == 1 ? 4 : 3; }

// Where a key's codes and scale are in this head, or -1 where no row sees it or its page is none.
struct Place {
  int64_t code, scale;
};
__device__ __forceinline__ Place place_of(const PagedAttnArgs& a, const Scales& sc, const Piece& c, const Found& f) {
  if (f.key >= c.k1 || !f.shown) return {-1, 0};
  if ((unsigned)f.page >= (unsigned)a.p.n_pages) {
    kv_report(a.p, UAD_KV_BAD_PAGE);
    return {-1, 0};
  }
  const int slot = f.token - (int)(a.p.page.div(f.token) * a.p.page.d);
  return {f.page * a.p.page_stride + slot * a.p.slot_stride + c.kvh * a.p.head_stride,
          f.page * sc.page + (slot >> sc.log_block) * sc.block + c.kvh * sc.head};
}

template <int DH, int NR>   // head dim; 8 NR query rows
__global__ void __launch_bounds__(kThreads, ctas8<DH, NR>()) paged_attn8_kernel(const PagedAttn8Args args) {
  constexpr int KT = slice_steps<DH, NR>(), KEYS = 16 * KT, SLOTS = ring_slots<DH, NR>(), AHEAD = (SLOTS + 1) / 2;
  constexpr int MT = (NR + 1) / 2, PITCH = row_pitch<DH>(), QPITCH = query_pitch<DH>(), SLOT = slot_bytes<DH, NR>(), SCALES = KEYS * PITCH;
  constexpr int STEPS = DH / 16, RING = ring8<DH, NR>(), EXTRA = receive_extra<DH, 8 * NR>(RING);
  constexpr int LANES = DH >= 128 ? 8 : DH / 16, AT_ONCE = 32 / LANES;   // lanes that copy 16 bytes each of a key; keys at once
  using S = Sums<DH, 8 * NR>;
  static_assert(kWarps * S::kBytes <= RING, "the warps' sums fit the ring");
  static_assert(AHEAD * KEYS <= 64, "the bits of the keys ahead");
  static_assert(SLOT % 16 == 0, "slots are aligned for 16-byte copies");
  extern __shared__ __align__(16) unsigned char smem[];
  const PagedAttnArgs& a = args.a;
  const uint32_t base = su32(smem);
  EndShared<8 * NR>* end = reinterpret_cast<EndShared<8 * NR>*>(smem + RING + EXTRA);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t sq = base + RING + EXTRA + sizeof(EndShared<8 * NR>) + (a.warp_heads ? warp * query_bytes<DH, NR>() : 0);
  const uint32_t sf = sq + 8 * NR * QPITCH;   // what each row's scores are multiplied by
  pdl_wait();
  pdl_trigger();
  Piece c;
  Found first[AHEAD + 1], found;
  if (!find_piece<AHEAD + 1, true>(a, 8 * NR, KEYS, &c, first) || no_keys(a, c)) return;
  const uint32_t ring = base + warp * (SLOTS * SLOT);
  const int slices = (c.k1 - c.k0 + KEYS - 1) / KEYS, mine = (slices - c.kw + c.wk - 1) / c.wk;
  const auto slice_key = [&](int i) { return c.k0 + (i * c.wk + c.kw) * KEYS; };

  uint64_t seen = 0;   // KEYS bits a slice, the next one lowest
  int64_t at[KEYS / AT_ONCE], scale_at = -1;
  int slot = 0;
  const uint32_t to = ring + lane / LANES * PITCH + lane % LANES * 16;
  const auto copy = [&](int i, const void* pool, const float* scales) {
    if (i < mine) {
#pragma unroll
      for (int h = 0; h < KEYS / AT_ONCE; ++h) {
        const char* src = static_cast<const char*>(pool) + (at[h] < 0 ? 0 : at[h]) + lane % LANES * 16;
#pragma unroll
        for (int x = 0; x < DH / (16 * LANES); ++x) cp16_or_zero(to + slot * SLOT + AT_ONCE * h * PITCH + x * 16 * LANES, src + x * 16 * LANES, at[h] >= 0);
      }
      if (lane < KEYS) cp4_or_zero(ring + slot * SLOT + SCALES + 4 * lane, scales + (scale_at < 0 ? 0 : scale_at), scale_at >= 0);
    }
    cp_commit();
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
  };
  const auto copy_k = [&](int i, int ahead, const Found& fnd) {
    Place e{-1, 0};
    if (i < mine) e = place_of(a, args.sc, c, fnd);
    seen |= (uint64_t)(__ballot_sync(0xffffffffu, e.code >= 0) & (0xffffffffu >> (32 - KEYS))) << (KEYS * ahead);
#pragma unroll
    for (int h = 0; h < KEYS / AT_ONCE; ++h) at[h] = __shfl_sync(0xffffffffu, e.code, AT_ONCE * h + lane / LANES);
    scale_at = e.code < 0 ? -1 : e.scale;
    copy(i, a.p.k, args.sc.k);
  };
  const auto next_k = [&](int i) {
    copy_k(i, AHEAD - 1, found);
    if (i + 1 < mine) found = find_key<true>(a, c.shift, slice_key(i + 1) + (lane & (KEYS - 1)));
  };
  const auto copy_v = [&](int i) { copy(i, a.p.v, args.sc.v); };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    if (i & 1) copy_v(i / 2);
    else copy_k(i / 2, i / 2, first[i / 2]);
  }
  found = first[AHEAD];

  // Queries as f16, each row times a power of two; dims 4 t .. 4 t + 3 of sixteen where an MMA has its 2 t, 2 t + 1, 2 t + 8, 2 t + 9.
  for (int r = a.warp_heads ? 0 : warp; r < 8 * NR; r += a.warp_heads ? 1 : kWarps) {
    constexpr int W = DH / 64;   // pairs of a lane
    uint32_t w[W] = {};
    if (r < c.rows) {
      const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + row_at(a, c, r, a.q_stride, DH) + 2 * W * lane;
      if constexpr (W == 1) w[0] = *reinterpret_cast<const uint32_t*>(src);
      else if constexpr (W == 2) { const uint2 v = *reinterpret_cast<const uint2*>(src); w[0] = v.x; w[1] = v.y; }
      else { const uint4 v = *reinterpret_cast<const uint4*>(src); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    }
    uint32_t top = 0;   // the largest exponent of a finite value
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const uint32_t e0 = w[i] >> 7 & 0xff, e1 = w[i] >> 23 & 0xff;
      top = max(top, max(e0 == 0xff ? 0u : e0, e1 == 0xff ? 0u : e1));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    const uint32_t e = min(127u + 13 + 127 - top, 253u);
    const float f = __uint_as_float(e << 23);
    if (lane == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(sf + 4 * r), "f"(a.scale_log2 * __uint_as_float((254 - e) << 23)) : "memory");
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int d = 2 * (W * lane + i), x = d & 15;
      sts_u32(sq + r * QPITCH + 2 * ((d & ~15) + (x >> 2) * 2 + (x & 2) * 4), pack_f16(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f));
    }
  }
  float o[STEPS][NR][4] = {}, m[2 * MT], l[2 * MT], rf[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) m[i] = -INFINITY, l[i] = 0.f;
  __syncthreads();   // the queries are there
#pragma unroll
  for (int j = 0; j < 2 * MT; ++j) rf[j] = j < NR ? lds_f(sf + 4 * (8 * j + g)) : 0.f;
  uint32_t q[NR == 1 ? STEPS : 1][4];   // one tile of rows stays in registers
  const uint32_t qa = sq + ((lane & 7) + (NR > 1 ? 8 * (lane >> 3 & 1) : 0)) * QPITCH + (NR > 1 ? lane >> 4 : lane >> 3 & 1) * 16;
  if constexpr (NR == 1) {
#pragma unroll
    for (int x = 0; x < STEPS; x += 2) {
      uint32_t r[4];   // dims 16 x .. + 31 of rows 0..7
      ldm4(r, sq + (lane & 7) * QPITCH + (lane >> 3) * 16 + x * 32);
      q[x][0] = r[0]; q[x][2] = r[1]; q[x + 1][0] = r[2]; q[x + 1][2] = r[3];
      q[x][1] = q[x][3] = q[x + 1][1] = q[x + 1][3] = 0;
    }
  }
  float ref = kLeastScale;   // a power of two, no value's scale so far is above it
  const uint32_t ka = ring + (lane & 7) * PITCH + (lane >> 3) * 16;                                    // 8 keys, 64 dims
  const uint32_t va = ring + ((lane & 7) + 8 * (lane >> 3 & 1)) * PITCH + (lane >> 4) * 16;            // 16 keys, 32 dims
  int use = 0;       // slot of the slice at hand
  for (int i = 0; i < mine; ++i) {
    cp_wait<SLOTS - 1>();
    __syncwarp();
    float s[MT][2 * KT][4] = {};
#pragma unroll
    for (int x = 0; x < STEPS; x += 4) {
      uint32_t kk[2 * KT][4];
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n) ldm4(kk[n], ka + use * SLOT + n * 8 * PITCH + x * 16);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        uint32_t qq[MT][4];
        if constexpr (NR > 1)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) ldm4(qq[mt], qa + mt * 16 * QPITCH + (x + y) * 32);
#pragma unroll
        for (int n = 0; n < 2 * KT; ++n) {
          const uint32_t b0 = e4m3_f16(kk[n][y]), b1 = e4m3_f16(kk[n][y] >> 16);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) mma16816h(s[mt][n], NR > 1 ? qq[mt] : q[NR == 1 ? x + y : 0], b0, b1);
        }
      }
    }
    float2 ks[2 * KT];   // the keys' scales
#pragma unroll
    for (int n = 0; n < 2 * KT; ++n) ks[n] = lds_f2(ring + use * SLOT + SCALES + 32 * n + 8 * t);
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
        for (int e = 0; e < (NR > 1 ? 4 : 2); ++e) {
          const float v = s[mt][n][e] * rf[2 * mt + (e >> 1)] * (e & 1 ? ks[n].y : ks[n].x);
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
            if (!(bits >> k & 1) || (key + k < from && key + k >= a.sinks) || key + k >= end_key) s[j >> 1][n][2 * (j & 1) + e] = -INFINITY;
          }
      }
    }
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
      if (top > m[j] + kLag) {
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

    cp_wait<SLOTS - 1>();
    __syncwarp();
    const uint32_t vs = va + use * SLOT;
    // the values' scales: a power of two that none is above goes before the sums
    const float own_scale = lds_f(ring + use * SLOT + SCALES + 4 * (lane & (KEYS - 1)));
    float raised = 1.f;
    if (__any_sync(0xffffffffu, own_scale > ref)) {
      const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(own_scale));
      const float now = __uint_as_float(min((most + 0x7fffffu) & 0xff800000u, 254u << 23));
      raised = ref / now;
      ref = now;
      grew = true;
    }
    if (i > 0 && __any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const float f0 = __shfl_sync(0xffffffffu, f[n], 8 * t) * raised, f1 = __shfl_sync(0xffffffffu, f[n], 8 * t + 4) * raised;
#pragma unroll
        for (int y = 0; y < STEPS; ++y) {
          o[y][n][0] *= f0;
          o[y][n][1] *= f1;
          o[y][n][2] *= f0;
          o[y][n][3] *= f1;
        }
      }
    }
    const float per_ref = __uint_as_float(((254u + kWeightBits) << 23) - __float_as_uint(ref));   // 2^kWeightBits / ref
    uint32_t p[NR][2 * KT];
#pragma unroll
    for (int k = 0; k < 2 * KT; ++k) {
      float2 w = lds_f2(ring + use * SLOT + SCALES + 32 * k + 8 * t);
      w.x *= per_ref;
      w.y *= per_ref;
#pragma unroll
      for (int n = 0; n < NR; ++n) p[n][k] = pack_f16(s[n >> 1][k][2 * (n & 1)] * w.x, s[n >> 1][k][2 * (n & 1) + 1] * w.y);
    }
    // Where rows see different keys, a value that one of them does not see must not reach it, not even as 0 times NaN:
    // NaN codes of such a slice are left out here and added row by row below.
    bool odd = false;
    if (mixed) {
      uint32_t any = 0;
#pragma unroll 4
      for (int x = lane; x < KEYS * DH / 16; x += 32) {
        const uint4 w = lds16(ring + use * SLOT + x / (DH / 16) * PITCH + x % (DH / 16) * 16);
        any |= nan_bits(w.x) | nan_bits(w.y) | nan_bits(w.z) | nan_bits(w.w);
      }
      odd = __any_sync(0xffffffffu, any != 0);
    }
#pragma unroll
    for (int x = 0; x < STEPS; x += 2)
#pragma unroll
      for (int u = 0; u < KT; ++u) {
        uint32_t v[4];   // dims 16 x .. + 15: keys 0..7, keys 8..15; the next sixteen dims
        ldm4t(v, vs + u * 16 * PITCH + x * 16);
        if (odd) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] &= ~nan_bytes(v[j]);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t w0 = __byte_perm(v[2 * y], 0, 0x3120), w1 = __byte_perm(v[2 * y + 1], 0, 0x3120);
          const uint32_t fr[4] = {e4m3_f16(w0), e4m3_f16(w0 >> 16), e4m3_f16(w1), e4m3_f16(w1 >> 16)};
#pragma unroll
          for (int n = 0; n < NR; ++n) mma16816h(o[x + y][n], fr, p[n][2 * u], p[n][2 * u + 1]);
        }
      }
    if (odd) {
#pragma unroll 1
      for (int k = 0; k < KEYS; ++k) {
        if (!(bits >> k & 1)) continue;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const int r = 8 * n + 2 * t;
          const bool see0 = row_sees<true>(a, c, r, key + k), see1 = row_sees<true>(a, c, r + 1, key + k);
          const uint32_t from = ring + use * SLOT + k * PITCH + 2 * g;
#pragma unroll
          for (int x = 0; x < STEPS; ++x) {
            const uint32_t w = nan_bits(lds_u16(from + x * 16));
            if (w & 0x80 && see0) o[x][n][0] = NAN;
            if (w & 0x80 && see1) o[x][n][1] = NAN;
            if (w & 0x8000 && see0) o[x][n][2] = NAN;
            if (w & 0x8000 && see1) o[x][n][3] = NAN;
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
  const float unit = ref * (1.f / (1 << kWeightBits));
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int r = 8 * n + 2 * t;
    const float f0 = a.warp_heads ? unit : unit * weight(end->m[warp][r], common_max(end, r));
    const float f1 = a.warp_heads ? unit : unit * weight(end->m[warp][r + 1], common_max(end, r + 1));
    float* dst = so + r * S::kPitch + 2 * g;
#pragma unroll
    for (int x = 0; x < STEPS; ++x) {
      *reinterpret_cast<float2*>(dst + 16 * x) = make_float2(o[x][n][0] * f0, o[x][n][2] * f0);
      *reinterpret_cast<float2*>(dst + 16 * x + S::kPitch) = make_float2(o[x][n][1] * f1, o[x][n][3] * f1);
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

template <int DH, int NR>
cudaError_t launch8(const PagedAttn8Args& a, cudaStream_t s) {
  static OncePerDevice once;
  return launch_attn(once, paged_attn8_kernel<DH, NR>, smem8<DH, NR>(a.a.warp_heads ? kWarps : 1), smem8<DH, NR>(kWarps), a.a, a, s);
}

template <int DH>
AttnFit8 fit8() {
  if constexpr (DH == 256) return {{ctas8<DH, 1>(), ctas8<DH, 2>(), 0}, {smem8<DH, 1>(kWarps), smem8<DH, 2>(kWarps), 0}};
  else return {{ctas8<DH, 1>(), ctas8<DH, 2>(), ctas8<DH, 4>()}, {smem8<DH, 1>(kWarps), smem8<DH, 2>(kWarps), smem8<DH, 4>(kWarps)}};
}

template <int DH>
cudaError_t launch_dh8(const PagedAttn8Args& a, cudaStream_t s) {
  cudaError_t e;
  if (a.a.row_tiles == 1) {
    e = launch8<DH, 1>(a, s);
  } else {
    if constexpr (DH == 256) e = launch8<DH, 2>(a, s);   // 16 rows at most
    else e = a.a.row_tiles == 2 ? launch8<DH, 2>(a, s) : launch8<DH, 4>(a, s);
  }
  if (e != cudaSuccess || a.a.pieces == 1 || a.a.clustered) return e;
  const dim3 grid((unsigned)a.a.n_heads * a.a.p.max_new, DH / 64, a.a.p.n_seqs);
  return launch_k(paged_join_kernel<BF16, DH>, grid, kThreads, 0, s, a.a);
}

int attn8_args(const uad_kv_pages8* pages, const uad_kv_seqs* seqs, const uad_attn* t, int sinks, bool device, PagedAttn8Args* a) {
  if (!t) return UAD_EINVAL;
  const int rc = pages8_args(pages, seqs, t->n_rows, device, &a->a.p, &a->sc);
  if (rc) return rc;
  const AttnFit8 fit = a->a.p.dh == 64 ? fit8<64>() : a->a.p.dh == 128 ? fit8<128>() : fit8<256>();
  return attn_split(seqs, t, sinks, device, &fit, &a->a);
}

}  // namespace
}  // namespace uad

using namespace uad;

extern "C" {

int64_t uad_paged_attention8_workspace(const uad_kv_pages8* pages, const uad_kv_seqs* seqs, const uad_attn* attn, int32_t sinks) {
  PagedAttn8Args a{};
  const int rc = attn8_args(pages, seqs, attn, sinks, false, &a);
  return rc ? rc : attn_bytes(a.a);
}

int uad_paged_attention8(const uad_kv_pages8* pages, const uad_kv_seqs* seqs, const uad_attn* attn, int32_t sinks, void* workspace,
                         size_t workspace_bytes, int32_t* status, void* stream) {
  PagedAttn8Args a{};
  const int rc = attn8_args(pages, seqs, attn, sinks, true, &a);
  if (rc) return rc;
  if (a.a.p.n_seqs == 0 || a.a.p.n_rows == 0) return UAD_OK;
  a.a.p.status = status;
  if (!attn_workspace(&a.a, workspace, workspace_bytes)) return UAD_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched(a.a.p.dh == 64 ? launch_dh8<64>(a, s) : a.a.p.dh == 128 ? launch_dh8<128>(a, s) : launch_dh8<256>(a, s));
}

}  // extern "C"
