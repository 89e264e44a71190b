// Attention of few new tokens over a paged key-value cache.
//
// out = sum_j softmax_j(scale q k_j) v_j is bound by reading the keys and values once: 4 Hq / Hkv new flops a byte of a bf16
// cache, far below the tensor cores' rate and too much for the CUDA cores (8 heads over one: 54 TFLOP/s at full bandwidth). So
// a sequence's keys are cut into pieces, one CTA a piece, key/value head and block of query rows; each keeps a running
// maximum and sum of its rows (base 2), and pieces are joined by a second kernel where there are several.
#include "kv_pages.cuh"
#include "once_per_device.h"
#include "ptx.cuh"

using namespace uad;
using namespace uad::ptx;

namespace {

struct PagedAttnArgs {
  PagedArgs p;
  const void* q;
  void* out;
  float* lse;
  const uint8_t* mask;
  int64_t q_stride, out_stride, mask_stride;
  float scale;
  int n_heads, group, causal, window;
  // how the work is split (attn_plan)
  int row_tiles, row_blocks, pieces, piece_keys;
  float* part_o;    // [row][head][piece][dh], unnormalised
  float2* part_ml;  // [row][head][piece]: maximum of the scores (base 2), sum of the weights relative to it
};

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kSlice = 16;   // keys that a warp takes at a time
// A seen key's score is at least this, a hidden one's -infinity: a row that sees nothing (0) and one whose every score
// is -infinity (undefined) stay apart.
constexpr float kLeast = -3.402823466e38f;

// The final division: what a row is from the sum of weighted values `x`, their weights' sum and the scores' maximum.
__device__ __forceinline__ float attn_value(float x, float m, float l) {
  return m == -INFINITY && l == 0.f ? 0.f : m == kLeast ? NAN : x / l;
}
__device__ __forceinline__ float attn_lse(float m, float l) {
  return m == -INFINITY && l == 0.f ? -INFINITY : m == kLeast ? NAN : (m + log2f(l)) * 0.6931471805599453f;
}
__device__ __forceinline__ float weight(float m, float top) { return m == top ? 1.f : exp2f(m - top); }

// The rows and keys of one CTA: rows r0 .. r0 + rows - 1 of (new token, head of the group), keys k0 .. k1 - 1.
struct Piece {
  SeqRows s;
  int r0, rows, kvh, piece, k0, k1;
  int first_pos, last_pos;   // positions of the first and the last row
};
// False: nothing to do.
__device__ __forceinline__ bool find_piece(const PagedAttnArgs& a, int block_rows, Piece* c) {
  const PagedArgs& p = a.p;
  const int b = blockIdx.z;
  c->s = seq_rows(p, b);
  const int rb = blockIdx.x % a.row_blocks;
  c->piece = blockIdx.x / a.row_blocks;
  c->kvh = blockIdx.y;
  if (c->s.n < 0) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) kv_report(p, UAD_KV_BAD_SEQ);
    return false;
  }
  c->r0 = rb * block_rows;
  c->rows = min(block_rows, c->s.n * a.group - c->r0);
  if (c->rows <= 0) return false;
  const int before = c->s.len - c->s.n;
  c->first_pos = before + c->r0 / a.group;
  c->last_pos = before + (c->r0 + c->rows - 1) / a.group;
  const int hi = a.causal ? c->last_pos + 1 : c->s.len;
  const int lo = a.window > 0 ? max(0, c->first_pos - a.window + 1) : 0;
  const int64_t from = lo + (int64_t)c->piece * a.piece_keys, to = from + a.piece_keys;
  c->k0 = from < hi ? (int)from : hi;
  c->k1 = c->piece == a.pieces - 1 || to > hi ? hi : (int)to;
  return true;
}
__device__ __forceinline__ int row_token(const PagedAttnArgs& a, const Piece& c, int r) { return c.s.first + (c.r0 + r) / a.group; }
__device__ __forceinline__ int row_head(const PagedAttnArgs& a, const Piece& c, int r) { return c.kvh * a.group + (c.r0 + r) % a.group; }

// Element offset of a key of this CTA's head, or -1 where no row sees it or its page is none.
__device__ __forceinline__ int64_t key_at(const PagedAttnArgs& a, const Piece& c, const int* row, int key) {
  if (key >= c.k1) return -1;
  const int b = blockIdx.z;
  if (a.mask && !a.mask[b * a.mask_stride + key]) return -1;
  const int64_t e = token_at(a.p, row, key);
  if (e < 0) {
    kv_report(a.p, UAD_KV_BAD_PAGE);
    return -1;
  }
  return e + c.kvh * a.p.head_stride;
}
// Row r sees key (which is one that somebody sees).
__device__ __forceinline__ bool row_sees(const PagedAttnArgs& a, const Piece& c, int r, int key) {
  const int pos = c.s.len - c.s.n + (c.r0 + r) / a.group;
  return (!a.causal || key <= pos) && (a.window == 0 || key > pos - a.window);
}

// What a CTA's merged rows become: `x` four dimensions from d of row r.
template <int T, int DH>
__device__ __forceinline__ void store_row(const PagedAttnArgs& a, const Piece& c, int r, int d, float4 x, float m, float l) {
  const int64_t t = row_token(a, c, r), h = row_head(a, c, r);
  if (a.pieces > 1) {
    const int64_t at = (t * a.n_heads + h) * a.pieces + c.piece;
    *reinterpret_cast<float4*>(a.part_o + at * DH + d) = x;
    if (d == 0) a.part_ml[at] = make_float2(m, l);
    return;
  }
  x = make_float4(attn_value(x.x, m, l), attn_value(x.y, m, l), attn_value(x.z, m, l), attn_value(x.w, m, l));
  const int64_t e = t * a.out_stride + h * DH + d;
  if constexpr (T == F32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + e) = x;
  else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + e) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
  if (a.lse && d == 0) a.lse[t * a.n_heads + h] = attn_lse(m, l);
}
// A piece without keys.
template <int T, int DH>
__device__ void store_nothing(const PagedAttnArgs& a, const Piece& c) {
  if (a.pieces > 1) {   // the join reads no values where the sum is 0
    for (int r = threadIdx.x; r < c.rows; r += blockDim.x)
      a.part_ml[((int64_t)row_token(a, c, r) * a.n_heads + row_head(a, c, r)) * a.pieces + c.piece] = make_float2(-INFINITY, 0.f);
    return;
  }
  for (int i = threadIdx.x; i < c.rows * (DH / 4); i += blockDim.x)
    store_row<T, DH>(a, c, i / (DH / 4), i % (DH / 4) * 4, make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f);
}

// ---- bf16 -------------------------------------------------------------------------------------------------------
//
// mma.sync m16n8k16: a warp takes 16 keys at a time by itself, with no barrier in the loop. Both products take their
// contraction in an order that suits the loads, so that every thread needs exactly the 16-byte pieces that it
// copies itself (cp.async, in a ring of its own in shared memory, lanes side by side: no bank conflict, no exchange):
//   S = Q K^T, A = Q (16 rows), B = 8 keys: lane (g, t) has key g, dims 32 c + 8 t .. + 7, two k-steps' worth;
//   O^T = V^T P^T, A = V^T (16 dims x 16 keys): lane (g, t) has keys 2t, 2t + 1, 2t + 8, 2t + 9, dims 64 c + 8 g .. + 7;
//   a k pair is two keys' halves put together, and B = P^T is S's own register layout.
// P goes in as two bf16 (the cut value and the rest): a second MMA where the pipe idles, for an error of 2^-16
// and not 2^-9. The tensor cores (tcgen05) would need 128 rows where there are 8 to 32.

__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes to shared memory, zeros where ok is false (the address is not read then).
__device__ __forceinline__ void cp16_or_zero(uint32_t s, const void* g, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(s), "l"(g), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t s) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(s) : "memory");
  return v;
}
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// Two bf16: whether either is infinite or NaN, and the pair with such ones as 0.
__device__ __forceinline__ uint32_t nonfinite2(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

template <int DH>
constexpr int ring_slots() { return DH == 256 ? 3 : DH == 128 ? 4 : 6; }   // K and V slices in turn, 32 DH bytes each
template <int DH, int NR>
constexpr size_t tc_smem() { return (size_t)kWarps * ring_slots<DH>() * 32 * DH + (size_t)((NR + 1) / 2) * 32 * DH + 2 * kWarps * 8 * NR * 4; }

template <int DH, int NR>   // head dim; 8 NR query rows
__global__ void __launch_bounds__(kThreads, DH == 256 || NR == 4 ? 2 : 3) paged_attn_tc_kernel(const PagedAttnArgs a, float scale_log2) {
  constexpr int SLOTS = ring_slots<DH>(), AHEAD = (SLOTS + 1) / 2, MT = (NR + 1) / 2, C = DH / 32, D = DH / 64, SLOT = 32 * DH;
  static_assert(SLOTS >= NR, "the warps' merge fits the ring");
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t base = su32(smem);
  const uint32_t sq = base + kWarps * SLOTS * SLOT;
  float* sm = reinterpret_cast<float*>(smem + kWarps * SLOTS * SLOT + MT * 32 * DH);
  float* sl = sm + kWarps * 8 * NR;
  pdl_wait();
  pdl_trigger();
  Piece c;
  if (!find_piece(a, 8 * NR, &c)) return;
  if (c.k0 >= c.k1) {
    store_nothing<BF16, DH>(a, c);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t ring = base + warp * (SLOTS * SLOT) + lane * 16;
  const int* row = a.p.table + blockIdx.z * a.p.table_stride;
  const __nv_bfloat16 *kp = static_cast<const __nv_bfloat16*>(a.p.k), *vp = static_cast<const __nv_bfloat16*>(a.p.v);
  const int slices = (c.k1 - c.k0 + kSlice - 1) / kSlice, mine = (slices - warp + kWarps - 1) / kWarps;
  const auto slice_key = [&](int i) { return c.k0 + (i * kWarps + warp) * kSlice; };
  // keys of a slice: lanes l and l + 16 look up key l
  const auto look_up = [&](int i) { return i < mine ? key_at(a, c, row, slice_key(i) + (lane & 15)) : (int64_t)-1; };

  uint64_t seen = 0;   // 16 bits a slice, the next one lowest
  int64_t next = look_up(0), cur = -1;
  int slot = 0;
  const auto copy_k = [&](int i, int at) {
    cur = next;
    seen |= (uint64_t)(__ballot_sync(0xffffffffu, cur >= 0) & 0xffffu) << (16 * at);
    if (i < mine) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int64_t e = __shfl_sync(0xffffffffu, cur, 8 * n + g);
        const __nv_bfloat16* src = kp + (e < 0 ? 0 : e) + 8 * t;
#pragma unroll
        for (int x = 0; x < C; ++x) cp16_or_zero(ring + slot * SLOT + (n * C + x) * 512, src + 32 * x, e >= 0);
      }
    }
    cp_commit();
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
    next = look_up(i + 1);
  };
  const auto copy_v = [&](int i) {
    if (i < mine) {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int64_t e = __shfl_sync(0xffffffffu, cur, 2 * t + (n & 1) + 8 * (n >> 1));
        const __nv_bfloat16* src = vp + (e < 0 ? 0 : e) + 8 * g;
#pragma unroll
        for (int x = 0; x < D; ++x) cp16_or_zero(ring + slot * SLOT + (n * D + x) * 512, src + 64 * x, e >= 0);
      }
    }
    cp_commit();
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
  };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    if (i & 1) copy_v(i / 2);
    else copy_k(i / 2, i / 2);
  }
  // the queries, in the order of the A operand
  for (int i = threadIdx.x; i < MT * C * 64; i += kThreads) {
    const int ln = i & 31, half = (i >> 5) & 1, x = (i >> 6) % C, mt = (i >> 6) / C, r = mt * 16 + half * 8 + (ln >> 2);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < c.rows)
      v = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + row_token(a, c, r) * a.q_stride +
                                          (int64_t)row_head(a, c, r) * DH + 32 * x + 8 * (ln & 3));
    *reinterpret_cast<uint4*>(smem + kWarps * SLOTS * SLOT + i * 16) = v;
  }
  __syncthreads();

  float o[DH / 16][NR][4] = {}, m[2 * MT], l[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) m[i] = -INFINITY, l[i] = 0.f;
  int use = 0;   // slot of the slice at hand
  for (int i = 0; i < mine; ++i) {
    cp_wait<SLOTS - 1>();
    float s[MT][2][4] = {};
#pragma unroll
    for (int x = 0; x < C; ++x) {
      uint4 kk[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) kk[n] = lds16(ring + use * SLOT + (n * C + x) * 512);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const uint4 q0 = lds16(sq + ((mt * C + x) * 2) * 512 + lane * 16);
        const uint4 q1 = NR > 1 ? lds16(sq + ((mt * C + x) * 2 + 1) * 512 + lane * 16) : make_uint4(0, 0, 0, 0);
        const uint32_t a0[4] = {q0.x, q1.x, q0.y, q1.y}, a1[4] = {q0.z, q1.z, q0.w, q1.w};
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          mma16816(s[mt][n], a0, kk[n].x, kk[n].y);
          mma16816(s[mt][n], a1, kk[n].z, kk[n].w);
        }
      }
    }
    use = use + 1 == SLOTS ? 0 : use + 1;
    const uint32_t bits = (uint32_t)seen & 0xffffu;
    seen >>= 16;
    if constexpr (SLOTS & 1) copy_v(i + AHEAD - 1);
    else copy_k(i + AHEAD, AHEAD - 1);

    // scores, base 2; hidden keys
    const int key = slice_key(i);
    const bool mixed = (a.causal && key + kSlice - 1 > c.first_pos) || (a.window > 0 && key <= c.last_pos - a.window);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = s[mt][n][e] * scale_log2;
          s[mt][n][e] = v < kLeast ? kLeast : v;
        }
    if (mixed || bits != 0xffffu) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int k = 8 * n + 2 * t + (e & 1);
            if (!(bits >> k & 1) || (mixed && !row_sees(a, c, mt * 16 + g + 8 * (e >> 1), key + k))) s[mt][n][e] = -INFINITY;
          }
    }
    // running maxima: kept until a score passes them by 2^8, which fp32 sums and bf16 weights bear
    float f[2 * MT];
    bool grew = false;
#pragma unroll
    for (int j = 0; j < (NR > 1 ? 2 * MT : 1); ++j) {
      float* v0 = s[j >> 1][0] + 2 * (j & 1);
      float* v1 = s[j >> 1][1] + 2 * (j & 1);
      float top = fmaxf(fmaxf(v0[0], v0[1]), fmaxf(v1[0], v1[1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      f[j] = 1.f;
      if (top > m[j] + 8.f) {
        f[j] = exp2f(m[j] - top);
        m[j] = top;
        grew = true;
      }
      const float mm = m[j] == -INFINITY ? 0.f : m[j];
      v0[0] = ex2_approx(v0[0] - mm);
      v0[1] = ex2_approx(v0[1] - mm);
      v1[0] = ex2_approx(v1[0] - mm);
      v1[1] = ex2_approx(v1[1] - mm);
      l[j] = l[j] * f[j] + ((v0[0] + v0[1]) + (v1[0] + v1[1]));
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const float f0 = __shfl_sync(0xffffffffu, f[n], 8 * t), f1 = __shfl_sync(0xffffffffu, f[n], 8 * t + 4);
#pragma unroll
        for (int y = 0; y < DH / 16; ++y) {
          o[y][n][0] *= f0;
          o[y][n][1] *= f1;
          o[y][n][2] *= f0;
          o[y][n][3] *= f1;
        }
      }
    }
    // weights as two bf16: cut to the upper half, and the rest (above 0 wherever the weight is, so that a weight times an
    // infinite value is no NaN)
    uint32_t hi[NR][2], lo[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float p0 = s[n >> 1][k][2 * (n & 1)], p1 = s[n >> 1][k][2 * (n & 1) + 1];
        const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
        hi[n][k] = __byte_perm(u0, u1, 0x7632);
        lo[n][k] = pack_bf16(fmaxf(p0 - __uint_as_float(u0 & 0xffff0000u), fminf(p0, 1e-30f)),
                             fmaxf(p1 - __uint_as_float(u1 & 0xffff0000u), fminf(p1, 1e-30f)));
      }

    cp_wait<SLOTS - 1>();
    const uint32_t vs = ring + use * SLOT;
    // Where rows see different keys, a value that one of them does not see must not reach it, not even as 0 times NaN:
    // infinite and NaN values of such a slice are left out here and added row by row below.
    bool odd = false;
    if (mixed) {
#pragma unroll 1
      for (int x = 0; x < 4 * D; ++x) {
        const uint4 w = lds16(vs + x * 512);
        odd |= (nonfinite2(w.x) | nonfinite2(w.y) | nonfinite2(w.z) | nonfinite2(w.w)) != 0;
      }
      odd = __any_sync(0xffffffffu, odd);
    }
#pragma unroll
    for (int x = 0; x < D; ++x) {
      uint32_t w[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const uint4 v = lds16(vs + (n * D + x) * 512);
        w[n][0] = v.x; w[n][1] = v.y; w[n][2] = v.z; w[n][3] = v.w;
      }
      if (odd) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) w[n][j] &= ~nonfinite2(w[n][j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t v[4] = {__byte_perm(w[0][j], w[1][j], 0x5410), __byte_perm(w[0][j], w[1][j], 0x7632),
                               __byte_perm(w[2][j], w[3][j], 0x5410), __byte_perm(w[2][j], w[3][j], 0x7632)};
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          mma16816(o[4 * x + j][n], v, hi[n][0], hi[n][1]);
          mma16816(o[4 * x + j][n], v, lo[n][0], lo[n][1]);
        }
      }
    }
    if (odd) {
      __syncwarp();   // every lane has waited for its copies: each may read the others'
#pragma unroll 1
      for (int k = 0; k < kSlice; ++k) {
        const int tt = (k & 7) >> 1, kn = (k >> 3) * 2 + (k & 1);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const float* pr = s[n >> 1][0] + 2 * (n & 1);
          const float* ps = s[n >> 1][1] + 2 * (n & 1);
          const float p = k < 8 ? (k & 1 ? pr[1] : pr[0]) : (k & 1 ? ps[1] : ps[0]);
          const float p0 = __shfl_sync(0xffffffffu, p, 8 * t + tt), p1 = __shfl_sync(0xffffffffu, p, 8 * t + 4 + tt);
#pragma unroll
          for (int x = 0; x < D; ++x) {
            const uint4 v = lds16(vs - lane * 16 + (g * 4 + tt) * 16 + (kn * D + x) * 512);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t bad = nonfinite2(w[j]);
              const float v0 = __uint_as_float(w[j] << 16), v1 = __uint_as_float(w[j] & 0xffff0000u);
              if (bad & 0xffffu) {
                if (p0 != 0.f) o[4 * x + j][n][0] += p0 * v0;
                if (p1 != 0.f) o[4 * x + j][n][1] += p1 * v0;
              }
              if (bad >> 16) {
                if (p0 != 0.f) o[4 * x + j][n][2] += p0 * v1;
                if (p1 != 0.f) o[4 * x + j][n][3] += p1 * v1;
              }
            }
          }
        }
      }
      __syncwarp();   // before anybody's slot is filled again
    }
    use = use + 1 == SLOTS ? 0 : use + 1;
    if constexpr (SLOTS & 1) copy_k(i + AHEAD, AHEAD - 1);
    else copy_v(i + AHEAD);
  }

  // the four warps' rows become one: relative to the common maximum, summed through shared memory
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    l[j] += __shfl_xor_sync(0xffffffffu, l[j], 1);
    l[j] += __shfl_xor_sync(0xffffffffu, l[j], 2);
    if (t == 0) sm[warp * 8 * NR + 8 * j + g] = m[j], sl[warp * 8 * NR + 8 * j + g] = l[j];
  }
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);   // [warp][row][dh]
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    float f[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 8 * n + 2 * t + e;
      float top = sm[r];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, sm[w * 8 * NR + r]);
      f[e] = weight(sm[warp * 8 * NR + r], top);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int x = 0; x < D; ++x) {
        float4* dst = reinterpret_cast<float4*>(so + (size_t)(warp * 8 * NR + 8 * n + 2 * t + e) * DH + 64 * x + 8 * g);
        dst[0] = make_float4(o[4 * x][n][e] * f[e], o[4 * x][n][2 + e] * f[e], o[4 * x + 1][n][e] * f[e], o[4 * x + 1][n][2 + e] * f[e]);
        dst[1] = make_float4(o[4 * x + 2][n][e] * f[e], o[4 * x + 2][n][2 + e] * f[e], o[4 * x + 3][n][e] * f[e], o[4 * x + 3][n][2 + e] * f[e]);
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < c.rows * (DH / 4); i += kThreads) {
    const int r = i / (DH / 4), d = i % (DH / 4) * 4;
    float4 x = *reinterpret_cast<const float4*>(so + (size_t)r * DH + d);
    float top = sm[r], sum = 0.f;
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      const float4 y = *reinterpret_cast<const float4*>(so + (size_t)(w * 8 * NR + r) * DH + d);
      x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      top = fmaxf(top, sm[w * 8 * NR + r]);
    }
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += sl[w * 8 * NR + r] * weight(sm[w * 8 * NR + r], top);
    store_row<BF16, DH>(a, c, r, d, x, top, sum);
  }
}

// ---- fp32 ---------------------------------------------------------------------------------------------------------

template <int DH>   // one CTA a row: every warp takes each kWarps-th key
__global__ void __launch_bounds__(kThreads) paged_attn_f32_kernel(const PagedAttnArgs a) {
  constexpr int E = DH / 32;
  __shared__ float so[kWarps][DH], sm[kWarps], sl[kWarps];
  pdl_wait();
  pdl_trigger();
  Piece c;
  if (!find_piece(a, 1, &c)) return;
  if (c.k0 >= c.k1) {
    store_nothing<F32, DH>(a, c);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int* row = a.p.table + blockIdx.z * a.p.table_stride;
  float q[E], o[E], m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) {
    q[e] = static_cast<const float*>(a.q)[row_token(a, c, 0) * a.q_stride + (int64_t)row_head(a, c, 0) * DH + lane + 32 * e] * a.scale * 1.4426950408889634f;
    o[e] = 0.f;
  }
  for (int key = c.k0 + warp; key < c.k1; key += kWarps) {
    const int64_t at = key_at(a, c, row, key);
    if (at < 0) continue;
    float d = 0.f;
    for (int e = 0; e < E; ++e) d += q[e] * static_cast<const float*>(a.p.k)[at + lane + 32 * e];
    d = warp_sum(d);
    if (d < kLeast) d = kLeast;
    const float mn = fmaxf(m, d), f = exp2f(m - mn), w = exp2f(d - mn);
    m = mn;
    l = l * f + w;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * static_cast<const float*>(a.p.v)[at + lane + 32 * e];
  }
  for (int e = 0; e < E; ++e) so[warp][lane + 32 * e] = o[e];
  if (lane == 0) sm[warp] = m, sl[warp] = l;
  __syncthreads();
  if (threadIdx.x >= DH / 4) return;
  const int d = threadIdx.x * 4;
  float top = sm[0], sum = 0.f;
  for (int w = 1; w < kWarps; ++w) top = fmaxf(top, sm[w]);
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int w = 0; w < kWarps; ++w) {
    const float f = weight(sm[w], top);
    sum += sl[w] * f;
    x.x += so[w][d] * f; x.y += so[w][d + 1] * f; x.z += so[w][d + 2] * f; x.w += so[w][d + 3] * f;
  }
  store_row<F32, DH>(a, c, 0, d, x, top, sum);
}

// ---- joining pieces ---------------------------------------------------------------------------------------------------

// One CTA a row and head: groups of DH / 4 threads take the pieces in turn.
template <int T, int DH>
__global__ void __launch_bounds__(kThreads) paged_join_kernel(const PagedAttnArgs a) {
  constexpr int TH = DH / 4, GR = kThreads / TH;
  __shared__ float4 so[GR][TH];
  __shared__ float sm[kWarps], sl[GR];
  pdl_wait();
  pdl_trigger();
  const SeqRows s = seq_rows(a.p, blockIdx.z);
  const int j = blockIdx.x / a.n_heads, h = blockIdx.x % a.n_heads;
  if (j >= s.n) return;
  const int64_t t = s.first + j, at = (t * a.n_heads + h) * a.pieces;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < a.pieces; i += kThreads) top = fmaxf(top, a.part_ml[at + i].x);
  top = warp_max(top);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = top;
  __syncthreads();
  top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const int gr = threadIdx.x / TH, d = threadIdx.x % TH;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
#pragma unroll 4
  for (int i = gr; i < a.pieces; i += GR) {
    const float2 ml = a.part_ml[at + i];
    if (ml.y == 0.f) continue;   // nothing was seen there, and no values written
    const float4 y = *reinterpret_cast<const float4*>(a.part_o + (at + i) * DH + 4 * d);
    const float f = weight(ml.x, top);
    x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
    sum += ml.y * f;
  }
  so[gr][d] = x;
  if (d == 0) sl[gr] = sum;
  __syncthreads();
  if (gr) return;
  sum = sl[0];
  for (int i = 1; i < GR; ++i) {
    const float4 y = so[i][d];
    x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    sum += sl[i];
  }
  x = make_float4(attn_value(x.x, top, sum), attn_value(x.y, top, sum), attn_value(x.z, top, sum), attn_value(x.w, top, sum));
  const int64_t e = t * a.out_stride + (int64_t)h * DH + 4 * d;
  if constexpr (T == F32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + e) = x;
  else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + e) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
  if (a.lse && d == 0) a.lse[t * a.n_heads + h] = attn_lse(top, sum);
}

// How many rows a CTA takes and how the keys are cut: enough pieces to fill the SMs twice over, so that sequences of
// different lengths even out, of 64 keys (one slice a warp) and more. From sizes alone: the workspace of a captured
// call holds for what its graph replays.
void attn_plan(const uad_kv_seqs* s, PagedAttnArgs* a) {
  const int dh = a->p.dh, most = a->p.dtype == F32 ? 0 : dh == 256 ? 2 : 4;
  const int64_t rows = (int64_t)a->p.max_new * a->group;
  a->row_tiles = 1;
  while (a->row_tiles < most && 8 * a->row_tiles < rows) a->row_tiles *= 2;
  const int block = most ? 8 * a->row_tiles : 1;
  a->row_blocks = (int)((rows + block - 1) / block);
  int64_t keys = s->max_len > 0 && s->max_len < a->p.capacity ? s->max_len : a->p.capacity;
  if (a->window > 0 && a->window + (int64_t)a->p.max_new - 1 < keys) keys = a->window + (int64_t)a->p.max_new - 1;
  const int64_t units = (int64_t)a->p.n_seqs * a->p.n_kv * a->row_blocks, target = 152 * 4;
  int64_t piece = (keys * units + target - 1) / target;
  piece = (piece + 63) / 64 * 64;
  if (piece < 64) piece = 64;
  a->piece_keys = (int)(piece < (1ll << 30) ? piece : 1ll << 30);
  a->pieces = (int)((keys + a->piece_keys - 1) / a->piece_keys);
  if (a->pieces < 1) a->pieces = 1;
}
// Bytes of the partial rows: maxima and sums, then values.
int64_t attn_bytes(const PagedAttnArgs& a) {
  return a.pieces > 1 ? (int64_t)a.p.n_rows * a.n_heads * a.pieces * (a.p.dh + 2) * 4 : 0;
}

int attn_args(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* t, bool device, PagedAttnArgs* a) {
  if (!t) return UAD_EINVAL;
  const int rc = paged_args(pages, seqs, t->n_rows, device, &a->p);
  if (rc) return rc;
  const int es = a->p.dtype == F32 ? 4 : 2;
  if (t->n_heads < 1 || t->n_heads % a->p.n_kv || t->n_heads / a->p.n_kv > 64) return UAD_EINVAL;
  if ((int64_t)t->n_heads * a->p.max_new >= (1ll << 31)) return UAD_EINVAL;
  if ((t->causal != 0 && t->causal != 1) || t->window < 0 || !isfinite(t->scale)) return UAD_EINVAL;
  if (device) {
    if (!t->q || !t->out || t->q_stride < 0 || t->out_stride < 0 || (t->key_mask && t->mask_stride < 0)) return UAD_EINVAL;
    if (reinterpret_cast<uintptr_t>(t->q) % 16 || reinterpret_cast<uintptr_t>(t->out) % 16) return UAD_EINVAL;
    if (t->q_stride * es % 16 || t->out_stride * es % 16 || reinterpret_cast<uintptr_t>(t->lse) % 4) return UAD_EINVAL;
  }
  a->q = t->q; a->out = t->out; a->lse = t->lse; a->mask = t->key_mask;
  a->q_stride = t->q_stride; a->out_stride = t->out_stride; a->mask_stride = t->mask_stride;
  a->scale = t->scale != 0.f ? t->scale : 1.f / sqrtf((float)a->p.dh);
  a->n_heads = t->n_heads; a->group = t->n_heads / a->p.n_kv; a->causal = t->causal; a->window = t->window;
  attn_plan(seqs, a);
  return UAD_OK;
}

// Kernels of more than 48 KB of shared memory opt in, once on each device.
template <int DH, int NR>
cudaError_t launch_tc(const PagedAttnArgs& a, cudaStream_t s) {
  static OncePerDevice once;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  constexpr int smem = (int)tc_smem<DH, NR>();
  e = (cudaError_t)once.run(dev, [&] { return (int)cudaFuncSetAttribute(paged_attn_tc_kernel<DH, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)a.row_blocks * a.pieces, a.p.n_kv, a.p.n_seqs);
  return launch_k(paged_attn_tc_kernel<DH, NR>, grid, kThreads, smem, s, a, a.scale * 1.4426950408889634f);
}

template <int DH>
cudaError_t launch_dh(const PagedAttnArgs& a, cudaStream_t s) {
  cudaError_t e;
  if (a.p.dtype == F32) {
    e = launch_k(paged_attn_f32_kernel<DH>, dim3((unsigned)a.row_blocks * a.pieces, a.p.n_kv, a.p.n_seqs), kThreads, 0, s, a);
  } else if (a.row_tiles == 1) {
    e = launch_tc<DH, 1>(a, s);
  } else if (a.row_tiles == 2) {
    e = launch_tc<DH, 2>(a, s);
  } else {
    if constexpr (DH < 256) e = launch_tc<DH, 4>(a, s);
    else e = cudaErrorInvalidValue;
  }
  if (e != cudaSuccess || a.pieces == 1) return e;
  const dim3 grid((unsigned)a.n_heads * a.p.max_new, 1, a.p.n_seqs);
  return a.p.dtype == F32 ? launch_k(paged_join_kernel<F32, DH>, grid, kThreads, 0, s, a) : launch_k(paged_join_kernel<BF16, DH>, grid, kThreads, 0, s, a);
}

}  // namespace

extern "C" {

int64_t uad_paged_attention_workspace(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn) {
  PagedAttnArgs a{};
  const int rc = attn_args(pages, seqs, attn, false, &a);
  return rc ? rc : attn_bytes(a);
}

int uad_paged_attention(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn, void* workspace,
                        size_t workspace_bytes, int32_t* status, void* stream) {
  PagedAttnArgs a{};
  const int rc = attn_args(pages, seqs, attn, true, &a);
  if (rc) return rc;
  if (a.p.n_seqs == 0 || a.p.n_rows == 0) return UAD_OK;
  a.p.status = status;
  const int64_t need = attn_bytes(a);
  if (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 || workspace_bytes < (size_t)need)) return UAD_EINVAL;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + (int64_t)a.p.n_rows * a.n_heads * a.pieces * a.p.dh);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = a.p.dh == 64 ? launch_dh<64>(a, s) : a.p.dh == 128 ? launch_dh<128>(a, s) : launch_dh<256>(a, s);
  return e == cudaSuccess ? UAD_OK : UAD_ECUDA;
}

}  // extern "C"
