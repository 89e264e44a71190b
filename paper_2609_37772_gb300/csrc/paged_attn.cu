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
  float scale, scale_log2;   // log2(e) scale
  int n_heads, group, causal, window;
  // how the work is split (attn_plan)
  int row_tiles;    // query rows of a CTA, in eights
  int row_blocks, pieces, piece_keys;
  int warp_heads;   // 1: a CTA's warps have a key/value head each; 0: they share one and take its keys in turn
  int clustered;    // 1: the pieces of a row block are one cluster, which joins them; 0: they go through the workspace
  FastDiv by_group, by_x;   // by_x: of blockIdx.x into row block and piece
  float* part_o;    // [row][head][piece][dh], unnormalised
  float2* part_ml;  // [row][head][piece]: maximum of the scores (base 2), sum of the weights relative to it
};

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kMaxCluster = 8;
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

// The rows and keys of a warp: rows r0 .. r0 + rows - 1 of (new token, head of the group), keys k0 .. k1 - 1, of which it
// takes the slices kw, kw + wk, ...
struct Piece {
  SeqRows s;
  int r0, rows, kvh, piece, k0, k1, kw, wk;
  int first_pos, last_pos;   // positions of the first and the last row
};
// A key's page and mask as they were loaded.
struct Found {
  int key, page;
  bool shown;
};
__device__ __forceinline__ Found find_key(const PagedAttnArgs& a, int key) {
  Found f{key, -1, false};
  if (key < a.p.capacity) {
    f.page = a.p.table[blockIdx.z * a.p.table_stride + a.p.page.div(key)];
    f.shown = !a.mask || a.mask[blockIdx.z * a.mask_stride + key] != 0;
  }
  return f;
}
// Element offset of the key in this head, or -1 where no row sees it or its page is none.
__device__ __forceinline__ int64_t key_at(const PagedAttnArgs& a, const Piece& c, const Found& f) {
  if (f.key >= c.k1 || !f.shown) return -1;
  if ((unsigned)f.page >= (unsigned)a.p.n_pages) {
    kv_report(a.p, UAD_KV_BAD_PAGE);
    return -1;
  }
  return f.page * a.p.page_stride + (f.key - (int)(a.p.page.div(f.key) * a.p.page.d)) * a.p.slot_stride + c.kvh * a.p.head_stride;
}
// What this warp has to do; `first`: the warp's first slice's keys (one a lane of `slice` lanes), already on their way.
// False: the whole CTA (and cluster) has nothing to do.
__device__ __forceinline__ bool find_piece(const PagedAttnArgs& a, int block_rows, int slice, Piece* c, Found* first) {
  const PagedArgs& p = a.p;
  const int b = blockIdx.z, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int x = (int)a.by_x.div(blockIdx.x), rest = blockIdx.x - x * (int)a.by_x.d;
  const int rb = a.clustered ? x : rest;
  c->piece = a.clustered ? rest : x;
  c->kvh = a.warp_heads ? blockIdx.y * kWarps + warp : blockIdx.y;
  c->kw = a.warp_heads ? 0 : warp;
  c->wk = a.warp_heads ? 1 : kWarps;
  c->s = seq_rows(p, b);
  c->r0 = rb * block_rows;
  // without a window the keys do not depend on the length: their pages are looked up along with it
  int lo = 0;
  const int before = c->s.len - c->s.n;
  if (a.window > 0) lo = max(0, before + (int)a.by_group.div(c->r0) - a.window + 1);
  const int64_t from = lo + (int64_t)c->piece * a.piece_keys;
  c->k0 = (int)(from < p.capacity ? from : p.capacity);
  *first = find_key(a, c->k0 + c->kw * slice + lane % slice);
  if (c->s.n < 0) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) kv_report(p, UAD_KV_BAD_SEQ);
    return false;
  }
  c->rows = min(block_rows, c->s.n * a.group - c->r0);
  if (c->rows <= 0) return false;
  c->first_pos = before + (int)a.by_group.div(c->r0);
  c->last_pos = before + (int)a.by_group.div(c->r0 + c->rows - 1);
  const int hi = a.causal ? c->last_pos + 1 : c->s.len;
  c->k0 = min(c->k0, hi);
  c->k1 = c->piece == a.pieces - 1 || from + a.piece_keys > hi ? hi : (int)(from + a.piece_keys);
  return true;
}
// Element offset of row r's head in a tensor of the token rows.
__device__ __forceinline__ int64_t row_at(const PagedAttnArgs& a, const Piece& c, int r, int64_t stride, int dh) {
  const int j = (int)a.by_group.div(c.r0 + r);
  return (c.s.first + j) * stride + (int64_t)(c.kvh * a.group + c.r0 + r - j * a.group) * dh;
}
// Row r sees key (which is one that somebody sees).
__device__ __forceinline__ bool row_sees(const PagedAttnArgs& a, const Piece& c, int r, int key) {
  const int pos = c.s.len - c.s.n + (int)a.by_group.div(c.r0 + r);
  return (!a.causal || key <= pos) && (a.window == 0 || key > pos - a.window);
}

__device__ __forceinline__ uint4 lds16(uint32_t s) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(s) : "memory");
  return v;
}
// 16 bytes to shared memory, zeros where ok is false (the address is not read then).
__device__ __forceinline__ void cp16_or_zero(uint32_t s, const void* g, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(s), "l"(g), "r"(ok ? 16 : 0) : "memory");
}
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer(uint32_t s, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(s), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 peer_f4(uint32_t s) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(s) : "memory");
  return v;
}
__device__ __forceinline__ float2 peer_f2(uint32_t s) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(s) : "memory");
  return v;
}

// A piece that has no keys says so and is done (in a cluster it takes part in the joining). True: it was one.
__device__ __forceinline__ bool no_keys(const PagedAttnArgs& a, const Piece& c) {
  if (c.k0 < c.k1 || a.pieces == 1 || a.clustered) return false;
  for (int r = a.warp_heads ? threadIdx.x & 31 : threadIdx.x; r < c.rows; r += a.warp_heads ? 32 : kThreads)
    a.part_ml[row_at(a, c, r, a.n_heads, 1) * a.pieces + c.piece] = make_float2(-INFINITY, 0.f);
  return true;
}

// CNT dimensions from d of row r, final or as a piece.
template <int T, int CNT>
__device__ __forceinline__ void put_row(const PagedAttnArgs& a, const Piece& c, int r, int d, const float* x, float m, float l, bool joined) {
  if (!joined) {
    const int64_t at = row_at(a, c, r, a.n_heads, 1) * a.pieces + c.piece;
    float* o = a.part_o + at * a.p.dh + d;
    if constexpr (CNT == 2) *reinterpret_cast<float2*>(o) = make_float2(x[0], x[1]);
#pragma unroll
    for (int i = 0; i + 4 <= CNT; i += 4) *reinterpret_cast<float4*>(o + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    if (d == 0) a.part_ml[at] = make_float2(m, l);
    return;
  }
  float y[CNT];
#pragma unroll
  for (int i = 0; i < CNT; ++i) y[i] = attn_value(x[i], m, l);
  const int64_t e = row_at(a, c, r, a.out_stride, a.p.dh) + d;
  if constexpr (T == F32) {
    float* o = static_cast<float*>(a.out) + e;
#pragma unroll
    for (int i = 0; i < CNT; i += 4) *reinterpret_cast<float4*>(o + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
  } else {
    uint32_t w[CNT / 2];
#pragma unroll
    for (int i = 0; i < CNT / 2; ++i) w[i] = pack_bf16(y[2 * i], y[2 * i + 1]);
    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(a.out) + e;
    if constexpr (CNT == 8) *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint32_t*>(o) = w[0];
  }
  if (a.lse && d == 0) a.lse[row_at(a, c, r, a.n_heads, 1)] = attn_lse(m, l);
}

// How a warp's sums lie in shared memory, in float4. FRAG (bf16): the accumulators' own order: [dims / 64][rows / 8][4][lane], lane
// (g, t) with dims 64 x + 8 g + 2 j, + 1 of rows 8 n + 2 t, + 1. Else (fp32): [row][dims / 4].
template <bool FRAG, int DH, int ROWS>
struct Sums {
  static constexpr int kItems = ROWS * DH / 4;
  __device__ static int row(int i) { return FRAG ? (i / 128 % (ROWS / 8)) * 8 + 2 * (i & 3) : i / (DH / 4); }
  __device__ static int dim(int i) { return FRAG ? i / 128 / (ROWS / 8) * 64 + (i >> 2 & 7) * 8 + (i >> 5 & 3) * 2 : i % (DH / 4) * 4; }
};

// The warps' rows become the CTA's, and those the cluster's or a piece. so [kWarps][items], sm, sl [kWarps][ROWS]: what the
// warps found; ml [ROWS]. Called by all threads after a barrier. Where a CTA's warps have a head each, every warp ends alone.
template <int T, bool FRAG, int DH, int ROWS>
__device__ __forceinline__ void finish(const PagedAttnArgs& a, const Piece& c, float4* so, const float* sm, const float* sl, float2* ml) {
  using S = Sums<FRAG, DH, ROWS>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int from = a.warp_heads ? warp : 0, n = a.warp_heads ? 1 : kWarps;
  constexpr int kJ = FRAG ? 4 : 1;   // items of a thread that go together: 8 dims of two rows, or 4 of one
  constexpr int kR = FRAG ? 2 : 1;
  for (int i = a.warp_heads ? lane : threadIdx.x; i < S::kItems / kJ; i += 32 * n) {
    const int at = FRAG ? (i >> 5) * 128 + (i & 31) : i, r = S::row(at), d = S::dim(at);
    float top[kR], sum[kR];
#pragma unroll
    for (int e = 0; e < kR; ++e) {
      top[e] = sm[from * ROWS + r + e];
      for (int w = 1; w < n; ++w) top[e] = fmaxf(top[e], sm[(from + w) * ROWS + r + e]);
      sum[e] = 0.f;
    }
    float4 x[kJ];
#pragma unroll
    for (int j = 0; j < kJ; ++j) x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = from; w < from + n; ++w) {
      float f[kR];
#pragma unroll
      for (int e = 0; e < kR; ++e) {
        f[e] = weight(sm[w * ROWS + r + e], top[e]);
        sum[e] += sl[w * ROWS + r + e] * f[e];
      }
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        const float4 y = so[w * S::kItems + at + 32 * j];
        x[j].x += y.x * f[0];
        x[j].y += y.y * f[FRAG ? 1 : 0];
        x[j].z += y.z * f[0];
        x[j].w += y.w * f[FRAG ? 1 : 0];
      }
    }
    if (a.clustered) {   // in place of the first warp's, which nobody else reads
#pragma unroll
      for (int j = 0; j < kJ; ++j) so[at + 32 * j] = x[j];
      if (d == 0) {
#pragma unroll
        for (int e = 0; e < kR; ++e) ml[r + e] = make_float2(top[e], sum[e]);
      }
    } else if constexpr (FRAG) {
      const float y0[8] = {x[0].x, x[0].z, x[1].x, x[1].z, x[2].x, x[2].z, x[3].x, x[3].z};
      const float y1[8] = {x[0].y, x[0].w, x[1].y, x[1].w, x[2].y, x[2].w, x[3].y, x[3].w};
      if (r < c.rows) put_row<T, 8>(a, c, r, d, y0, top[0], sum[0], a.pieces == 1);
      if (r + 1 < c.rows) put_row<T, 8>(a, c, r + 1, d, y1, top[kR - 1], sum[kR - 1], a.pieces == 1);
    } else {
      const float y[4] = {x[0].x, x[0].y, x[0].z, x[0].w};
      if (r < c.rows) put_row<T, 4>(a, c, r, d, y, top[0], sum[0], a.pieces == 1);
    }
  }
  if (!a.clustered) return;
  cluster_sync();
  const uint32_t o = su32(so), s = su32(ml);
  for (int i = c.piece * kThreads + threadIdx.x; i < S::kItems; i += a.pieces * kThreads) {   // a share of the items
    const int r = S::row(i), d = S::dim(i);
    if (r >= c.rows) continue;
    float2 q[kMaxCluster][kR];
    float4 y[kMaxCluster];
#pragma unroll
    for (int k = 0; k < kMaxCluster; ++k)
      if (k < a.pieces) {
        y[k] = peer_f4(peer(o + i * 16, k));
#pragma unroll
        for (int e = 0; e < kR; ++e) q[k][e] = peer_f2(peer(s + (r + e) * 8, k));
      }
    float top[kR], sum[kR];
#pragma unroll
    for (int e = 0; e < kR; ++e) {
      top[e] = q[0][e].x;
      sum[e] = 0.f;
#pragma unroll
      for (int k = 1; k < kMaxCluster; ++k)
        if (k < a.pieces) top[e] = fmaxf(top[e], q[k][e].x);
    }
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kMaxCluster; ++k)
      if (k < a.pieces) {
        float f[kR];
#pragma unroll
        for (int e = 0; e < kR; ++e) {
          f[e] = weight(q[k][e].x, top[e]);
          sum[e] += q[k][e].y * f[e];
        }
        x.x += y[k].x * f[0];
        x.y += y[k].y * f[FRAG ? 1 : 0];
        x.z += y[k].z * f[0];
        x.w += y[k].w * f[FRAG ? 1 : 0];
      }
    if constexpr (FRAG) {
      const float y0[2] = {x.x, x.z}, y1[2] = {x.y, x.w};
      put_row<T, 2>(a, c, r, d, y0, top[0], sum[0], true);
      if (r + 1 < c.rows) put_row<T, 2>(a, c, r + 1, d, y1, top[kR - 1], sum[kR - 1], true);
    } else {
      const float y0[4] = {x.x, x.y, x.z, x.w};
      put_row<T, 4>(a, c, r, d, y0, top[0], sum[0], true);
    }
  }
  cluster_sync();   // nobody leaves while another CTA reads its shared memory
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
// and not 2^-9. The tensor cores' own form (tcgen05) would need 128 rows where there are 8 to 32.

constexpr int kSlice = 16;

__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two bf16: ones in the halves that are infinite or NaN.
__device__ __forceinline__ uint32_t nonfinite2(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

template <int DH, int NR>   // K and V slices in turn, 32 DH bytes each
constexpr int ring_slots() { return DH == 256 ? (NR == 1 ? 2 : 3) : DH == 128 ? 4 : 6; }
template <int DH, int NR>   // a head's queries
constexpr int tc_q_bytes() { return ((NR + 1) / 2) * (NR > 1 ? 2 : 1) * 16 * DH; }
template <int DH, int NR>
constexpr size_t tc_smem(int heads) { return (size_t)kWarps * ring_slots<DH, NR>() * 32 * DH + heads * tc_q_bytes<DH, NR>() + 8 * NR * (2 * kWarps * 4 + 8); }
template <int DH, int NR>
constexpr int tc_ctas() { return NR == 4 || (DH == 256 && NR == 2) ? 2 : DH == 64 && NR == 1 ? 4 : 3; }

template <int DH, int NR>   // head dim; 8 NR query rows
__global__ void __launch_bounds__(kThreads, tc_ctas<DH, NR>()) paged_attn_tc_kernel(const PagedAttnArgs a) {
  constexpr int SLOTS = ring_slots<DH, NR>(), AHEAD = (SLOTS + 1) / 2, MT = (NR + 1) / 2, C = DH / 32, D = DH / 64, SLOT = 32 * DH;
  constexpr int QH = NR > 1 ? 2 : 1, QB = tc_q_bytes<DH, NR>();
  static_assert(SLOTS >= NR, "the warps' sums fit the ring");
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t base = su32(smem);
  float* sm = reinterpret_cast<float*>(smem + kWarps * SLOTS * SLOT);   // [warp][row]
  float* sl = sm + kWarps * 8 * NR;
  float2* ml = reinterpret_cast<float2*>(sl + kWarps * 8 * NR);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t sq = base + kWarps * SLOTS * SLOT + 8 * NR * (2 * kWarps * 4 + 8) + (a.warp_heads ? warp * QB : 0);
  pdl_wait();
  pdl_trigger();
  Piece c;
  Found found;
  if (!find_piece(a, 8 * NR, kSlice, &c, &found) || no_keys(a, c)) return;
  // the queries, in the order of the A operand
  for (int i = a.warp_heads ? lane : threadIdx.x; i < MT * C * QH * 32; i += a.warp_heads ? 32 : kThreads) {
    const int ln = i & 31, half = QH == 2 ? i >> 5 & 1 : 0, x = i / (32 * QH) % C, mt = i / (32 * QH * C), r = mt * 16 + half * 8 + (ln >> 2);
    const bool ok = r < c.rows;
    cp16_or_zero(sq + i * 16, static_cast<const __nv_bfloat16*>(a.q) + (ok ? row_at(a, c, r, a.q_stride, DH) + 32 * x + 8 * (ln & 3) : 0), ok);
  }
  const uint32_t ring = base + warp * (SLOTS * SLOT) + lane * 16;
  const __nv_bfloat16 *kp = static_cast<const __nv_bfloat16*>(a.p.k), *vp = static_cast<const __nv_bfloat16*>(a.p.v);
  const int slices = (c.k1 - c.k0 + kSlice - 1) / kSlice, mine = (slices - c.kw + c.wk - 1) / c.wk;
  const auto slice_key = [&](int i) { return c.k0 + (i * c.wk + c.kw) * kSlice; };

  uint64_t seen = 0;   // 16 bits a slice, the next one lowest
  int64_t cur = -1;
  int slot = 0;
  const auto copy_k = [&](int i, int at) {   // lanes l and l + 16 have looked up key l
    cur = i < mine ? key_at(a, c, found) : -1;
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
    if (i + 1 < mine) found = find_key(a, slice_key(i + 1) + (lane & 15));
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
  float o[DH / 16][NR][4] = {}, m[2 * MT], l[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) m[i] = -INFINITY, l[i] = 0.f;
  cp_wait<SLOTS - 1>();
  __syncthreads();   // the queries are there
  int use = 0;       // slot of the slice at hand
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
        const uint4 q0 = lds16(sq + ((mt * C + x) * QH) * 512 + lane * 16);
        const uint4 q1 = QH > 1 ? lds16(sq + ((mt * C + x) * QH + 1) * 512 + lane * 16) : make_uint4(0, 0, 0, 0);
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
          const float v = s[mt][n][e] * a.scale_log2;
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
        f[j] = ex2_approx(m[j] - top);
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
    if (i > 0 && __any_sync(0xffffffffu, grew)) {
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

  // the warps' sums, in the accumulators' order
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();   // the ring becomes the sums' place, of any warp
  float4* so = reinterpret_cast<float4*>(smem);
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    l[j] += __shfl_xor_sync(0xffffffffu, l[j], 1);
    l[j] += __shfl_xor_sync(0xffffffffu, l[j], 2);
    if (t == 0) sm[warp * 8 * NR + 8 * j + g] = m[j], sl[warp * 8 * NR + 8 * j + g] = l[j];
  }
#pragma unroll
  for (int x = 0; x < D; ++x)
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        so[warp * (2 * NR * DH) + ((x * NR + n) * 4 + j) * 32 + lane] = make_float4(o[4 * x + j][n][0], o[4 * x + j][n][1], o[4 * x + j][n][2], o[4 * x + j][n][3]);
  __syncthreads();
  finish<BF16, true, DH, 8 * NR>(a, c, so, sm, sl, ml);
}

// ---- fp32 ---------------------------------------------------------------------------------------------------------
//
// CUDA cores, packed FMAs. A warp takes a slice of keys by itself: lane (kq, dq) sums the products of KEYS / 4 keys and 8 rows
// over the dims 32 c + 4 dq .. + 3, the eight dq meet in a butterfly that leaves lane (kq, dq) row dq; then every lane has
// DH / 32 dims of all rows. Keys, values and queries come from shared memory (fp32 keys and values are half of what the
// memory of the SM can deliver at 8 rows; the FMAs take as long).

template <int DH>
constexpr int f32_slice() { return DH == 256 ? 8 : 16; }
template <int DH>
constexpr int f32_slots() { return DH == 64 ? 4 : 3; }
template <int DH>
constexpr size_t f32_smem() { return (size_t)kWarps * f32_slots<DH>() * f32_slice<DH>() * DH * 4 + 8 * DH * 4 + kWarps * f32_slice<DH>() * 8 * 4 + 8 * (2 * kWarps * 4 + 8); }

__device__ __forceinline__ void fma2(float2& d, float2 x, float2 y) {
  asm("{\n .reg .b64 a, b, c;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%0, %1};\n fma.rn.f32x2 c, a, b, c;\n mov.b64 {%0, %1}, c;\n}\n"
      : "+f"(d.x), "+f"(d.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
}
__device__ __forceinline__ float4 lds_f4(uint32_t s) {
  const uint4 v = lds16(s);
  return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 2) paged_attn_f32_kernel(const PagedAttnArgs a) {
  constexpr int KEYS = f32_slice<DH>(), SLOTS = f32_slots<DH>(), AHEAD = (SLOTS + 1) / 2, SLOT = KEYS * DH * 4, KJ = KEYS / 4, E = DH / 32;
  static_assert(SLOTS * KEYS >= 8, "the warps' sums fit the ring");
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t base = su32(smem), sq = base + kWarps * SLOTS * SLOT;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, kq = lane >> 3, dq = lane & 7;
  float* sp = reinterpret_cast<float*>(smem + kWarps * SLOTS * SLOT + 8 * DH * 4) + warp * KEYS * 8;   // weights [key][row]
  float* sm = reinterpret_cast<float*>(smem + kWarps * SLOTS * SLOT + 8 * DH * 4 + kWarps * KEYS * 8 * 4);
  float* sl = sm + kWarps * 8;
  float2* ml = reinterpret_cast<float2*>(sl + kWarps * 8);
  pdl_wait();
  pdl_trigger();
  Piece c;
  Found found;
  if (!find_piece(a, 8, KEYS, &c, &found) || no_keys(a, c)) return;
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
  const auto copy_k = [&](int i, int at) {
    cur = i < mine ? key_at(a, c, found) : -1;
    seen |= (uint64_t)(__ballot_sync(0xffffffffu, cur >= 0) & ((1u << KEYS) - 1)) << (16 * at);
    copy(i, a.p.k);
    if (i + 1 < mine) found = find_key(a, slice_key(i + 1) + lane % KEYS);
  };
  const auto copy_v = [&](int i) { copy(i, a.p.v); };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    if (i & 1) copy_v(i / 2);
    else copy_k(i / 2, i / 2);
  }
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
    else copy_k(i + AHEAD, AHEAD - 1);

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
      if (!(bits >> k & 1) || (mixed && !row_sees(a, c, dq, key + k))) s[j] = -INFINITY;
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
    if constexpr (SLOTS & 1) copy_k(i + AHEAD, AHEAD - 1);
    else copy_v(i + AHEAD);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  float4* so = reinterpret_cast<float4*>(smem);   // [warp][row][dim]
  l += __shfl_xor_sync(0xffffffffu, l, 8);
  l += __shfl_xor_sync(0xffffffffu, l, 16);
  if (kq == 0) sm[warp * 8 + dq] = m, sl[warp * 8 + dq] = l;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    float* row = reinterpret_cast<float*>(so) + (size_t)(warp * 8 + r) * DH;
    if constexpr (E == 2) {
      *reinterpret_cast<float2*>(row + 2 * lane) = o[r][0];
    } else {
#pragma unroll
      for (int x = 0; x < E / 4; ++x)
        *reinterpret_cast<float4*>(row + 128 * x + 4 * lane) = make_float4(o[r][2 * x].x, o[r][2 * x].y, o[r][2 * x + 1].x, o[r][2 * x + 1].y);
    }
  }
  __syncthreads();
  finish<F32, false, DH, 8>(a, c, so, sm, sl, ml);
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

// How many rows a CTA takes and how the keys are cut: into pieces of 64 keys (a slice a warp) and more, so many that the SMs
// are filled twice over and sequences of different lengths even out. From sizes alone: the workspace of a captured
// call holds for what its graph replays.
void attn_plan(const uad_kv_seqs* s, PagedAttnArgs* a) {
  const int dh = a->p.dh, most = a->p.dtype == F32 ? 1 : dh == 256 ? 2 : 4;
  const int64_t rows = (int64_t)a->p.max_new * a->group;
  a->row_tiles = 1;
  while (a->row_tiles < most && 8 * a->row_tiles < rows) a->row_tiles *= 2;
  a->row_blocks = (int)((rows + 8 * a->row_tiles - 1) / (8 * a->row_tiles));
  int64_t keys = s->max_len > 0 && s->max_len < a->p.capacity ? s->max_len : a->p.capacity;
  if (a->window > 0 && a->window + (int64_t)a->p.max_new - 1 < keys) keys = a->window + (int64_t)a->p.max_new - 1;
  int64_t units = (int64_t)a->p.n_seqs * a->p.n_kv * a->row_blocks;
  const int sms = 152;
  a->warp_heads = a->p.dtype == BF16 && a->p.n_kv % kWarps == 0 && units >= 4 * sms;
  if (a->warp_heads) units /= kWarps;
  const int64_t target = sms * 6;
  int64_t piece = (keys * units + target - 1) / target;
  piece = (piece + 63) / 64 * 64;
  if (piece < 64) piece = 64;
  if ((keys + piece - 1) / piece > kMaxCluster && keys <= kMaxCluster * 512) piece = ((keys + kMaxCluster - 1) / kMaxCluster + 63) / 64 * 64;
  a->piece_keys = (int)(piece < (1ll << 30) ? piece : 1ll << 30);
  a->pieces = (int)((keys + a->piece_keys - 1) / a->piece_keys);
  if (a->pieces < 1) a->pieces = 1;
  a->clustered = a->pieces > 1 && a->pieces <= kMaxCluster && !a->warp_heads;
  a->by_group = FastDiv((uint32_t)a->group);
  a->by_x = FastDiv((uint32_t)(a->clustered ? a->pieces : a->row_blocks));
}
// Bytes of the partial rows: maxima and sums, then values.
int64_t attn_bytes(const PagedAttnArgs& a) {
  return a.pieces > 1 && !a.clustered ? (int64_t)a.p.n_rows * a.n_heads * a.pieces * (a.p.dh + 2) * 4 : 0;
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
  a->scale_log2 = a->scale * 1.4426950408889634f;
  a->n_heads = t->n_heads; a->group = t->n_heads / a->p.n_kv; a->causal = t->causal; a->window = t->window;
  attn_plan(seqs, a);
  return UAD_OK;
}

// Kernels of more than 48 KB of shared memory opt in, once on each device. Kernel: its address; most: the largest that it is
// launched with.
template <typename Kernel>
cudaError_t launch_attn(OncePerDevice& once, Kernel kernel, size_t smem, size_t most, const PagedAttnArgs& a, cudaStream_t s) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = (cudaError_t)once.run(dev, [&] { return (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most); });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)a.row_blocks * a.pieces, a.warp_heads ? a.p.n_kv / kWarps : a.p.n_kv, a.p.n_seqs);
  return launch_cluster(kernel, grid, dim3(kThreads), smem, a.clustered ? a.pieces : 1, s, a);
}
template <int DH, int NR>
cudaError_t launch_tc(const PagedAttnArgs& a, cudaStream_t s) {
  static OncePerDevice once;
  return launch_attn(once, paged_attn_tc_kernel<DH, NR>, tc_smem<DH, NR>(a.warp_heads ? kWarps : 1), tc_smem<DH, NR>(kWarps), a, s);
}
template <int DH>
cudaError_t launch_f32(const PagedAttnArgs& a, cudaStream_t s) {
  static OncePerDevice once;
  return launch_attn(once, paged_attn_f32_kernel<DH>, f32_smem<DH>(), f32_smem<DH>(), a, s);
}

template <int DH>
cudaError_t launch_dh(const PagedAttnArgs& a, cudaStream_t s) {
  cudaError_t e;
  if (a.p.dtype == F32) {
    e = launch_f32<DH>(a, s);
  } else if (a.row_tiles == 1) {
    e = launch_tc<DH, 1>(a, s);
  } else if (a.row_tiles == 2) {
    e = launch_tc<DH, 2>(a, s);
  } else {
    if constexpr (DH < 256) e = launch_tc<DH, 4>(a, s);
    else e = cudaErrorInvalidValue;
  }
  if (e != cudaSuccess || a.pieces == 1 || a.clustered) return e;
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
