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
  int warp_heads;   // 1: a CTA's warps have a key/value head each, in one piece; 0: they share one and take its keys in turn
  int f32_ctas;     // CTAs of an SM that the fp32 kernel is compiled for
  int clustered;    // 1: the pieces of a row block are one cluster, which joins them; 0: they go through the workspace
  FastDiv by_group, by_x;   // by_x: of blockIdx.x into row block and piece
  float* part_o;    // [row][head][piece][dh], unnormalised
  float2* part_ml;  // [row][head][piece]: maximum of the scores (base 2), sum of the weights relative to it
};

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kSms = 152;
constexpr int kMaxCluster = 16;   // more than 8 need the opt-in of non-portable sizes
// A seen key's score is at least this, a hidden one's -infinity: a row that sees nothing (0) and one whose every score
// is -infinity (undefined) stay apart.
constexpr float kLeast = -3.402823466e38f;

// 1 / l: what a row's weighted values are multiplied by in the end, from their weights' sum and the scores' maximum.
__device__ __forceinline__ float row_factor(float m, float l) {
  const float f = 1.f / l;
  return m == -INFINITY && l == 0.f ? 0.f : m == kLeast ? NAN : f;
}
__device__ __forceinline__ float row_lse(float m, float l) {
  return m == -INFINITY && l == 0.f ? -INFINITY : m == kLeast ? NAN : (m + log2f(l)) * 0.6931471805599453f;
}
// 2^(m - top), 1 also where both are infinite. Without a branch: a CTA's end is a chain of such steps.
__device__ __forceinline__ float weight(float m, float top) { return ex2_approx(m == top ? 0.f : m - top); }

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
// What this warp has to do; found[N]: the keys of its first N slices (one a lane of `slice` lanes), already on their way.
// False: the whole CTA (and cluster) has nothing to do.
template <int N>
__device__ __forceinline__ bool find_piece(const PagedAttnArgs& a, int block_rows, int slice, Piece* c, Found* found) {
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
#pragma unroll
  for (int i = 0; i < N; ++i) found[i] = find_key(a, c->k0 + (i * c->wk + c->kw) * slice + lane % slice);
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

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer(uint32_t s, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(s), "r"(rank));
  return r;
}
__device__ __forceinline__ void put_peer(uint32_t s, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(s), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void put_peer(uint32_t s, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(s), "f"(v.x), "f"(v.y) : "memory");
}

// A piece that has no keys says so and is done (in a cluster it takes part in the joining). True: it was one.
__device__ __forceinline__ bool no_keys(const PagedAttnArgs& a, const Piece& c) {
  if (c.k0 < c.k1 || a.pieces == 1 || a.clustered) return false;
  for (int r = threadIdx.x; r < c.rows; r += kThreads)
    a.part_ml[row_at(a, c, r, a.n_heads, 1) * a.pieces + c.piece] = make_float2(-INFINITY, 0.f);
  return true;
}

// Four dimensions from d of row r, final or as a piece.
template <int T>
__device__ __forceinline__ void put_row(const PagedAttnArgs& a, const Piece& c, int r, int d, float4 x, float m, float l, bool joined) {
  if (!joined) {
    const int64_t at = row_at(a, c, r, a.n_heads, 1) * a.pieces + c.piece;
    *reinterpret_cast<float4*>(a.part_o + at * a.p.dh + d) = x;
    if (d == 0) a.part_ml[at] = make_float2(m, l);
    return;
  }
  const float f = row_factor(m, l);
  const int64_t e = row_at(a, c, r, a.out_stride, a.p.dh) + d;
  if constexpr (T == F32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + e) = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
  else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + e) = make_uint2(pack_bf16(x.x * f, x.y * f), pack_bf16(x.z * f, x.w * f));
  if (a.lse && d == 0) a.lse[row_at(a, c, r, a.n_heads, 1)] = row_lse(m, l);
}

// A warp's sums lie in shared memory as [row][dim], rows DH + 4 floats apart (so that the accumulators of mma.sync go there
// without bank conflicts). They are handled in groups of 32 float4: 128 dims of a row, or two rows of 64.
template <int DH, int ROWS>
struct Sums {
  static constexpr int kGroups = ROWS * DH / 128, kPitch = DH + 4, kBytes = ROWS * kPitch * 4;
  __device__ static int row(int gr, int lane) { return (gr * 32 + lane) / (DH / 4); }
  __device__ static int dim(int gr, int lane) { return (gr * 32 + lane) % (DH / 4) * 4; }
};
// Shared memory of a CTA's end: the maxima and sums of its warps' rows, and what the cluster's CTAs send it: their
// maxima and sums, and their sums of its share of the groups (which lie in the ring, behind the warps' sums, where they fit).
template <int ROWS>
struct EndShared {
  float m[kWarps][ROWS], l[kWarps][ROWS];
  float2 ml[ROWS], ml_of[kMaxCluster][ROWS];
};
template <int DH, int ROWS>
constexpr int receive_bytes() { return (Sums<DH, ROWS>::kGroups + kMaxCluster - 1) * 512; }
template <int DH, int ROWS>
constexpr int receive_extra(int ring) { return kWarps * Sums<DH, ROWS>::kBytes + receive_bytes<DH, ROWS>() <= ring ? 0 : receive_bytes<DH, ROWS>(); }

// A CTA's four sets of sums, which its warps have scaled to the rows' common maxima e->ml[row].x, become the CTA's, and
// those the cluster's or a piece. so [kWarps]: the sums; receive: where the cluster's share arrives. By all threads, after a
// barrier; in a cluster, each of its CTAs has arrived at the cluster's barrier once its ring was free.
template <int T, int DH, int ROWS>
__device__ __forceinline__ void finish(const PagedAttnArgs& a, const Piece& c, const float* so, EndShared<ROWS>* e, float4* receive) {
  using S = Sums<DH, ROWS>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (a.clustered) cluster_wait();   // every CTA's receiving place is free
  const int share = a.clustered ? (S::kGroups + a.pieces - 1) / a.pieces : 0;
#pragma unroll 2
  for (int gr = warp; gr < S::kGroups; gr += kWarps) {
    const int r = S::row(gr, lane), d = S::dim(gr, lane);
    const float* at = so + r * S::kPitch + d;
    float4 x = *reinterpret_cast<const float4*>(at);
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      const float4 y = *reinterpret_cast<const float4*>(at + w * (S::kBytes / 4));
      x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    if (a.clustered) {   // group i goes to CTA i % pieces, [from][i / pieces]
      put_peer(peer(su32(receive + (c.piece * share + gr / a.pieces) * 32 + lane), gr % a.pieces), x);
    } else if (r < c.rows) {
      const float2 ml = e->ml[r];
      put_row<T>(a, c, r, d, x, ml.x, ml.y, a.pieces == 1);
    }
  }
  if (!a.clustered) return;
  for (int i = threadIdx.x; i < ROWS * a.pieces; i += kThreads) put_peer(peer(su32(&e->ml_of[c.piece][i % ROWS]), i / ROWS), e->ml[i % ROWS]);
  cluster_arrive();
  cluster_wait();   // everybody's share is here; nothing is sent after this
  for (int i = warp; i < share; i += kWarps) {
    const int gr = i * a.pieces + c.piece;
    if (gr >= S::kGroups) break;
    const int r = S::row(gr, lane), d = S::dim(gr, lane);
    float top = -INFINITY, sum = 0.f;
    for (int k = 0; k < a.pieces; ++k) top = fmaxf(top, e->ml_of[k][r].x);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int k = 0; k < a.pieces; ++k) {
      const float4 y = receive[(k * share + i) * 32 + lane];
      const float2 q = e->ml_of[k][r];
      const float f = weight(q.x, top);
      sum += q.y * f;
      x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
    }
    if (r < c.rows) put_row<T>(a, c, r, d, x, top, sum, true);
  }
}
// The rows' common maxima and sums, by the first ROWS threads, after a barrier behind the writes of e->m and e->l.
template <int ROWS>
__device__ __forceinline__ float common_max(const EndShared<ROWS>* e, int r) {
  return fmaxf(fmaxf(e->m[0][r], e->m[1][r]), fmaxf(e->m[2][r], e->m[3][r]));
}
template <int ROWS>
__device__ __forceinline__ void common_rows(EndShared<ROWS>* e) {
  const int r = threadIdx.x;
  if (r >= ROWS) return;
  const float top = common_max(e, r);
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) sum += e->l[w][r] * weight(e->m[w][r], top);
  e->ml[r] = make_float2(top, sum);
}

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

template <int DH, int NR>   // head dim; 8 NR query rows
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
  if (!find_piece<AHEAD + 1>(a, 8 * NR, KEYS, &c, first) || no_keys(a, c)) return;
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
    if (i + 1 < mine) found = find_key(a, slice_key(i + 1) + (lane & (KEYS - 1)));
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
          const int pos = c.s.len - c.s.n + (int)a.by_group.div(c.r0 + 8 * j + g);
          if (a.causal) end_key = pos + 1;
          if (a.window > 0) from = pos - a.window + 1;
        }
#pragma unroll
        for (int n = 0; n < 2 * KT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int k = 8 * n + 2 * t + e;
            if (!(bits >> k & 1) || key + k < from || key + k >= end_key) s[j >> 1][n][2 * (j & 1) + e] = -INFINITY;
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

template <int DH, int CTAS>   // CTAs of an SM
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
  if (!find_piece<AHEAD + 1>(a, 8, KEYS, &c, first) || no_keys(a, c)) return;
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
    if (i + 1 < mine) found = find_key(a, slice_key(i + 1) + lane % KEYS);
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

// ---- joining pieces ---------------------------------------------------------------------------------------------------

// One CTA 64 dims of a row and head: groups of 16 threads take the pieces in turn, 128 pieces at a time, whose weights the threads
// have worked out before, so that the values are requested together (a CTA a row: 60 us against 40 for 8 heads of 256 over
// 131071 keys, whose 304 pieces eight CTAs read).
template <int T, int DH>
__global__ void __launch_bounds__(kThreads) paged_join_kernel(const PagedAttnArgs a) {
  constexpr int TH = 16, GR = kThreads / TH;
  __shared__ float4 so[GR][TH];
  __shared__ float sm[kWarps], sl[kWarps], sw[kThreads];
  pdl_wait();
  pdl_trigger();
  const SeqRows s = seq_rows(a.p, blockIdx.z);
  const int j = blockIdx.x / a.n_heads, h = blockIdx.x % a.n_heads;
  if (j >= s.n) return;
  const int64_t t = s.first + j, at = (t * a.n_heads + h) * a.pieces;
  const float2 none = make_float2(-INFINITY, 0.f);
  float2 ml = threadIdx.x < a.pieces ? a.part_ml[at + threadIdx.x] : none;
  float top = ml.x;
  for (int i = threadIdx.x + kThreads; i < a.pieces; i += kThreads) top = fmaxf(top, a.part_ml[at + i].x);
  top = warp_max(top);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = top;
  __syncthreads();
  top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const int gr = threadIdx.x / TH, d = threadIdx.x % TH;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
  for (int base = 0; base < a.pieces; base += kThreads) {
    if (base > 0) {
      ml = base + (int)threadIdx.x < a.pieces ? a.part_ml[at + base + threadIdx.x] : none;
      __syncthreads();   // the weights before these have been read
    }
    const float w = ml.y == 0.f ? -1.f : weight(ml.x, top);   // -1: nothing was seen there, and no values written
    if (ml.y != 0.f) sum += ml.y * w;
    sw[threadIdx.x] = w;
    __syncthreads();
    const int n = min(kThreads, a.pieces - base);
#pragma unroll 8
    for (int i = gr; i < n; i += GR) {
      const float f = sw[i];
      if (f == -1.f) continue;
      const float4 y = *reinterpret_cast<const float4*>(a.part_o + (at + base + i) * DH + 64 * blockIdx.y + 4 * d);
      x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
    }
  }
  so[gr][d] = x;
  sum = warp_sum(sum);
  if ((threadIdx.x & 31) == 0) sl[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (gr) return;
  sum = (sl[0] + sl[1]) + (sl[2] + sl[3]);
  for (int i = 1; i < GR; ++i) {
    const float4 y = so[i][d];
    x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
  }
  const float f = row_factor(top, sum);
  x = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
  const int64_t e = t * a.out_stride + (int64_t)h * DH + 64 * blockIdx.y + 4 * d;
  if constexpr (T == F32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + e) = x;
  else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + e) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
  if (a.lse && d == 0 && blockIdx.y == 0) a.lse[t * a.n_heads + h] = row_lse(top, sum);
}

// How many rows a CTA takes and how the keys are cut, from sizes alone (the workspace of a captured call holds for what its
// graph replays). A CTA costs about 5 us before and after its keys, so there are no more of them than the SMs hold at once
// (`slots`), and pieces are not shorter than 256 keys (fp32: 64) but where everything is one small wave. A cluster
// joins its pieces in 1 us, the workspace and a second kernel take 3; but clusters are placed as a whole, which leaves
// SMs idle once there are many of them or they are large. Long pieces are cut further, up to four waves, so that
// sequences of different lengths even out; but less than 1.75 waves cost more than one. In us, pieces with / without a
// cluster:
//   1 x 817 keys, 8 heads over 1 of 256:   13: 7.1 / 9.1,  7: 8.3 / 9.6
//   64 x 282..1129, the same:               4: 16.3 / 18.4,  8: 23.3 / 17.1
//   6 x 2001..8003, 5 new tokens:          12: 31.8 / 32.8,  16: 48.1 / 27.5
//   2 x 32768, 131071, 32 over 8 of 128:   28: - / 130,  80: - / 117
//   16 x 4000, 32 over 8 of 128:            3: - / 50,  4: - / 57
//   16 x 700, 8 new tokens, 24 of 64:       1: 16.5,  2: - / 22.6
//   64 x 4000, 4 new tokens, 8 over 1 of 256: 2: - / 75,  4: - / 86
// With more heads than the SMs hold CTAs and up to 512 keys, a CTA's warps may have a key/value head each, which needs no joining. Its
// queries then take four times the shared memory, so that fewer CTAs fit an SM (heads of 256: one and not two), and their number is a
// quarter. Both forms cost their rounds (about 4 us a round, 40000 / head_dim keys of a head, before and after the keys) and the keys
// of the fullest SM, an eighth more where warps have heads, half more where they have 32 rows and are alone on their SM. In us, one
// token, with / without, and what the costs choose:
//   51 x 5 keys, 24 heads of 64:                4.7 / 9.0, with         256 x 60, the same:     21.7 / 40.2, with
//   26 x 512, the same:                        22.7 / 18.9, without     64 x 300, the same:     23.8 / 25.5, with
//   64 x 60, 32 over 8 of 128:                  8.1 / 9.8, with         102 x 512, the same:    40.3 / 37.0, without
//   51 x 60, 8 of 256:                         10.5 / 11.4, with        38 x 300, the same:     28.9 / 19.1, without
//   102 x 60, 128 over 4 of 128:               13.8 / 14.8, with        76 x 512, the same:     49.1 / 20.4, without
// Keys past 512 gain nothing (64 x up to 2000 keys of 24 heads of 64: 106 / 86).
size_t warp_heads_smem(int dh, int row_tiles) {
  if (dh == 64) return row_tiles == 1 ? tc_smem<64, 1>(kWarps) : row_tiles == 2 ? tc_smem<64, 2>(kWarps) : tc_smem<64, 4>(kWarps);
  if (dh == 128) return row_tiles == 1 ? tc_smem<128, 1>(kWarps) : row_tiles == 2 ? tc_smem<128, 2>(kWarps) : tc_smem<128, 4>(kWarps);
  return row_tiles == 1 ? tc_smem<256, 1>(kWarps) : tc_smem<256, 2>(kWarps);
}
struct Split {
  int pieces, piece_keys, clustered;
};
// `keys` in at most n pieces.
Split cut_keys(int64_t keys, int64_t n, int64_t units, int64_t slots) {
  const int64_t piece = ((keys + n - 1) / n + 63) / 64 * 64;
  Split c;
  c.piece_keys = (int)(piece < (1ll << 30) ? piece : 1ll << 30);
  c.pieces = (int)((keys + c.piece_keys - 1) / c.piece_keys);
  const int64_t ctas = units * c.pieces;
  c.clustered = c.pieces > 1 && ((c.pieces <= kMaxCluster && ctas <= kSms) || (c.pieces <= 8 && ctas * 20 <= slots * 17));
  return c;
}
Split split_keys(int64_t keys, int64_t units, int64_t slots, int64_t least) {
  const auto most = [&](int64_t n) { return (keys + n - 1) / n; };   // pieces of at least n keys
  int64_t n;
  if (keys <= kMaxCluster * 256 && units * (most(64) < kMaxCluster ? most(64) : kMaxCluster) <= kSms) {
    n = most(64) < kMaxCluster ? most(64) : kMaxCluster;
  } else {
    n = units * 5 >= slots * 3 ? 1 : units * 2 > slots ? 2 : slots / units;
    if (n > 1 && n <= 8 && units * n * 20 > slots * 17) n = slots * 17 / (units * 20) > 1 ? slots * 17 / (units * 20) : n;
    if (n > most(least)) n = most(least);
    const int64_t waves = 4 * slots / units < most(1024) ? 4 * slots / units : most(1024);
    if (waves > n) n = waves;
    if (n > 2 && units * n > slots && units * n * 4 < slots * 7) n = slots / units > 1 ? slots / units : n;
  }
  return cut_keys(keys, n, units, slots);
}
void attn_plan(const uad_kv_seqs* s, int ctas_per_sm, PagedAttnArgs* a) {
  const int64_t all = s->max_len > 0 && s->max_len < a->p.capacity ? s->max_len : a->p.capacity;
  const int64_t keys = a->window > 0 && a->window + (int64_t)a->p.max_new - 1 < all ? a->window + (int64_t)a->p.max_new - 1 : all;
  const int64_t units = (int64_t)a->p.n_seqs * a->p.n_kv * a->row_blocks, slots = kSms * ctas_per_sm;
  const int64_t least = a->p.dtype == F32 ? 64 : 256;
  a->warp_heads = 0;
  if (a->p.dtype == BF16 && a->p.n_kv % kWarps == 0 && keys <= 512) {
    const int64_t fit = 228 * 1024 / ((int64_t)warp_heads_smem(a->p.dh, a->row_tiles) + 1024);   // an SM's, and what it keeps of each CTA's
    const int64_t ctas = units / kWarps, held = kSms * (fit < ctas_per_sm ? fit : ctas_per_sm), round = 8 * (40000 / a->p.dh);
    const int64_t with = (ctas + held - 1) / held * round + (ctas + kSms - 1) / kSms * kWarps * keys * (a->row_tiles == 4 ? 12 : 9);
    const int64_t without = (units + slots - 1) / slots * round + (units + kSms - 1) / kSms * keys * 8;
    a->warp_heads = with < without;
  }
  Split c = split_keys(keys, units, slots, least);
  if (keys < all && c.pieces > 1 && !c.clustered) {
    // Fewer keys can be more pieces, or as many that are no cluster: no more than there are without the window, so that what
    // a call without one needs is enough for every window. (What makes a cluster of so many pieces makes one of fewer.)
    const int most = split_keys(all, units, slots, least).pieces;
    if (most < c.pieces) c = cut_keys(keys, most, units, slots);
  }
  a->pieces = c.pieces;
  a->piece_keys = c.piece_keys;
  a->clustered = c.clustered;
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
  if (a->p.n_seqs == 0 || a->p.n_rows == 0) return UAD_OK;   // nothing to split: no pieces, no workspace, no launch
  // rows of a CTA: 8, 16 or 32, as many as there are, within what the registers hold
  const int dh = a->p.dh, tiles = a->p.dtype == F32 ? 1 : dh == 256 ? 2 : 4;
  const int64_t rows = (int64_t)a->p.max_new * a->group;
  a->row_tiles = 1;
  while (a->row_tiles < tiles && 8 * a->row_tiles < rows) a->row_tiles *= 2;
  a->row_blocks = (int)((rows + 8 * a->row_tiles - 1) / (8 * a->row_tiles));
  // fp32, 64 dims: three CTAs an SM hide more, two have the registers that make a lone one faster (64 x 8000 keys of two heads 119 us
  // against 132, 33 x 600 with 4 new tokens 10.7 against 12.7; but 28.7 against 22.8 with 16, where two an SM are one wave)
  const int64_t units = (int64_t)a->p.n_seqs * a->p.n_kv * a->row_blocks;
  a->f32_ctas = dh == 64 && (units > 304 || units * 5 < 304 * 3) ? 3 : 2;
  attn_plan(seqs, a->p.dtype == F32 ? a->f32_ctas : a->row_tiles == 4 || dh == 256 ? 2 : dh == 64 && a->row_tiles == 1 ? 4 : 3, a);
  a->by_group = FastDiv((uint32_t)a->group);
  a->by_x = FastDiv((uint32_t)(a->clustered ? a->pieces : a->row_blocks));
  return UAD_OK;
}

// Kernels of more than 48 KB of shared memory opt in, once on each device. Kernel: its address; most: the largest that it is
// launched with.
template <typename Kernel>
cudaError_t launch_attn(OncePerDevice& once, Kernel kernel, size_t smem, size_t most, const PagedAttnArgs& a, cudaStream_t s) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = (cudaError_t)once.run(dev, [&] {
    const cudaError_t f = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return (int)(f != cudaSuccess ? f : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most));
  });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)a.row_blocks * a.pieces, a.warp_heads ? a.p.n_kv / kWarps : a.p.n_kv, a.p.n_seqs);
  return launch_cluster(kernel, grid, dim3(kThreads), smem, a.clustered ? a.pieces : 1, s, a);
}
template <int DH, int NR>
cudaError_t launch_tc(const PagedAttnArgs& a, cudaStream_t s) {
  static OncePerDevice once;
  return launch_attn(once, paged_attn_tc_kernel<DH, NR>, tc_smem<DH, NR>(a.warp_heads ? kWarps : 1), tc_smem<DH, NR>(kWarps), a, s);
}
template <int DH, int CTAS>
cudaError_t launch_f32(const PagedAttnArgs& a, cudaStream_t s) {
  static OncePerDevice once;
  return launch_attn(once, paged_attn_f32_kernel<DH, CTAS>, f32_smem<DH>(), f32_smem<DH>(), a, s);
}

template <int DH>
cudaError_t launch_dh(const PagedAttnArgs& a, cudaStream_t s) {
  cudaError_t e;
  if (a.p.dtype == F32) {
    if constexpr (DH == 64) e = a.f32_ctas == 3 ? launch_f32<DH, 3>(a, s) : launch_f32<DH, 2>(a, s);
    else e = launch_f32<DH, 2>(a, s);
  } else if (a.row_tiles == 1) {
    e = launch_tc<DH, 1>(a, s);
  } else {
    if constexpr (DH == 256) e = launch_tc<DH, 2>(a, s);   // 16 rows at most
    else e = a.row_tiles == 2 ? launch_tc<DH, 2>(a, s) : launch_tc<DH, 4>(a, s);
  }
  if (e != cudaSuccess || a.pieces == 1 || a.clustered) return e;
  const dim3 grid((unsigned)a.n_heads * a.p.max_new, DH / 64, a.p.n_seqs);
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
  return launched(e);
}

}  // extern "C"
