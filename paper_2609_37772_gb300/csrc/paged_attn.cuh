// Attention of few new tokens over a paged key-value cache.
//
// out = sum_j softmax_j(scale q k_j) v_j is bound by reading the keys and values once: 4 Hq / Hkv new flops a byte of a bf16
// cache, far below the tensor cores' rate and too much for the CUDA cores (8 heads over one: 54 TFLOP/s at full bandwidth). So
// a sequence's keys are cut into pieces, one CTA a piece, key/value head and block of query rows; each keeps a running
// maximum and sum of its rows (base 2), and pieces are joined by a second kernel where there are several.
//
// Here: what the kernels of all types share. paged_attn_kernels.cuh has those of bf16 and fp32 caches, paged_attn8.cu those of
// 8 bits, paged_attn.cu the split of the work and the checks.
#pragma once
#include "kv_pages.cuh"
#include "once_per_device.h"
#include "ptx.cuh"

namespace uad {

struct PagedAttnArgs {
  PagedArgs p;
  const void* q;
  void* out;
  float* lse;
  const uint8_t* mask;
  int64_t q_stride, out_stride, mask_stride;
  float scale, scale_log2;   // log2(e) scale
  int n_heads, group, causal, window;
  int sinks;        // first tokens that a window does not hide (kernels with SINKS)
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

constexpr int kAttnSms = 152;
// What an 8-bit cache's kernel holds and takes, by the logarithm of its rows in eights: CTAs of an SM; shared memory of a CTA whose
// warps have heads of their own.
struct AttnFit8 {
  int ctas[3];
  size_t smem[3];
  int round[3];   // keys that the warps of a CTA take at once
};
// paged_attn.cu: the checks of the arguments and how the work is split; attn_split: behind the checks of the pages, of an 8-bit
// cache with what its kernels hold.
int attn_args(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* t, int sinks, bool device, PagedAttnArgs* a);
int attn_split(const uad_kv_seqs* seqs, const uad_attn* t, int sinks, bool device, const AttnFit8* eight, PagedAttnArgs* a);
// Bytes of the partial rows: maxima and sums, then values; and their place in a workspace (false: it does not hold them).
int64_t attn_bytes(const PagedAttnArgs& a);
bool attn_workspace(PagedAttnArgs* a, void* workspace, size_t bytes);
// paged_attn_sinks.cu: the kernels of bf16 and fp32 caches over a window and the first tokens.
cudaError_t launch_paged_sinks(const PagedAttnArgs& a, cudaStream_t s);

namespace {

using namespace ptx;

constexpr int kWarps = 4, kThreads = 32 * kWarps;
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
  int b, r0, rows, kvh, piece, k0, k1, kw, wk;   // b: the sequence
  int first_pos, last_pos;   // positions of the first and the last row
  // Where a window leaves the first tokens visible (SINKS), keys are counted without those that it hides from every row: key i is
  // token i of the sequence below a.sinks and token i + shift from there on. Positions are lowered by shift too.
  int shift;
};
// A key's page and mask as they were loaded; token: its place in the sequence.
struct Found {
  int key, page;
  bool shown;
  int token;
};
template <bool SINKS>
__device__ __forceinline__ Found find_key(const PagedAttnArgs& a, int b, int shift, int key) {
  const int token = SINKS && key >= a.sinks ? key + shift : key;
  Found f{key, -1, false, token};
  if (SINKS ? (unsigned)token < (unsigned)a.p.capacity : token < a.p.capacity) {
    f.page = a.p.table[b * a.p.table_stride + a.p.page.div(token)];
    f.shown = !a.mask || a.mask[b * a.mask_stride + token] != 0;
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
  return f.page * a.p.page_stride + (f.token - (int)(a.p.page.div(f.token) * a.p.page.d)) * a.p.slot_stride + c.kvh * a.p.head_stride;
}
// What this warp has to do; found[N]: the keys of its first N slices (one a lane of `slice` lanes), already on their way.
// False: the whole CTA (and cluster) has nothing to do.
template <int N, bool SINKS>
__device__ __forceinline__ bool find_piece(const PagedAttnArgs& a, int block_rows, int slice, Piece* c, Found* found) {
  const PagedArgs& p = a.p;
  const int b = blockIdx.z, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int x = (int)a.by_x.div(blockIdx.x), rest = blockIdx.x - x * (int)a.by_x.d;
  const int rb = a.clustered ? x : rest;
  c->b = b;
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
  c->shift = SINKS ? min(max(0, lo - a.sinks), p.capacity) : 0;   // a block without rows may lie behind the last token
  const int64_t from = (SINKS ? 0 : lo) + (int64_t)c->piece * a.piece_keys;
  c->k0 = (int)(from < p.capacity - c->shift ? from : p.capacity - c->shift);
#pragma unroll
  for (int i = 0; i < N; ++i) found[i] = find_key<SINKS>(a, b, c->shift, c->k0 + (i * c->wk + c->kw) * slice + lane % slice);
  if (c->s.n < 0) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) kv_report(p, UAD_KV_BAD_SEQ);
    return false;
  }
  c->rows = min(block_rows, c->s.n * a.group - c->r0);
  if (c->rows <= 0) return false;
  c->first_pos = before - c->shift + (int)a.by_group.div(c->r0);
  c->last_pos = before - c->shift + (int)a.by_group.div(c->r0 + c->rows - 1);
  const int hi = a.causal ? c->last_pos + 1 : c->s.len - c->shift;
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
template <bool SINKS>
__device__ __forceinline__ bool row_sees(const PagedAttnArgs& a, const Piece& c, int r, int key) {
  const int pos = c.s.len - c.s.n - c.shift + (int)a.by_group.div(c.r0 + r);
  return (!a.causal || key <= pos) && (a.window == 0 || key > pos - a.window || (SINKS && key < a.sinks));
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
  const int share = a.clustered ? (int)a.by_x.div(S::kGroups + a.pieces - 1) : 0;
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
      const int at_peer = (int)a.by_x.div(gr);
      put_peer(peer(su32(receive + (c.piece * share + at_peer) * 32 + lane), gr - at_peer * a.pieces), x);
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
#pragma unroll 8
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

// Kernels of more than 48 KB of shared memory opt in, once on each device. Kernel: its address; most: the largest that it is
// launched with; args: what it takes.
template <typename Kernel, typename Args>
cudaError_t launch_attn(OncePerDevice& once, Kernel kernel, size_t smem, size_t most, const PagedAttnArgs& a, const Args& args, cudaStream_t s) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = (cudaError_t)once.run(dev, [&] {
    const cudaError_t f = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return (int)(f != cudaSuccess ? f : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most));
  });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)a.row_blocks * a.pieces, a.warp_heads ? a.p.n_kv / kWarps : a.p.n_kv, a.p.n_seqs);
  return launch_cluster(kernel, grid, dim3(kThreads), smem, a.clustered ? a.pieces : 1, s, args);
}

}  // namespace
}  // namespace uad
