// The append to a paged cache that is held in 8 bits: rotation, the blocks' scales, rounding to e4m3.
#include "kv_pages8.cuh"

#include <algorithm>

using namespace uad;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

struct Append8Args {
  PagedArgs p;
  Scales sc;
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  void* q_out;
  int n_heads, rot, log_chunks;
  // keys and values: blocks of the grid's x that are theirs; head groups of the keys (and of the values); threads of a head
  int kv_blocks, kv_groups, log_items;
  FastDiv by_group;   // of a block's number into block of tokens and head group: 2 kv_groups
  // queries
  int groups, block_rows;
  FastDiv row_threads, row_blocks;
};

__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : 0.f;
}
// The least power of two that takes `top` (twice: 2 top) to 448 or below, 2^-100 at the least. From the bits: 448 is 1.75 2^8.
__device__ __forceinline__ float scale_of(float top, bool twice) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u) + (twice ? 1 : 0);
  return __uint_as_float((uint32_t)max(e, 27) << 23);
}
// Two values as e4m3, the first one lower: nearest, ties to even; not finite: NaN.
__device__ __forceinline__ uint32_t e4m3_2(float a, float b) {
  a = fabsf(a) == INFINITY ? NAN : a;
  b = fabsf(b) == INFINITY ? NAN : b;
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
// x / s: a multiplication where s is a power of two, as the scales of this append are.
__device__ __forceinline__ float over(float x, float s, float inv, bool exact) { return exact ? x * inv : __fdiv_rn(x, s); }
__device__ __forceinline__ uint2 round8(const float* x, float s, float inv, bool exact) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = over(x[i], s, inv, exact);
  return make_uint2(e4m3_2(y[0], y[1]) | e4m3_2(y[2], y[3]) << 16, e4m3_2(y[4], y[5]) | e4m3_2(y[6], y[7]) << 16);
}
// Four codes of scale `from` as codes of scale s.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float from, float s, float inv, bool exact) {
  float y[4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float2 f = e4m3_pair(h ? w >> 16 : w);
    y[2 * h] = over(f.x * from, s, inv, exact);
    y[2 * h + 1] = over(f.y * from, s, inv, exact);
  }
  return e4m3_2(y[0], y[1]) | e4m3_2(y[2], y[3]) << 16;
}

// The queries: one thread 16 dimensions of one row, in every a.groups-th of its heads, as in the append of the other types.
template <int IN>
__device__ __forceinline__ void rotate_queries(const Append8Args& a, const uad_rope& rope, const SeqRows& s, int block) {
  const int bj = a.row_blocks.div(block), tj = a.row_threads.div(threadIdx.x);
  if (tj >= a.block_rows) return;
  const int64_t j = (int64_t)bj * a.block_rows + tj;
  const int r = (block - bj * (int)a.row_blocks.d) * kThreads + threadIdx.x - tj * (int)a.row_threads.d;
  if (j >= s.n || r >= (int)a.row_threads.d) return;
  const int group = r >> a.log_chunks, c = r - (group << a.log_chunks), half = a.rot / 2, lo = c * 8;
  const int64_t row = s.first + j;
  const bool turn = lo < half;
  const int e_lo = turn ? lo : c * kItem, e_hi = turn ? lo + half : c * kItem + 8;
  float cs[8], sn[8], x[8], y[8];
  const auto load = [&](int h) {
    const int64_t at = row * a.q_stride + (int64_t)h * a.p.dh;
    load8<IN>(a.q, at + e_lo, x);
    load8<IN>(a.q, at + e_hi, y);
  };
  load(group);
  if (turn)
#pragma unroll
    for (int i = 0; i < 8; ++i) rotation((uint32_t)(s.len - s.n + (int)j), rope.turn[lo + i], cs + i, sn + i);
  for (int h = group;;) {
    if (turn)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = x[i] * cs[i] - y[i] * sn[i], w = y[i] * cs[i] + x[i] * sn[i];
        x[i] = u;
        y[i] = w;
      }
    const int64_t at = row * a.q_out_stride + (int64_t)h * a.p.dh;
    store8<BF16>(a.q_out, at + e_lo, x);
    store8<BF16>(a.q_out, at + e_hi, y);
    h += a.groups;
    if (h >= a.n_heads) break;
    load(h);
  }
}

// Keys and values: a CTA has one block of tokens and some heads of the keys or of the values. A thread holds 16 dimensions of one
// token (ITEMS tokens where a head of the block has more than the threads), as 8 pairs where they are rotated; all
// threads of a head find its largest value, which gives the scale before anything is rotated: a rotation grows no value by more than
// sqrt(2), so keys take twice the largest, and the scale does not hang on how sines round. Earlier tokens of the block,
// which the first block of a sequence can have, belong to threads of their own and are rounded again where the scale has grown:
// exactly, as long as they stay normal numbers.
template <int IN, int ITEMS>
__global__ void __launch_bounds__(kThreads, ITEMS == 1 ? 4 : 2) append8_kernel(const Append8Args a, const __grid_constant__ uad_rope rope) {
  __shared__ uint32_t s_top[2][kWarps];
  pdl_wait();
  pdl_trigger();
  const PagedArgs& p = a.p;
  const int b = blockIdx.y;
  const SeqRows s = seq_rows(p, b);
  if (s.n < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) kv_report(p, UAD_KV_BAD_SEQ);
    return;
  }
  if ((int)blockIdx.x >= a.kv_blocks) {
    rotate_queries<IN>(a, rope, s, blockIdx.x - a.kv_blocks);
    return;
  }
  if (s.n == 0) return;
  const int u = a.by_group.div(blockIdx.x), z = blockIdx.x - u * 2 * a.kv_groups;
  const bool is_v = z >= a.kv_groups;
  const int group = is_v ? z - a.kv_groups : z, p0 = s.len - s.n;
  const int i0 = (int)p.page.div(p0), in_page = p0 - i0 * (int)p.page.d;
  const int number = (in_page >> a.sc.log_block) + u, ahead = (int)a.sc.per_page.div(number);
  const int sub = number - ahead * (int)a.sc.per_page.d, lo_slot = sub << a.sc.log_block;
  const int64_t first64 = (int64_t)(i0 + ahead) * p.page.d + lo_slot;
  if (first64 >= s.len) return;
  const int first = (int)first64, slots = min(1 << a.sc.log_block, (int)p.page.d - lo_slot);
  const int page = p.table[b * p.table_stride + i0 + ahead];
  if ((unsigned)page >= (unsigned)p.n_pages) {
    if (threadIdx.x == 0) kv_report(p, UAD_KV_BAD_PAGE);
    return;
  }
  const bool joins = first < p0;   // earlier tokens are in the block
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int items = 1 << a.log_items, per_pass = ITEMS > 1 ? 1 : kThreads >> a.log_items;
  const int mine = ITEMS > 1 ? threadIdx.x : threadIdx.x & (items - 1), at_once = ITEMS > 1 ? 0 : threadIdx.x >> a.log_items;
  const int c = mine & ((1 << a.log_chunks) - 1), half = a.rot / 2, lo = c * 8;
  const bool turn = !is_v && lo < half, twice = !is_v && a.rot > 0;
  const int e_lo = turn ? lo : c * kItem, e_hi = turn ? lo + half : c * kItem + 8;
  const int warps = ITEMS > 1 ? kWarps : items >> 5, warp0 = warp & ~(warps - 1);   // those of this thread's head
  int pos[ITEMS];
  bool fresh[ITEMS], old[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int j = (i * kThreads + mine) >> a.log_chunks;
    pos[i] = first + j;
    fresh[i] = j < slots && pos[i] >= p0 && pos[i] < s.len;
    old[i] = pos[i] < p0;
  }
  float cs[8], sn[8];
  if (ITEMS == 1 && turn && fresh[0])
#pragma unroll
    for (int i = 0; i < 8; ++i) rotation((uint32_t)pos[0], rope.turn[lo + i], cs + i, sn + i);
  char* const pool = static_cast<char*>(is_v ? p.v : p.k) + page * p.page_stride + lo_slot * p.slot_stride;
  float* const scales = (is_v ? a.sc.v : a.sc.k) + page * a.sc.page + sub * a.sc.block;
  const void* const from = is_v ? a.v : a.k;
  const int64_t from_stride = is_v ? a.v_stride : a.k_stride;
  int buf = 0;
  for (int h0 = group * per_pass; h0 < p.n_kv; h0 += a.kv_groups * per_pass) {
    const int h = h0 + at_once;
    const bool here = h < p.n_kv;
    float x[ITEMS][8], y[ITEMS][8];
    uint4 codes[ITEMS];
    float top = 0.f, before = 0.f;
    if (here) {
      if (joins) before = scales[h * a.sc.head];
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        if (fresh[i]) {
          const int64_t at = (s.first + (int64_t)(pos[i] - p0)) * from_stride + h * p.dh;
          load8<IN>(from, at + e_lo, x[i]);
          load8<IN>(from, at + e_hi, y[i]);
#pragma unroll
          for (int d = 0; d < 8; ++d) top = fmaxf(top, fmaxf(finite_abs(x[i][d]), finite_abs(y[i][d])));
        } else if (old[i]) {
          codes[i] = *reinterpret_cast<const uint4*>(pool + (pos[i] - first) * p.slot_stride + h * p.head_stride + c * kItem);
        }
      }
    }
    const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
    if (lane == 0) s_top[buf][warp] = most;
    __syncthreads();   // this buffer is written again after the next barrier
    uint32_t all = 0;
    for (int w = 0; w < warps; ++w) all = max(all, s_top[buf][warp0 + w]);
    buf ^= 1;
    if (!here) continue;
    float scale = scale_of(__uint_as_float(all), twice);
    if (joins) scale = fmaxf(scale, before);
    const bool exact = (__float_as_uint(scale) & 0x7fffffu) == 0;
    const float inv = 1.f / scale;
    if (mine == 0 && (!joins || scale != before)) scales[h * a.sc.head] = scale;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      char* const to = pool + (pos[i] - first) * p.slot_stride + h * p.head_stride;
      if (fresh[i]) {
        if (turn) {
          if constexpr (ITEMS > 1)
#pragma unroll
            for (int d = 0; d < 8; ++d) rotation((uint32_t)pos[i], rope.turn[lo + d], cs + d, sn + d);
#pragma unroll
          for (int d = 0; d < 8; ++d) {
            const float v = x[i][d] * cs[d] - y[i][d] * sn[d], w = y[i][d] * cs[d] + x[i][d] * sn[d];
            x[i][d] = v;
            y[i][d] = w;
          }
        }
        const uint2 r0 = round8(x[i], scale, inv, exact), r1 = round8(y[i], scale, inv, exact);
        if (turn) {
          *reinterpret_cast<uint2*>(to + e_lo) = r0;
          *reinterpret_cast<uint2*>(to + e_hi) = r1;
        } else {
          *reinterpret_cast<uint4*>(to + e_lo) = make_uint4(r0.x, r0.y, r1.x, r1.y);
        }
      } else if (old[i] && scale != before) {
        uint4 w = codes[i];
        w.x = rescale4(w.x, before, scale, inv, exact);
        w.y = rescale4(w.y, before, scale, inv, exact);
        w.z = rescale4(w.z, before, scale, inv, exact);
        w.w = rescale4(w.w, before, scale, inv, exact);
        *reinterpret_cast<uint4*>(to + c * kItem) = w;
      }
    }
  }
}

template <int IN>
cudaError_t launch_items(int items, dim3 grid, cudaStream_t s, const Append8Args& a, const uad_rope& r) {
  return items <= kThreads       ? launch_k(append8_kernel<IN, 1>, grid, kThreads, 0, s, a, r)
         : items == 2 * kThreads ? launch_k(append8_kernel<IN, 2>, grid, kThreads, 0, s, a, r)
                                 : launch_k(append8_kernel<IN, 4>, grid, kThreads, 0, s, a, r);
}

int log2_of(int n) {
  int l = 0;
  while ((1 << l) < n) ++l;
  return l;
}

}  // namespace

int uad::pages8_args(const uad_kv_pages8* g, const uad_kv_seqs* s, int n_rows, bool device, PagedArgs* p, Scales* sc) {
  if (!g || !g->k_scale || !g->v_scale) return UAD_EINVAL;
  if (g->block != 16 && g->block != 32 && g->block != 64) return UAD_EINVAL;
  if (g->scale_page_stride < 1 || g->scale_block_stride < 1 || g->scale_head_stride < 1) return UAD_EINVAL;
  if (reinterpret_cast<uintptr_t>(g->k_scale) % 4 || reinterpret_cast<uintptr_t>(g->v_scale) % 4) return UAD_EINVAL;
  const int rc = paged_args(&g->pages, s, n_rows, device, p, true);
  if (rc) return rc;
  sc->k = g->k_scale; sc->v = g->v_scale;
  sc->page = g->scale_page_stride; sc->block = g->scale_block_stride; sc->head = g->scale_head_stride;
  sc->log_block = log2_of(g->block);
  sc->per_page = FastDiv((uint32_t)((g->pages.page_size + g->block - 1) / g->block));
  return UAD_OK;
}

extern "C" int uad_kv_append8(const uad_kv_pages8* pages, const uad_kv_seqs* seqs, const uad_kv_rows* rows, const uad_rope* rope,
                              int32_t* status, void* stream) {
  if (!rows) return UAD_EINVAL;
  Append8Args a{};
  const int rc = pages8_args(pages, seqs, rows->n_rows, true, &a.p, &a.sc);
  if (rc) return rc;
  if (rows->dtype != UAD_DTYPE_F32 && rows->dtype != UAD_DTYPE_BF16) return UAD_EINVAL;
  const int es = rows->dtype == UAD_DTYPE_F32 ? 4 : 2;
  if (!rows->k != !rows->v || (!rows->q && !rows->k)) return UAD_EINVAL;
  if (rows->q ? rows->n_heads < 1 || rows->n_heads > 65536 || !rows->q_out : rows->n_heads != 0) return UAD_EINVAL;
  if (bad_address(rows->q, rows->q_stride, es) || bad_address(rows->k, rows->k_stride, es) || bad_address(rows->v, rows->v_stride, es) ||
      bad_address(rows->q_out, rows->q_out_stride, 2))
    return UAD_EINVAL;
  // in place, a thread writes the bytes that it has read: not where an element of the output has another size or place
  if (rows->q && rows->q == rows->q_out && (es != 2 || (rows->q_stride != rows->q_out_stride && rows->n_rows > 1))) return UAD_EINVAL;
  if (rope && (rope->dim < 16 || rope->dim > a.p.dh || rope->dim % 16)) return UAD_EINVAL;
  if (a.p.n_seqs == 0 || a.p.n_rows == 0) return UAD_OK;
  a.p.status = status;
  a.q = rows->q; a.k = rows->k; a.v = rows->v;
  a.q_stride = rows->q_stride; a.k_stride = rows->k_stride; a.v_stride = rows->v_stride;
  a.q_out = rows->q_out; a.q_out_stride = rows->q_out_stride;
  a.n_heads = rows->n_heads; a.rot = rope ? rope->dim : 0;
  const uad_rope none{};
  const int chunks = a.p.dh / kItem, block = pages->block, page = pages->pages.page_size, items = block * chunks;
  a.log_chunks = log2_of(chunks);
  a.log_items = log2_of(items);
  int64_t kv_blocks = 0, q_blocks = 0;
  if (a.k) {
    // the most blocks that max_new tokens in a row can touch
    const int64_t n = a.p.max_new, per_page = a.sc.per_page.d;
    const int64_t touched = page % block == 0 ? (n + block - 2) / block + 1 : (n - 1) / page * per_page + std::min<int64_t>(per_page + 1, (n - 1) % page + 1);
    // Heads of a CTA: those that it holds at once, and up to five times as many where that leaves the SMs eight CTAs: they
    // share sines and cosines.
    const int per_pass = std::max(1, kThreads / items), all = (a.p.n_kv + per_pass - 1) / per_pass;
    const int64_t ctas = std::min<int64_t>(touched * a.p.n_seqs, (int64_t)a.p.n_rows + a.p.n_seqs) * 2 * all;
    const int passes = (int)std::min<int64_t>({5, all, std::max<int64_t>(1, ctas / (152 * 8))});
    a.kv_groups = (all + passes - 1) / passes;
    a.by_group = FastDiv((uint32_t)(2 * a.kv_groups));
    kv_blocks = touched * 2 * a.kv_groups;
  }
  if (a.q) {
    const int64_t tokens = std::min<int64_t>((int64_t)a.p.max_new * a.p.n_seqs, a.p.n_rows);
    const int per = (int)std::min<int64_t>({5, a.n_heads, std::max<int64_t>(1, tokens * a.n_heads * chunks / (152 * 192))});
    a.groups = (a.n_heads + per - 1) / per;
    const int row_threads = a.groups * chunks, row_blocks = (row_threads + kThreads - 1) / kThreads;
    a.block_rows = row_threads < kThreads ? kThreads / row_threads : 1;
    a.row_threads = FastDiv((uint32_t)row_threads);
    a.row_blocks = FastDiv((uint32_t)row_blocks);
    q_blocks = ((int64_t)a.p.max_new + a.block_rows - 1) / a.block_rows * row_blocks;
  }
  if (kv_blocks + q_blocks > 0x7fffffff) return UAD_EINVAL;
  a.kv_blocks = (int)kv_blocks;
  const dim3 grid((unsigned)(kv_blocks + q_blocks), (unsigned)a.p.n_seqs);
  const uad_rope& r = rope ? *rope : none;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched(es == 4 ? launch_items<F32>(items, grid, s, a, r) : launch_items<BF16>(items, grid, s, a, r));
}
