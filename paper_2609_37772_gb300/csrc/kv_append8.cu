// The append to a paged cache that is held in 8 bits: rotation, the blocks' scales, rounding to e4m3.
#include "kv_pages8.cuh"

#include <algorithm>

using namespace uad;

namespace {

constexpr int kMostThreads = 1024;   // of a CTA: 256 to 1024, a new token's 16 dimensions each

struct Append8Args {
  PagedArgs p;
  Scales sc;
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  void* q_out;
  int n_heads, rot, log_chunks;
  // keys and values: blocks of the grid's x that are theirs; groups of their heads
  int kv_blocks, kv_groups;
  FastDiv by_group;   // of a block's number into block of tokens and group of heads
  // queries
  int groups, block_rows;
  FastDiv row_threads, row_blocks;
};

constexpr uint32_t kInfinite = 0x7f800000u;   // bits of absolute values from here on are not finite
// The largest of eight absolute values and m, by their bits.
__device__ __forceinline__ uint32_t top_of(const float* x, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  return m;
}
// The same of those that are finite.
__device__ __forceinline__ uint32_t finite_top_of(const float* x, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = __float_as_uint(x[i]) & 0x7fffffffu;
    m = max(m, u < kInfinite ? u : 0);
  }
  return m;
}
// The least power of two that takes a value (twice: twice the value) to 448 or below, 2^-100 at the least. From its bits: 448 is 1.75 2^8.
__device__ __forceinline__ float scale_of(uint32_t u, bool twice) {
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u) + (twice ? 1 : 0);
  return __uint_as_float((uint32_t)max(e, 27) << 23);
}
// The least power of two that is no less (of a cache that was rounded elsewhere: this append's scales are powers of two).
__device__ __forceinline__ float power_above(float s) { return __uint_as_float((__float_as_uint(s) + 0x7fffffu) & 0xff800000u); }
// Two values as e4m3, the first one lower: nearest, ties to even; NaN stays.
__device__ __forceinline__ uint32_t e4m3_2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
// inv: one over the scale. bad: some of the thread's values are not finite; infinities become NaN.
__device__ __forceinline__ uint2 round8(const float* x, float inv, bool bad) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
  if (bad)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] += y[i] - y[i];
  return make_uint2(e4m3_2(y[0], y[1]) | e4m3_2(y[2], y[3]) << 16, e4m3_2(y[4], y[5]) | e4m3_2(y[6], y[7]) << 16);
}
// Four codes times f.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  const float2 a = e4m3_pair(w), b = e4m3_pair(w >> 16);
  return e4m3_2(a.x * f, a.y * f) | e4m3_2(b.x * f, b.y * f) << 16;
}

// The queries: one thread 16 dimensions of one row, in every a.groups-th of its heads, as in the append of the other types.
template <int IN>
__device__ __forceinline__ void rotate_queries(const Append8Args& a, const uad_rope& rope, const SeqRows& s, int block) {
  const int bj = a.row_blocks.div(block), tj = a.row_threads.div(threadIdx.x);
  if (tj >= a.block_rows) return;
  const int64_t j = (int64_t)bj * a.block_rows + tj;
  const int r = (block - bj * (int)a.row_blocks.d) * (int)blockDim.x + threadIdx.x - tj * (int)a.row_threads.d;
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

// Keys and values: a CTA has one block of tokens and some heads of the keys and of the values. A thread holds 16 dimensions of one
// new token, as 8 pairs where they are rotated; a head has as many threads as its new tokens need, rounded up to a power of two, and a
// CTA as many heads at a time as that leaves room for: a decoding step's single token takes 4 to 16 threads a head, a prompt's block
// all of them. The threads of a head find its largest value, which gives the scale before anything is rotated: a rotation grows no
// value by more than sqrt(2), so keys take twice the largest, and the scale does not hang on how sines round. Where the
// scale of a block with earlier tokens has grown, the head's threads round those again: exactly, as long as they stay normal numbers.
//
// Bound by memory for prompts: 64 ragged prompts of up to 816 tokens of 8 + 2 heads of 256 from fp32 rows take 66.7 us (5.8 TB/s, 87% of a
// copy's; as many tokens in prompts of one length 61.7), 64 x 300 tokens of 24 heads of 64 83 us (5.7 TB/s), a single token 3.3 us, of which a
// launch is 2.5. 64 registers, so that an SM holds 1024 threads: with the next head's values requested ahead of the barrier it
// is 768, and the queries, most of the bytes, take longer (82 us).
template <int IN>
__global__ void __launch_bounds__(kMostThreads, 1) append8_kernel(const Append8Args a, const __grid_constant__ uad_rope rope) {
  __shared__ uint32_t s_top[2][kMostThreads / 32];
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
  const int u = a.by_group.div(blockIdx.x), group = blockIdx.x - u * a.kv_groups, p0 = s.len - s.n;
  const int i0 = (int)p.page.div(p0), in_page = p0 - i0 * (int)p.page.d;
  const int number = (in_page >> a.sc.log_block) + u, ahead = (int)a.sc.per_page.div(number);
  const int sub = number - ahead * (int)a.sc.per_page.d, lo_slot = sub << a.sc.log_block;
  const int64_t first64 = (int64_t)(i0 + ahead) * p.page.d + lo_slot;
  if (first64 >= s.len) return;
  const int first = (int)first64, end = min(first + min(1 << a.sc.log_block, (int)p.page.d - lo_slot), s.len);
  const int begin = max(first, p0), fresh = end - begin, old = begin - first;   // new tokens of the block, earlier ones
  const int log_lanes = (fresh > 1 ? 32 - __clz(fresh - 1) : 0) + a.log_chunks, lanes = 1 << log_lanes;   // of a head
  const int per_pass = (int)blockDim.x >> log_lanes, heads = 2 * p.n_kv;   // the keys', then the values'
  if (group * per_pass >= heads) return;
  const int page = p.table[b * p.table_stride + i0 + ahead];
  const int warp = threadIdx.x >> 5, mine = threadIdx.x & (lanes - 1), at_once = threadIdx.x >> log_lanes;
  const int c = mine & ((1 << a.log_chunks) - 1), half = a.rot / 2, lo = c * 8;
  const int token = mine >> a.log_chunks;   // of the new ones
  const int64_t row = s.first + (int64_t)(begin - p0 + token);
  const auto load = [&](int h, float* x, float* y) {
    if (h >= heads || token >= fresh) return;
    const bool is_v = h >= p.n_kv, turn = !is_v && lo < half;
    const int64_t at = is_v ? row * a.v_stride + (h - p.n_kv) * p.dh : row * a.k_stride + h * p.dh;
    const void* from = is_v ? a.v : a.k;
    load8<IN>(from, at + (turn ? lo : c * kItem), x);
    load8<IN>(from, at + (turn ? lo + half : c * kItem + 8), y);
  };
  float x[8], y[8];
  load(group * per_pass + at_once, x, y);
  if ((unsigned)page >= (unsigned)p.n_pages) {
    if (threadIdx.x == 0) kv_report(p, UAD_KV_BAD_PAGE);
    return;
  }
  float cs[8], sn[8];
  if (lo < half && token < fresh && group * per_pass < p.n_kv)
#pragma unroll
    for (int i = 0; i < 8; ++i) rotation((uint32_t)(begin + token), rope.turn[lo + i], cs + i, sn + i);
  const int64_t place = page * p.page_stride + lo_slot * p.slot_stride, scale_place = page * a.sc.page + sub * a.sc.block;
  int buf = 0;
  for (int h0 = group * per_pass; h0 < heads; h0 += a.kv_groups * per_pass) {
    const int hh = h0 + at_once;
    const bool here = hh < heads, is_v = hh >= p.n_kv, turn = !is_v && lo < half, mover = here && token < fresh;
    const int h = is_v ? hh - p.n_kv : hh;
    float* const held = (is_v ? a.sc.v : a.sc.k) + scale_place + h * a.sc.head;
    uint32_t most = 0;
    bool bad = false;
    float before = 0.f;
    if (here && old && (lanes > 32 || mine == 0)) before = *held;   // read by all before the barrier, or by the one that writes it
    if (mover) {
      most = top_of(y, top_of(x, 0));
      bad = most >= kInfinite;
      if (bad) most = finite_top_of(y, finite_top_of(x, 0));
      if (turn)
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          const float v = x[d] * cs[d] - y[d] * sn[d], w = y[d] * cs[d] + x[d] * sn[d];
          x[d] = v;
          y[d] = w;
        }
    }
    if (lanes < 32) {
      for (int d = lanes / 2; d > 0; d /= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
    } else {
      most = __reduce_max_sync(0xffffffffu, most);
    }
    if (lanes <= 32) {
      before = __shfl_sync(0xffffffffu, before, threadIdx.x & 31 & ~(lanes - 1));
    } else {
      if ((threadIdx.x & 31) == 0) s_top[buf][warp] = most;
      __syncthreads();   // this buffer is written again after the next barrier
      const int warp0 = warp & ~(lanes / 32 - 1);
      for (int w = 0; w < lanes / 32; ++w) most = max(most, s_top[buf][warp0 + w]);
      buf ^= 1;
    }
    if (here) {
      float scale = scale_of(most, !is_v && a.rot > 0);
      if (old) scale = fmaxf(scale, power_above(before));
      const float inv = __uint_as_float((254u << 23) - __float_as_uint(scale));   // a power of two as well
      char* const head = static_cast<char*>(is_v ? p.v : p.k) + place + h * p.head_stride;
      if (mover) {
        const uint2 r0 = round8(x, inv, bad), r1 = round8(y, inv, bad);
        char* const to = head + (old + token) * p.slot_stride;
        if (turn) {
          *reinterpret_cast<uint2*>(to + lo) = r0;
          *reinterpret_cast<uint2*>(to + lo + half) = r1;
        } else {
          *reinterpret_cast<uint4*>(to + c * kItem) = make_uint4(r0.x, r0.y, r1.x, r1.y);
        }
      }
      if (!old || scale != before) {
        for (int i = mine; i < old << a.log_chunks; i += lanes) {
          uint4* const at = reinterpret_cast<uint4*>(head + (i >> a.log_chunks) * p.slot_stride + c * kItem);
          uint4 w = *at;
          w.x = rescale4(w.x, before * inv);
          w.y = rescale4(w.y, before * inv);
          w.z = rescale4(w.z, before * inv);
          w.w = rescale4(w.w, before * inv);
          *at = w;
        }
        if (mine == 0) *held = scale;
      }
    }
    load(hh + a.kv_groups * per_pass, x, y);
  }
}

// One block a token: 16 codes a thread, keys and values in turn.
__global__ void __launch_bounds__(256) gather8_kernel(const PagedArgs p, const Scales sc, const int* table, float* k, float* v) {
  pdl_wait();
  pdl_trigger();
  const int per_head = p.dh / 16, all = p.n_kv * per_head, i0 = (int)p.page.div(blockIdx.x), page = table[i0];
  if ((unsigned)page >= (unsigned)p.n_pages) return;
  const int slot = blockIdx.x - i0 * (int)p.page.d;
  for (int i = threadIdx.x; i < 2 * all; i += blockDim.x) {
    const bool is_v = i >= all;
    const int r = is_v ? i - all : i, h = r / per_head;
    const char* from = static_cast<const char*>(is_v ? p.v : p.k) + page * p.page_stride + slot * p.slot_stride + h * p.head_stride + (r - h * per_head) * 16;
    const float s = (is_v ? sc.v : sc.k)[page * sc.page + (slot >> sc.log_block) * sc.block + h * sc.head];
    const uint4 w = *reinterpret_cast<const uint4*>(from);
    float4* to = reinterpret_cast<float4*>((is_v ? v : k) + ((int64_t)blockIdx.x * all + r) * 16);
    const uint32_t c[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 a = e4m3_pair(c[j]), b = e4m3_pair(c[j] >> 16);
      to[j] = make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
    }
  }
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
  if (device && s->n_seqs > 0 && n_rows > 0 && (!on_current_device(g->k_scale) || !on_current_device(g->v_scale))) return UAD_EINVAL;
  sc->k = g->k_scale; sc->v = g->v_scale;
  sc->page = g->scale_page_stride; sc->block = g->scale_block_stride; sc->head = g->scale_head_stride;
  sc->log_block = log2_of(g->block);
  sc->per_page = FastDiv((uint32_t)((g->pages.page_size + g->block - 1) / g->block));
  return UAD_OK;
}

cudaError_t uad::launch_kv_gather8(const PagedArgs& p, const Scales& sc, const int* table, int n, void* k, void* v, cudaStream_t s) {
  return launch_k(gather8_kernel, dim3((unsigned)n), 256, 0, s, p, sc, table, static_cast<float*>(k), static_cast<float*>(v));
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
  const int chunks = a.p.dh / kItem, block = pages->block, page = pages->pages.page_size;
  // a head's threads: those of the most new tokens that a block gets
  const int lanes = (1 << log2_of(std::min({a.p.max_new, block, page}))) * chunks, threads = std::max(lanes, 256);
  a.log_chunks = log2_of(chunks);
  int64_t kv_blocks = 0, q_blocks = 0;
  if (a.k) {
    // the most blocks that max_new tokens in a row can touch
    const int64_t n = a.p.max_new, per_page = a.sc.per_page.d;
    const int64_t touched = page % block == 0 ? (n + block - 2) / block + 1 : (n - 1) / page * per_page + std::min<int64_t>(per_page + 1, (n - 1) % page + 1);
    // Heads of a CTA: those that it holds at once, and up to five times as many where that leaves the SMs eight CTAs: they
    // share sines and cosines.
    const int per_pass = threads / lanes, all = (2 * a.p.n_kv + per_pass - 1) / per_pass;
    const int64_t ctas = std::min<int64_t>(touched * a.p.n_seqs, (int64_t)a.p.n_rows + a.p.n_seqs) * all;
    const int passes = (int)std::min<int64_t>({5, all, std::max<int64_t>(1, ctas * threads / (152 * 2048))});
    a.kv_groups = (all + passes - 1) / passes;
    a.by_group = FastDiv((uint32_t)a.kv_groups);
    kv_blocks = touched * a.kv_groups;
  }
  if (a.q) {
    const int64_t tokens = std::min<int64_t>((int64_t)a.p.max_new * a.p.n_seqs, a.p.n_rows);
    const int per = (int)std::min<int64_t>({5, a.n_heads, std::max<int64_t>(1, tokens * a.n_heads * chunks / (152 * 192))});
    a.groups = (a.n_heads + per - 1) / per;
    const int row_threads = a.groups * chunks, row_blocks = (row_threads + threads - 1) / threads;
    a.block_rows = row_threads < threads ? threads / row_threads : 1;
    a.row_threads = FastDiv((uint32_t)row_threads);
    a.row_blocks = FastDiv((uint32_t)row_blocks);
    q_blocks = ((int64_t)a.p.max_new + a.block_rows - 1) / a.block_rows * row_blocks;
  }
  if (kv_blocks + q_blocks > 0x7fffffff) return UAD_EINVAL;
  a.kv_blocks = (int)kv_blocks;
  const dim3 grid((unsigned)(kv_blocks + q_blocks), (unsigned)a.p.n_seqs);
  const uad_rope& r = rope ? *rope : none;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched(es == 4 ? launch_k(append8_kernel<F32>, grid, dim3(threads), 0, s, a, r) : launch_k(append8_kernel<BF16>, grid, dim3(threads), 0, s, a, r));
}
