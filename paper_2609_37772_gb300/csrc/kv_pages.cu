// The paged key-value cache: argument checks, the rotation's frequencies and the append of new tokens.
#include "kv_pages.cuh"

#include <algorithm>
#include <cmath>

using namespace uad;

namespace {

struct AppendArgs {
  PagedArgs p;
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  void* q_out;
  int n_heads, rot, groups, log_chunks, block_rows;
  FastDiv row_threads, row_blocks;   // threads of a row, blocks of a row
};

// One thread: a chunk of 16 dimensions (8 pairs) of one row, in every a.groups-th of its heads. Eight sines and cosines cost
// about as many cycles as 150 bytes of memory, so that with one head a thread they bound the kernel; they depend on the
// position alone. 4 blocks an SM is what the registers hold without spilling (63): 52224 ragged tokens of 8 + 2 heads of
// 256 from fp32 rows take 64 us (92% of the bandwidth of a copy).
template <int IN, int CACHE>
__global__ void __launch_bounds__(256, 4) append_kernel(const AppendArgs a, const __grid_constant__ uad_rope rope) {
  pdl_wait();
  pdl_trigger();
  const PagedArgs& p = a.p;
  const int b = blockIdx.y;
  const SeqRows s = seq_rows(p, b);
  if (s.n < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) kv_report(p, UAD_KV_BAD_SEQ);
    return;
  }
  const int bj = a.row_blocks.div(blockIdx.x), tj = a.row_threads.div(threadIdx.x);
  if (tj >= a.block_rows) return;
  const int64_t j = (int64_t)bj * a.block_rows + tj;
  const int r = (blockIdx.x - bj * (int)a.row_blocks.d) * (int)blockDim.x + threadIdx.x - tj * (int)a.row_threads.d;
  if (j >= s.n || r >= (int)a.row_threads.d) return;
  const int group = r >> a.log_chunks, c = r - (group << a.log_chunks);
  const int64_t row = s.first + j;
  const int pos = s.len - s.n + (int)j, heads = a.n_heads + (a.k ? 2 * p.n_kv : 0);
  int64_t slot = 0;
  if (a.k) {
    slot = token_at(p, p.table + b * p.table_stride, pos);
    if (slot < 0) kv_report(p, UAD_KV_BAD_PAGE);
  }
  const int half = a.rot / 2, lo = c * 8;
  const bool turned = lo < half;
  float cs[8], sn[8], x[8], y[8];
  void* to = nullptr;
  bool turn = false;
  int e_lo = 0, e_hi = 0;
  const auto load = [&](int h) {
    const int kv = h - a.n_heads, v = kv - p.n_kv;
    to = nullptr;
    if (kv >= 0 && slot < 0) return;
    turn = turned && v < 0;
    // pairs (lo + i, hi + i); past the rotated dimensions, 16 neighbours
    e_lo = turn ? lo : c * kItem;
    e_hi = turn ? lo + half : c * kItem + 8;
    const void* from = kv < 0 ? a.q : v < 0 ? a.k : a.v;
    const int64_t src = kv < 0 ? row * a.q_stride + (int64_t)h * p.dh : v < 0 ? row * a.k_stride + kv * p.dh : row * a.v_stride + v * p.dh;
    const int64_t dst = kv < 0 ? row * a.q_out_stride + (int64_t)h * p.dh : slot + (v < 0 ? kv : v) * p.head_stride;
    to = static_cast<char*>(kv < 0 ? a.q_out : v < 0 ? p.k : p.v) + dst * (CACHE == F32 ? 4 : 2);
    load8<IN>(from, src + e_lo, x);
    load8<IN>(from, src + e_hi, y);
  };
  load(group);
  if (turned)
#pragma unroll
    for (int i = 0; i < 8; ++i) rotation((uint32_t)pos, rope.turn[lo + i], cs + i, sn + i);
  for (int head = group;;) {
    if (to) {
      if (turn)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float u = x[i] * cs[i] - y[i] * sn[i], w = y[i] * cs[i] + x[i] * sn[i];
          x[i] = u;
          y[i] = w;
        }
      store8<CACHE>(to, e_lo, x);
      store8<CACHE>(to, e_hi, y);
    }
    head += a.groups;
    if (head >= heads) break;
    load(head);
  }
}

// One block a token: a copy in 16-byte pieces, keys and values in turn.
__global__ void __launch_bounds__(256) gather_kernel(const PagedArgs p, const int* table, char* k, char* v) {
  pdl_wait();
  pdl_trigger();
  const int es = p.dtype == F32 ? 4 : 2, per_head = p.dh * es / 16, all = p.n_kv * per_head;
  const int64_t at = token_at(p, table, blockIdx.x);
  if (at < 0) return;
  for (int i = threadIdx.x; i < 2 * all; i += blockDim.x) {
    const bool is_v = i >= all;
    const int r = is_v ? i - all : i, h = r / per_head;
    const char* from = static_cast<const char*>(is_v ? p.v : p.k) + (at + h * p.head_stride) * es + (r - h * per_head) * 16;
    *reinterpret_cast<uint4*>((is_v ? v : k) + ((int64_t)blockIdx.x * all + r) * 16) = *reinterpret_cast<const uint4*>(from);
  }
}

}  // namespace

bool uad::on_current_device(const void* p) {
  int dev = 0;
  cudaPointerAttributes at{};
  if (cudaGetDevice(&dev) != cudaSuccess || cudaPointerGetAttributes(&at, p) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return (at.type == cudaMemoryTypeDevice && at.device == dev) || at.type == cudaMemoryTypeManaged;
}

cudaError_t uad::launch_kv_gather(const PagedArgs& p, const int* table, int n, void* k, void* v, cudaStream_t s) {
  return launch_k(gather_kernel, dim3((unsigned)n), 256, 0, s, p, table, static_cast<char*>(k), static_cast<char*>(v));
}

int uad::paged_args(const uad_kv_pages* g, const uad_kv_seqs* s, int n_rows, bool device, PagedArgs* p, bool eight) {
  if (!g || !s || !g->k || !g->v) return UAD_EINVAL;
  if (eight ? g->dtype != UAD_DTYPE_E4M3 : g->dtype != UAD_DTYPE_F32 && g->dtype != UAD_DTYPE_BF16) return UAD_EINVAL;
  const int es = eight ? 1 : g->dtype == UAD_DTYPE_F32 ? 4 : 2;
  if (g->head_dim != 64 && g->head_dim != 128 && g->head_dim != 256) return UAD_EINVAL;
  if (g->n_pages < 1 || g->page_size < 1 || g->page_size > 65536 || g->n_kv_heads < 1 || g->n_kv_heads > 1024) return UAD_EINVAL;
  if (g->page_stride < 1 || g->slot_stride < 1 || g->head_stride < 1) return UAD_EINVAL;
  if (bad_address(g->k, g->page_stride, es) || bad_address(g->v, g->slot_stride, es) || bad_address(nullptr, g->head_stride, es))
    return UAD_EINVAL;
  if (s->n_seqs < 0 || s->n_seqs > 65535 || s->max_new < 1 || s->max_len < 0 || s->table_width < 1) return UAD_EINVAL;
  if ((int64_t)s->table_width * g->page_size > (1ll << 31) - (1 << 17) || s->table_stride < s->table_width) return UAD_EINVAL;
  if (n_rows < 0 || (!s->start && n_rows < s->n_seqs)) return UAD_EINVAL;
  if (device && s->n_seqs > 0 && n_rows > 0) {
    if (!s->table || !s->len) return UAD_EINVAL;
    if (!on_current_device(g->k) || !on_current_device(g->v)) return UAD_EINVAL;
  }
  p->k = g->k; p->v = g->v;
  p->page_stride = g->page_stride; p->slot_stride = g->slot_stride; p->head_stride = g->head_stride;
  p->table = s->table; p->len = s->len; p->start = s->start; p->table_stride = s->table_stride;
  p->page = FastDiv((uint32_t)g->page_size);
  p->n_pages = g->n_pages; p->n_kv = g->n_kv_heads; p->dh = g->head_dim; p->dtype = eight ? E4M3 : g->dtype == UAD_DTYPE_F32 ? F32 : BF16;
  p->n_seqs = s->n_seqs; p->n_rows = n_rows; p->max_new = s->max_new < n_rows ? s->max_new : (n_rows > 0 ? n_rows : 1);
  p->capacity = s->table_width * g->page_size;
  return UAD_OK;
}

extern "C" {

int uad_rope_init(double theta, int32_t dim, uad_rope* out) {
  if (!out || dim < 16 || dim > 256 || dim % 16 || !(theta > 0) || !std::isfinite(theta)) return UAD_EINVAL;
  *out = uad_rope{};
  out->dim = dim;
  for (int i = 0; i < dim / 2; ++i) {
    // turns a position; whole ones drop out. In long double (64 bits of mantissa and more): a double's last bit is
    // 2e-7 rad of the first angles at 2^31 tokens
    const long double t = std::pow((long double)theta, -2.0L * i / dim) * 0.159154943091895335768883763372514362L;
    out->turn[i] = (uint64_t)std::ldexp(t - std::floor(t), 64);
  }
  return UAD_OK;
}

int uad_kv_append(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_kv_rows* rows, const uad_rope* rope,
                  int32_t* status, void* stream) {
  if (!rows) return UAD_EINVAL;
  AppendArgs a{};
  const int rc = paged_args(pages, seqs, rows->n_rows, true, &a.p);
  if (rc) return rc;
  if (rows->dtype != UAD_DTYPE_F32 && rows->dtype != UAD_DTYPE_BF16) return UAD_EINVAL;
  const int es = rows->dtype == UAD_DTYPE_F32 ? 4 : 2, ces = a.p.dtype == F32 ? 4 : 2;
  if (!rows->k != !rows->v || (!rows->q && !rows->k)) return UAD_EINVAL;
  if (rows->q ? rows->n_heads < 1 || rows->n_heads > 65536 || !rows->q_out : rows->n_heads != 0) return UAD_EINVAL;
  if (bad_address(rows->q, rows->q_stride, es) || bad_address(rows->k, rows->k_stride, es) || bad_address(rows->v, rows->v_stride, es) ||
      bad_address(rows->q_out, rows->q_out_stride, ces))
    return UAD_EINVAL;
  // in place, a thread writes the bytes that it has read: not where an element of the output has another size or place
  if (rows->q && rows->q == rows->q_out && (es != ces || (rows->q_stride != rows->q_out_stride && rows->n_rows > 1))) return UAD_EINVAL;
  if (rope && (rope->dim < 16 || rope->dim > a.p.dh || rope->dim % 16)) return UAD_EINVAL;
  if (a.p.n_seqs == 0 || a.p.n_rows == 0) return UAD_OK;
  a.p.status = status;
  a.q = rows->q; a.k = rows->k; a.v = rows->v;
  a.q_stride = rows->q_stride; a.k_stride = rows->k_stride; a.v_stride = rows->v_stride;
  a.q_out = rows->q_out; a.q_out_stride = rows->q_out_stride;
  a.n_heads = rows->n_heads; a.rot = rope ? rope->dim : 0;
  const uad_rope none{};
  const int heads = a.n_heads + (a.k ? 2 * a.p.n_kv : 0), chunks = a.p.dh / kItem;
  while ((1 << a.log_chunks) < chunks) ++a.log_chunks;
  const int64_t tokens = std::min<int64_t>((int64_t)a.p.max_new * a.p.n_seqs, a.p.n_rows);
  const int64_t items = tokens * heads * chunks;
  // Heads a thread: one where that leaves the SMs six warps or fewer (latency bounds: 3.4 us against 4.3 of
  // two groups for 64 tokens of 10 heads of 256), up to five beyond, which share the angles' cosines and sines (1024 such
  // tokens: 5.4 us against 8.2; 52224: 64 against 173). More do not pay: eight take 41 us where five take 35 (52224 tokens of
  // 8 heads of 64, fp32) and 219 against 230 (48 heads of 128).
  const int per = (int)std::min<int64_t>({5, heads, std::max<int64_t>(1, items / (152 * 192))});
  a.groups = (heads + per - 1) / per;
  const int row_threads = a.groups * chunks, row_blocks = (row_threads + 255) / 256;
  a.block_rows = row_threads < 256 ? 256 / row_threads : 1;
  a.row_threads = FastDiv((uint32_t)row_threads);
  a.row_blocks = FastDiv((uint32_t)row_blocks);
  const int64_t blocks = ((int64_t)a.p.max_new + a.block_rows - 1) / a.block_rows * row_blocks;
  if (blocks > 0x7fffffff) return UAD_EINVAL;
  const dim3 grid((unsigned)blocks, (unsigned)a.p.n_seqs);
  const uad_rope& r = rope ? *rope : none;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool in32 = rows->dtype == UAD_DTYPE_F32, out32 = a.p.dtype == F32;
  const cudaError_t e = in32 ? (out32 ? launch_k(append_kernel<F32, F32>, grid, 256, 0, s, a, r) : launch_k(append_kernel<F32, BF16>, grid, 256, 0, s, a, r))
                             : (out32 ? launch_k(append_kernel<BF16, F32>, grid, 256, 0, s, a, r) : launch_k(append_kernel<BF16, BF16>, grid, 256, 0, s, a, r));
  return launched(e);
}

}  // extern "C"
