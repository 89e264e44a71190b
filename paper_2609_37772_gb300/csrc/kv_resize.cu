// Bookkeeping of a paged cache on the GPU: from the lengths that sequences have and shall have, the pages they take from
// a ring of free ones or give back to it, their tables, first rows and slot maps.
#include "kv_pages.cuh"

#include <algorithm>

using namespace uad;

namespace {

constexpr int kThreads = 512, kOwn = 4, kChunk = kThreads * kOwn;   // sequences of a thread, of a chunk

struct ResizeArgs {
  int* table;
  const int* len;
  const int* want;
  int* len_out;
  int* start;
  int64_t* slot;
  int* row_seq;
  int* row_pos;
  int* ring;
  const int* state;
  int* state_out;
  int* status;
  int64_t table_stride;
  FastDiv page;
  int n_seqs, capacity, n_rows, n_pages;
  int fill, update;   // what this launch writes: tables, ring and rows; lengths and the ring's state
};

__device__ __forceinline__ int64_t shfl_up64(int64_t v, int d) { return __shfl_up_sync(0xffffffffu, v, d); }

// Exclusive sums over the block's threads of N values each, and the block's totals. s: [kThreads / 32][N].
template <int N>
__device__ __forceinline__ void block_scan(int64_t* v, int64_t* total, int64_t (*s)[N]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t mine[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    mine[i] = v[i];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t u = shfl_up64(v[i], d);
      if (lane >= d) v[i] += u;
    }
    if (lane == 31) s[warp][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
      const int64_t x = s[w][i];
      if (w < warp) before += x;
      all += x;
    }
    v[i] += before - mine[i];
    total[i] = all;
  }
}

// The last i with off[i] <= item: the owner of the item, where off are n exclusive sums and item is below their total.
__device__ __forceinline__ int owner_of(const int* off, int n, int item) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= item) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Sums over the sequences give everybody's place. A block holds the sums of 2048 sequences in shared memory, and every block works
// them out for itself, which takes it 1 to 2 us a chunk and spares an exchange. The items (pages taken, pages given back,
// rows) are then spread evenly over all blocks' threads, each finding its owner by bisection, so that one long sequence costs
// no more than many short ones.
__global__ void __launch_bounds__(kThreads) resize_kernel(const ResizeArgs a) {
  __shared__ int take_at[kChunk], give_at[kChunk], row_at[kChunk], had[kChunk], kept[kChunk];   // kept: pages that it shall have
  __shared__ int64_t sums[kThreads / 32][3], row_sums[kThreads / 32][1];
  __shared__ int taken_end;
  if (threadIdx.x == 0) taken_end = 0;
  pdl_wait();
  pdl_trigger();
  const bool lead = blockIdx.x == 0;
  const int first = a.state[0], n = a.n_pages;
  int count = a.state[1];
  const bool sound = first >= 0 && first < n && count >= 0 && count <= n;
  const int full = count;
  if (!sound) count = 0;
  const int room = sound ? n - count : 0;   // free places of the ring
  int64_t asked_pages = 0, asked_rows = 0, given = 0;   // of the chunks before
  int rows = 0, taken = 0;
  int report = sound ? 0 : UAD_KV_BAD_POOL;
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x, step = gridDim.x * kThreads;
  const auto on_ring = [&](uint32_t i) {   // i <= n places behind the first
    const uint32_t x = (uint32_t)first + i;
    return x >= (uint32_t)n ? x - n : x;
  };
  const auto pages_of = [&](int tokens) { return tokens > 0 ? (int)a.page.div(tokens - 1) + 1 : 0; };
  __syncthreads();   // taken_end; the state has been read
  for (int base = 0; base < a.n_seqs; base += kChunk) {
    int len[kOwn], want[kOwn];
    int64_t v[3] = {0, 0, 0}, total[3];   // pages to take, pages to give back, rows
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int b = base + threadIdx.x * kOwn + i;
      len[i] = want[i] = 0;
      if (b >= a.n_seqs) continue;
      len[i] = a.len[b];
      want[i] = a.want[b];
      if ((unsigned)len[i] > (unsigned)a.capacity || (unsigned)want[i] > (unsigned)a.capacity) {
        bad = true;
        want[i] = len[i];   // stays as it is
      }
      const int d = want[i] == len[i] ? 0 : pages_of(want[i]) - pages_of(len[i]);
      if (d > 0) v[0] += d;
      else v[1] -= d;
      if (want[i] > len[i]) v[2] += want[i] - len[i];
    }
    if (bad) report |= UAD_KV_BAD_SEQ;
    block_scan<3>(v, total, sums);   // its barrier: the chunk before has been read by all
    // Who is served: in order, as far as pages and rows go. The sums count everybody, so that behind one who is not served nobody
    // is who needs more of the same: the pages taken are the first ones without a gap.
    int64_t pages_end = asked_pages + v[0], back = given + v[1], rows_end = asked_rows + v[2];
    int64_t served[1] = {0}, all_served[1];
    bool ok[kOwn];
    int most = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int k = threadIdx.x * kOwn + i, add = want[i] - len[i];
      const int held = add ? pages_of(len[i]) : 0, need = add ? pages_of(want[i]) : 0;
      ok[i] = true;
      had[k] = len[i];
      kept[k] = need;
      take_at[k] = (int)min(pages_end, (int64_t)0x7fffffff);
      give_at[k] = (int)min(back, (int64_t)0x7fffffff);
      if (add > 0) {
        pages_end += need - held;
        rows_end += add;
        ok[i] = (need == held || pages_end <= count) && rows_end <= a.n_rows;
        if (!ok[i]) report |= UAD_KV_NO_ROOM;
        else served[0] += add;
        if (ok[i] && need > held) most = (int)pages_end;
      } else {
        back += held - need;
        if (back > room && held > need) report |= UAD_KV_BAD_POOL;
      }
    }
    most = (int)__reduce_max_sync(0xffffffffu, (unsigned)most);
    if (most && (threadIdx.x & 31) == 0) atomicMax(&taken_end, most);
    block_scan<1>(served, all_served, row_sums);
    int64_t at = rows + served[0];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int k = threadIdx.x * kOwn + i, b = base + k;
      row_at[k] = (int)at;
      if (b < a.n_seqs && lead) {
        if (a.fill) a.start[b] = (int)at;
        if (a.update) a.len_out[b] = ok[i] ? want[i] : len[i];
      }
      if (ok[i] && want[i] > len[i]) at += want[i] - len[i];
    }
    __syncthreads();   // places and taken_end
    const int m = min(kChunk, a.n_seqs - base), rows_to = rows + (int)all_served[0], taken_to = taken_end;
    const int given_from = (int)min(given, (int64_t)room), given_to = (int)min(given + total[1], (int64_t)room);
    if (a.fill) {
      for (uint32_t i = id; i < (uint32_t)(taken_to - taken); i += step) {
        const int t = taken + (int)i, k = owner_of(take_at, m, t);
        a.table[(base + k) * a.table_stride + pages_of(had[k]) + t - take_at[k]] = a.ring[on_ring(t)];
      }
      for (uint32_t i = id; i < (uint32_t)(given_to - given_from); i += step) {
        const int t = given_from + (int)i, k = owner_of(give_at, m, t);
        a.ring[on_ring(count + t)] = a.table[(base + k) * a.table_stride + kept[k] + t - give_at[k]];
      }
      if (a.slot || a.row_seq || a.row_pos) {
        for (uint32_t i = id; i < (uint32_t)(rows_to - rows); i += step) {
          const int r = rows + (int)i, k = owner_of(row_at, m, r), pos = had[k] + r - row_at[k];
          if (a.row_seq) a.row_seq[r] = base + k;
          if (a.row_pos) a.row_pos[r] = pos;
          if (!a.slot) continue;
          const int pi = (int)a.page.div(pos), held = pages_of(had[k]);
          const int page = pi < held ? a.table[(base + k) * a.table_stride + pi] : a.ring[on_ring(take_at[k] + pi - held)];
          const bool there = (unsigned)page < (unsigned)n;
          if (!there) report |= UAD_KV_BAD_PAGE;
          a.slot[r] = there ? (int64_t)page * a.page.d + (pos - pi * (int)a.page.d) : -1;
        }
      }
    }
    asked_pages += total[0];
    given += total[1];
    asked_rows += total[2];
    rows = rows_to;
    taken = taken_to;
  }
  if (a.fill) {
    if (a.slot || a.row_seq || a.row_pos) {   // rows of nobody
      for (uint32_t i = id; i < (uint32_t)(a.n_rows - rows); i += step) {
        const int r = rows + (int)i;
        if (a.slot) a.slot[r] = -1;
        if (a.row_seq) a.row_seq[r] = -1;
        if (a.row_pos) a.row_pos[r] = -1;
      }
    }
    if (lead && threadIdx.x == 0) a.start[a.n_seqs] = rows;
    // what the lengths say is every block's finding: one tells it
    if (!lead) report &= UAD_KV_BAD_PAGE;
    if (report && a.status) atomicOr(a.status, report);
  }
  if (a.update && lead && threadIdx.x == 0) {
    const int head = sound ? (int)on_ring(taken) : first, left = sound ? count - taken + (int)min(given, (int64_t)room) : full;
    a.state_out[0] = head;
    a.state_out[1] = left;
  }
}

}  // namespace

extern "C" int uad_kv_resize(const uad_page_pool* pool, const uad_kv_wanted* w, int32_t* status, void* stream) {
  if (!pool || !w || !pool->ring || !pool->state || !pool->state_out || pool->n_pages < 1 || pool->n_pages > (1 << 30)) return UAD_EINVAL;
  if (pool->page_size < 1 || pool->page_size > 65536) return UAD_EINVAL;
  if (w->n_seqs < 0 || w->n_seqs > 65535 || w->table_width < 1 || w->table_stride < w->table_width || w->n_rows < 0) return UAD_EINVAL;
  if ((int64_t)w->table_width * pool->page_size > (1ll << 31) - (1 << 17)) return UAD_EINVAL;
  if (!w->start || (w->n_seqs > 0 && (!w->table || !w->len || !w->want || !w->len_out))) return UAD_EINVAL;
  if (!on_current_device(pool->ring)) return UAD_EINVAL;
  ResizeArgs a{};
  a.table = w->table; a.len = w->len; a.want = w->want; a.len_out = w->len_out; a.start = w->start;
  a.slot = w->slot; a.row_seq = w->row_seq; a.row_pos = w->row_pos;
  a.ring = pool->ring; a.state = pool->state; a.state_out = pool->state_out; a.status = status;
  a.table_stride = w->table_stride;
  a.page = FastDiv((uint32_t)pool->page_size);
  a.n_seqs = w->n_seqs; a.capacity = w->table_width * pool->page_size; a.n_rows = w->n_rows; a.n_pages = pool->n_pages;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool maps = w->slot || w->row_seq || w->row_pos;
  const int blocks = std::max(1, std::min(152, maps ? (int)(((int64_t)w->n_rows + 2047) / 2048) : w->n_seqs / 64));
  // In place, blocks would read lengths or a state that another has already replaced: a launch of its own replaces them.
  const bool apart = blocks > 1 && (w->len_out == w->len || w->len_out == w->want || pool->state_out == pool->state);
  a.fill = 1;
  a.update = !apart;
  cudaError_t e = launch_k(resize_kernel, dim3(blocks), dim3(kThreads), 0, s, a);
  if (e == cudaSuccess && apart) {
    a.fill = 0;
    a.update = 1;
    e = launch_k(resize_kernel, dim3(1), dim3(kThreads), 0, s, a);
  }
  return launched(e);
}
