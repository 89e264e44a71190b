// Bookkeeping of a paged cache on the GPU: from the lengths that sequences have and shall have, the pages they take from
// a ring of free ones or give back to it, their tables, first rows and slot maps.
#include "kv_pages.cuh"

#include <algorithm>

using namespace uad;

namespace {

constexpr int kThreads = 1024, kOwn = 2, kChunk = kThreads * kOwn;   // the most of a block; sequences of a thread; the most of a chunk

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
  int settle;         // 1: the only block, which answers for what is given back; 0: a launch behind this one does
  int maps, wide;     // whether slot maps are wanted; whether they are 16-byte aligned
};

static_assert(kThreads == 1024, "a lane for each warp's total");
// Exclusive sums over the block's threads of N values each, and the block's totals. s: [kThreads / 32][N].
template <int N, typename T>
__device__ __forceinline__ void block_scan(T* v, T* total, T (*s)[N]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T mine[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    mine[i] = v[i];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const T u = __shfl_up_sync(0xffffffffu, v[i], d);
      if (lane >= d) v[i] += u;
    }
    if (lane == 31) s[warp][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {   // every warp sums the warps' totals up, lane w that of warp w
    const T own = lane < (int)blockDim.x / 32 ? s[lane][i] : 0;
    T upto = own;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const T u = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += u;
    }
    v[i] += __shfl_sync(0xffffffffu, upto - own, warp) - mine[i];
    total[i] = __shfl_sync(0xffffffffu, upto, 31);
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

// Four rows from r of which those from..to - 1 are written: slot, sequence, position.
struct Rows4 {
  int64_t slot[4];
  int seq[4], pos[4];
};
__device__ __forceinline__ void put_rows(const ResizeArgs& a, int r, int from, int to, const Rows4& x) {
  if (a.wide && from <= r && r <= to - 4) {   // r + 4 may pass 31 bits
    if (a.slot) {
      longlong2* at = reinterpret_cast<longlong2*>(a.slot + r);
      at[0] = make_longlong2(x.slot[0], x.slot[1]);
      at[1] = make_longlong2(x.slot[2], x.slot[3]);
    }
    if (a.row_seq) *reinterpret_cast<int4*>(a.row_seq + r) = make_int4(x.seq[0], x.seq[1], x.seq[2], x.seq[3]);
    if (a.row_pos) *reinterpret_cast<int4*>(a.row_pos + r) = make_int4(x.pos[0], x.pos[1], x.pos[2], x.pos[3]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (r + i < from || r + i >= to) continue;
    if (a.slot) a.slot[r + i] = x.slot[i];
    if (a.row_seq) a.row_seq[r + i] = x.seq[i];
    if (a.row_pos) a.row_pos[r + i] = x.pos[i];
  }
}

// Sums over the sequences give everybody's place. A block holds the sums of 2048 sequences in shared memory, and every block works
// them out for itself, which spares an exchange. The items (pages taken, pages given back, rows in fours) are then spread evenly
// over all blocks' threads, each finding its owner by bisection, so that one long sequence costs no more than many short ones. T: what
// the sums of a chunk fit in.
// Places of a table that hold no page (an episode behind a window) do not come onto the ring when they are given back. The lengths do not tell of them, and
// there are none most of the time: pages given back are put onto the ring as if there were none, and where one is found (or they
// were more than fit) one block puts them there again, without gaps. Several blocks leave that to a second launch of one, which reads what they have put
// (1.5 us, and 3 more for 88000 pages given back; a cluster of eight takes 2.8 and 5 in all).
// A decoding step of 64 sequences takes 5.7 us, a launch and two rounds of dependent loads; 4000 sequences of which 2800 get 1 to 816 tokens 19 us
// (26 MB of slot maps, 1.3 TB/s): sums of two chunks, then the rows, at 0.6 instructions a cycle and scheduler, 16 us; then the second launch.
template <typename T>
__global__ void __launch_bounds__(kThreads) resize_kernel(const ResizeArgs a) {
  __shared__ int take_at[kChunk], give_at[kChunk], row_at[kChunk], had[kChunk], kept[kChunk];   // kept: pages that it shall have
  __shared__ T sums[kThreads / 32][3], row_sums[kThreads / 32][1];
  __shared__ int taken_here;
  constexpr int64_t most_of_t = sizeof(T) == 4 ? 0x7fffffff : 0x7fffffffffffffff;
  const auto clip = [](T x) { return sizeof(T) == 4 ? (int)x : (int)min((int64_t)x, (int64_t)0x7fffffff); };
  pdl_wait();
  pdl_trigger();
  int len[kOwn], want[kOwn];
  const auto load = [&](int base) {
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int b = base + threadIdx.x * kOwn + i;
      len[i] = b < a.n_seqs ? a.len[b] : 0;
      want[i] = b < a.n_seqs ? a.want[b] : 0;
    }
  };
  load(0);
  const bool lead = blockIdx.x == 0;
  const int first = a.state[0], n = a.n_pages, full = a.state[1];
  const bool sound = first >= 0 && first < n && full >= 0 && full <= n;
  const int count = sound ? full : 0, room = sound ? n - full : 0;   // pages, and free places of the ring
  int64_t asked_pages = 0, asked_rows = 0, given = 0;   // of the chunks before
  int rows = 0, taken = 0, placed = 0;                  // placed: of those given back, the pages on the ring (settle)
  int report = sound ? 0 : UAD_KV_BAD_POOL;
  const int chunk = (int)blockDim.x * kOwn;
  // Chunks are worked out by every block in turn, and filled in by a share of the blocks each, at about the same time.
  const uint32_t shares = min((a.n_seqs + chunk - 1) / chunk, (int)gridDim.x), share = shares > 1 ? blockIdx.x % shares : 0;
  const uint32_t id = (shares > 1 ? blockIdx.x / shares : blockIdx.x) * blockDim.x + threadIdx.x;
  const uint32_t step = (shares > 1 ? (gridDim.x - share + shares - 1) / shares : gridDim.x) * blockDim.x;
  const auto on_ring = [&](uint32_t i) {   // i <= n places behind the first
    const uint32_t x = (uint32_t)first + i;
    return x >= (uint32_t)n ? x - n : x;
  };
  // Whether one of the n_put entries `from` places behind the first is no page, of those that this thread reads.
  const auto no_page = [&](int from, int n_put) {
    unsigned most = 0;
    for (int at = (int)on_ring((uint32_t)from); n_put > 0; at = 0) {   // to the ring's end, then from its beginning
      const int run = min(n_put, n - at), *p = a.ring + at, skip = min(run, (int)(-(reinterpret_cast<uintptr_t>(p) / 4) & 3)), fours = (run - skip) / 4;
      const int ends = run - 4 * fours;   // before and behind them, 6 at the most
      if ((int)threadIdx.x < ends) most = max(most, (unsigned)p[(int)threadIdx.x < skip ? threadIdx.x : 4 * fours + threadIdx.x]);
      const int4* p4 = reinterpret_cast<const int4*>(p + skip);
      for (int i0 = threadIdx.x; i0 < fours; i0 += 8 * (int)blockDim.x) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = i0 + j * (int)blockDim.x;
          if (i < fours) {
            const int4 x = p4[i];
            most = max(max(most, max((unsigned)x.x, (unsigned)x.y)), max((unsigned)x.z, (unsigned)x.w));
          }
        }
      }
      n_put -= run;
    }
    return most >= (unsigned)n;
  };
  const auto pages_of = [&](int tokens) { return tokens > 0 ? (int)a.page.div(tokens - 1) + 1 : 0; };
  if (a.n_seqs == 0) __syncthreads();   // the state has been read
  if (a.settle && !a.fill && !a.update) {   // the launch before has written its state: is it right?
    const int head = a.state_out[0], left = a.state_out[1];
    if (!sound) return;
    if (head >= 0) {   // everything had a place
      const int gone = head >= first ? head - first : head - first + n, put = room > 0 ? left - count + gone : 0;
      if (!__syncthreads_or(no_page(count, put))) return;
    }
  }
  uint32_t turn = 0;
  for (int base = 0; base < a.n_seqs; base += chunk) {
    T v[3] = {0, 0, 0}, total[3];   // pages to take, pages to give back, rows
    int held[kOwn], need[kOwn];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      if ((unsigned)len[i] > (unsigned)a.capacity || (unsigned)want[i] > (unsigned)a.capacity) {
        bad = true;
        want[i] = len[i];   // stays as it is
      }
      const bool moves = want[i] != len[i];
      held[i] = moves ? pages_of(len[i]) : 0;
      need[i] = moves ? pages_of(want[i]) : 0;
      v[0] += max(need[i] - held[i], 0);
      v[1] += max(held[i] - need[i], 0);
      if (moves) v[2] += max(want[i] - len[i], 0);
    }
    if (bad) report |= UAD_KV_BAD_SEQ;
    block_scan<3, T>(v, total, sums);   // its barrier: the chunk before has been read by all
    // Who is served: in order, as far as pages and rows go. The sums count everybody, so that behind one who is not served nobody
    // is who needs more of the same: the pages taken are the first ones without a gap.
    // Places are counted from the chunk's beginning.
    const bool everybody = asked_pages + total[0] <= count && asked_rows + total[2] <= a.n_rows && asked_rows == rows;
    const T pages_left = (T)max(min(count - asked_pages, most_of_t), (int64_t)-1), rows_left = (T)max(min(a.n_rows - asked_rows, most_of_t), (int64_t)-1);
    T served[1] = {0}, all_served = total[2];
    bool ok[kOwn];
    int most = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int k = threadIdx.x * kOwn + i, add = want[i] == len[i] ? 0 : want[i] - len[i];
      ok[i] = true;
      had[k] = len[i];
      kept[k] = need[i];
      take_at[k] = clip(v[0]);
      give_at[k] = clip(v[1]);
      row_at[k] = clip(v[2]);   // where everybody is served
      v[0] += max(need[i] - held[i], 0);
      v[1] += max(held[i] - need[i], 0);
      v[2] += max(add, 0);
      if (add > 0 && !everybody) {
        ok[i] = (need[i] == held[i] || v[0] <= pages_left) && v[2] <= rows_left;
        if (!ok[i]) report |= UAD_KV_NO_ROOM;
        else served[0] += add;
        if (ok[i] && need[i] > held[i]) most = (int)v[0];
      }
    }
    if (!everybody) {   // rows and pages once more, of those who are served
      most = (int)__reduce_max_sync(0xffffffffu, (unsigned)most);
      if (base > 0) __syncthreads();   // the chunk before has read it
      if (threadIdx.x == 0) taken_here = 0;
      __syncthreads();
      if ((threadIdx.x & 31) == 0) atomicMax(&taken_here, most);
      T all[1];
      block_scan<1, T>(served, all, row_sums);
      all_served = all[0];
      int at = (int)served[0];
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        row_at[threadIdx.x * kOwn + i] = at;
        if (ok[i] && want[i] > len[i]) at += want[i] - len[i];
      }
    }
    if (lead) {
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const int k = threadIdx.x * kOwn + i, b = base + k;
        if (b >= a.n_seqs) continue;
        if (a.fill) a.start[b] = rows + row_at[k];
        if (a.update) a.len_out[b] = ok[i] ? want[i] : len[i];
      }
    }
    __syncthreads();   // places and taken_here
    load(base + chunk);   // the next chunk, on its way meanwhile
    const int m = min(chunk, a.n_seqs - base), n_rows = (int)all_served, n_taken = everybody ? (int)total[0] : taken_here;
    // pages given back that are put behind those before as if all of them were pages
    const int put_at = a.settle ? placed : (int)min(given, (int64_t)room);
    const int n_given = (int)min((int64_t)total[1], (int64_t)(room - put_at));
    const auto given_page = [&](int i) {
      const int k = owner_of(give_at, m, i), page = a.table[(base + k) * a.table_stride + kept[k] + i - give_at[k]];
      if (page < -1 || page >= n) report |= UAD_KV_BAD_PAGE;
      return page;
    };
    bool odd = false;   // an entry of this thread's is no page
    if (a.fill && turn == share) {
      // Rows, pages taken and pages given back begin with different threads, so that few of each are worked on at the same time.
      for (uint32_t i = step - 1 - id; i < (uint32_t)n_taken; i += step) {
        const int k = owner_of(take_at, m, (int)i), page = a.ring[on_ring(taken + i)];
        a.table[(base + k) * a.table_stride + pages_of(had[k]) + (int)i - take_at[k]] = page;
        if ((unsigned)page >= (unsigned)n) report |= UAD_KV_BAD_PAGE;
      }
      for (uint32_t i = id < step / 2 ? id + step / 2 : id - step / 2; i < (uint32_t)n_given; i += step) {
        const int page = given_page((int)i);
        a.ring[on_ring((uint32_t)(count + put_at) + i)] = page;
        odd |= (unsigned)page >= (unsigned)n;
      }
      if (a.maps) {
        for (uint32_t i = (uint32_t)rows / 4 + id; i < ((uint32_t)(rows + n_rows) + 3) / 4; i += step) {
          const int r0 = (int)i * 4, begin = max(r0, rows);
          int k = owner_of(row_at, m, begin - rows), last = -1, page = 0;
          Rows4 x;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int r = r0 + j - rows;
            if (r < 0 || r >= n_rows) continue;
            if (k + 1 < m && row_at[k + 1] <= r) {   // the next one, or behind a run of those without rows
              ++k;
              if (k + 1 < m && row_at[k + 1] <= r) k += 1 + owner_of(row_at + k + 1, m - k - 1, r);
              last = -1;
            }
            const int pos = had[k] + r - row_at[k], pi = (int)a.page.div(pos);
            if (a.slot && pi != last) {
              const int own = pages_of(had[k]);
              page = pi < own ? a.table[(base + k) * a.table_stride + pi] : a.ring[on_ring(taken + take_at[k] + pi - own)];
              last = pi;
              if ((unsigned)page >= (unsigned)n) report |= UAD_KV_BAD_PAGE;
            }
            x.seq[j] = base + k;
            x.pos[j] = pos;
            x.slot[j] = (unsigned)page < (unsigned)n ? (int64_t)page * a.page.d + (pos - pi * (int)a.page.d) : -1;
          }
          put_rows(a, r0, rows, rows + n_rows, x);
        }
      }
    }
    if (a.settle && sound && total[1] > 0) {
      bool again = (int64_t)total[1] > n_given || (!a.fill && placed != given);
      if (!again) again = __syncthreads_or(a.fill ? odd : no_page(count + placed, n_given));
      if (!again) {
        placed += n_given;
      } else {
        const uint32_t items = (uint32_t)min((int64_t)total[1], (int64_t)0x7fffffff);
        for (uint32_t i0 = 0; i0 < items; i0 += blockDim.x) {
          const uint32_t i = i0 + threadIdx.x;
          const int page = i < items ? given_page((int)i) : -1;
          const bool is = (unsigned)page < (unsigned)n;
          T at[1] = {is}, all[1];
          block_scan<1, T>(at, all, row_sums);
          if (is && at[0] < room - placed) a.ring[on_ring((uint32_t)(count + placed) + (uint32_t)at[0])] = page;
          if (all[0] > room - placed) report |= UAD_KV_BAD_POOL;
          placed = (int)min((int64_t)placed + all[0], (int64_t)room);
          __syncthreads();   // the sums have been read
        }
      }
    }
    turn = turn + 1 >= shares ? 0 : turn + 1;
    asked_pages += total[0];
    given += total[1];
    asked_rows += total[2];
    rows += n_rows;
    taken += n_taken;
  }
  if (a.fill) {
    if (a.maps) {   // rows of nobody
      const Rows4 none = {{-1, -1, -1, -1}, {-1, -1, -1, -1}, {-1, -1, -1, -1}};
      for (uint32_t i = (uint32_t)rows / 4 + blockIdx.x * blockDim.x + threadIdx.x; i < ((uint32_t)a.n_rows + 3) / 4; i += gridDim.x * blockDim.x) put_rows(a, (int)i * 4, rows, a.n_rows, none);
    }
    if (lead && threadIdx.x == 0) a.start[a.n_seqs] = rows;
  }
  // what the lengths say is every block's finding: one tells it
  if (!lead) report &= UAD_KV_BAD_PAGE;
  if (report && a.status) atomicOr(a.status, report);
  if ((a.update || a.settle) && lead && threadIdx.x == 0) {
    const int head = sound ? (int)on_ring(taken) : first, left = sound ? count - taken + (a.settle ? placed : (int)min(given, (int64_t)room)) : full;
    a.state_out[0] = !a.settle && sound && given > room ? -1 : head;   // -1: for the launch behind, which settles it
    a.state_out[1] = left;
  }
}

cudaError_t launch_resize(const ResizeArgs& a, int blocks, cudaStream_t s) {
  const int threads = blocks == 1 && a.n_seqs <= 512 && a.n_rows <= 1024 ? 256 : kThreads;   // a decoding step: fewer to wait for
  // sums of 2048 lengths below 2^20 stay within 31 bits
  return a.capacity < 1 << 20 ? launch_k(resize_kernel<int>, dim3(blocks), dim3(threads), 0, s, a)
                              : launch_k(resize_kernel<int64_t>, dim3(blocks), dim3(threads), 0, s, a);
}

}  // namespace

extern "C" int uad_kv_resize(const uad_page_pool* pool, const uad_kv_wanted* w, int32_t* status, void* stream) {
  if (!pool || !w || !pool->ring || !pool->state || !pool->state_out || pool->n_pages < 1 || pool->n_pages > (1 << 30)) return UAD_EINVAL;
  if (pool->page_size < 1 || pool->page_size > 65536) return UAD_EINVAL;
  if (w->n_seqs < 0 || w->n_seqs > 65535 || w->table_width < 1 || w->table_stride < w->table_width || w->n_rows < 0) return UAD_EINVAL;
  if ((int64_t)w->table_width * pool->page_size > (1ll << 31) - (1 << 17)) return UAD_EINVAL;
  if (!w->start || (w->n_seqs > 0 && (!w->table || !w->len || !w->want || !w->len_out))) return UAD_EINVAL;
  const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if ((at(pool->ring) | at(pool->state) | at(pool->state_out) | at(w->table) | at(w->len) | at(w->want) | at(w->len_out) | at(w->start) | at(w->row_seq) |
       at(w->row_pos) | at(status)) % 4 || at(w->slot) % 8)
    return UAD_EINVAL;
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
  a.maps = maps;
  a.wide = (reinterpret_cast<uintptr_t>(w->slot) | reinterpret_cast<uintptr_t>(w->row_seq) | reinterpret_cast<uintptr_t>(w->row_pos)) % 16 == 0;
  // Without maps, one block spares 128 to 255 sequences the second launch: a token more for 200 in place 6.6 us against 9.9 (4.1 against 5.5 not in
  // place), whole prompts 10.1 against 11.3 (7.3 against 6.4); for 500 prompts it is 15.1 against 11.1.
  const int blocks = std::max(1, std::min(152, maps ? (int)(((int64_t)w->n_rows + 4095) / 4096) : w->n_seqs < 256 ? 1 : w->n_seqs / 64));
  // In place, blocks would read lengths or a state that another has already replaced: the second launch replaces them.
  const bool apart = blocks > 1 && (w->len_out == w->len || w->len_out == w->want || pool->state_out == pool->state);
  a.fill = 1;
  a.update = !apart;
  a.settle = blocks == 1;
  cudaError_t e = launch_resize(a, blocks, s);
  if (e == cudaSuccess && blocks > 1) {
    a.fill = 0;
    a.update = apart;
    a.settle = 1;
    e = launch_resize(a, 1, s);
  }
  return launched(e);
}
