// The paged key-value cache's operators: what their kernels share (arguments as the kernels take them, the checks of
// what only the device knows, the place of a token).
#pragma once
#include <math.h>
#include <stdint.h>

#include "../../include/uad.h"
#include "fast_div.h"
#include "uad_internal.cuh"

namespace uad {

struct PagedArgs {
  void *k = nullptr, *v = nullptr;
  int64_t page_stride = 0, slot_stride = 0, head_stride = 0;
  const int* table = nullptr;
  const int* len = nullptr;
  const int* start = nullptr;
  int64_t table_stride = 0;
  int* status = nullptr;
  FastDiv page;            // division by the page size
  int n_pages = 0, n_kv = 0, dh = 0, dtype = F32;
  int n_seqs = 0, n_rows = 0, max_new = 0, capacity = 0;
};

struct SeqRows {
  int first, n, len;   // first row, new tokens, length; n < 0: left out
};
__device__ __forceinline__ void kv_report(const PagedArgs& p, int bit) {
  if (p.status) atomicOr(p.status, bit);
}
// Sequence b's rows, or n = -1 where tables and lengths do not fit together (nothing of it is read or written then).
__device__ __forceinline__ SeqRows seq_rows(const PagedArgs& p, int b) {
  const int first = p.start ? p.start[b] : b, end = p.start ? p.start[b + 1] : b + 1, len = p.len[b];
  const bool ok = first >= 0 && first <= end && end <= p.n_rows && end - first <= p.max_new && len >= end - first && len <= p.capacity;
  return {first, ok ? end - first : -1, len};
}
// Element offset of token `pos` of a sequence (head 0), or -1 where its page is none. pos < capacity.
__device__ __forceinline__ int64_t token_at(const PagedArgs& p, const int* row, int pos) {
  const int i = p.page.div(pos), page = row[i];
  if ((unsigned)page >= (unsigned)p.n_pages) return -1;
  return page * p.page_stride + (pos - i * (int)p.page.d) * p.slot_stride;
}

// kv_pages.cu: the checks of the structures; UAD_OK with the kernels' arguments, or UAD_EINVAL. device: also that the
// pages are memory of the current device (tables and lengths may be null otherwise).
int paged_args(const uad_kv_pages* pages, const uad_kv_seqs* seqs, int n_rows, bool device, PagedArgs* out);
// Tokens 0 .. n - 1 of a sequence, whose pages are table[0 ..] (device memory, checked), next to each other: k, v [n][n_kv][dh] of the
// pages' type, 16-byte aligned.
cudaError_t launch_kv_gather(const PagedArgs& p, const int* table, int n, void* k, void* v, cudaStream_t s);
// Whether p is memory of the current device.
bool on_current_device(const void* p);
// What an entry returns for its launches. Their error is this call's: the next one, which may ask for the last error, does not find it.
inline int launched(cudaError_t e) {
  if (e == cudaSuccess) return UAD_OK;
  cudaGetLastError();
  return UAD_ECUDA;
}

}  // namespace uad
