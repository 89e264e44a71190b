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

// ---- what the appends share ----

constexpr int kItem = 16;   // dimensions that a thread takes of a head: 8 pairs, or 16 that are not rotated

// cos and sin of position * turn / 2^64 turns. The product wraps at whole turns, which is exact; what is left is
// taken to the nearest quarter, so that its rounding to fp32 is below 2^-28 of a turn.
__device__ __forceinline__ void rotation(uint32_t pos, uint64_t turn, float* c, float* s) {
  const uint64_t ph = (uint64_t)pos * turn + (1ull << 61);
  const int quarter = (int)(ph >> 62);
  const int64_t rest = (int64_t)(ph & ((1ull << 62) - 1)) - (1ll << 61);   // within an eighth of a turn
  float cr, sr;
  sincospif((float)(int32_t)(rest >> 32) * 4.656612873077393e-10f, &sr, &cr);   // 2^-31: half turns of 2^-32 turns
  const float a = quarter & 1 ? -sr : cr, b = quarter & 1 ? cr : sr;
  *c = quarter & 2 ? -a : a;
  *s = quarter & 2 ? -b : b;
}

template <int T>
__device__ __forceinline__ void load8(const void* base, int64_t e, float* x) {
  if constexpr (T == F32) {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(base) + e);
    const float4 a = f[0], b = f[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) + e);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
template <int T>
__device__ __forceinline__ void store8(void* base, int64_t e, const float* x) {
  if constexpr (T == F32) {
    float4* f = reinterpret_cast<float4*>(static_cast<float*>(base) + e);
    f[0] = make_float4(x[0], x[1], x[2], x[3]);
    f[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + e) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// kv_pages.cu: the checks of the structures; UAD_OK with the kernels' arguments, or UAD_EINVAL. device: also that the
// pages are memory of the current device (tables and lengths may be null otherwise). eight: pages of e4m3, and no others.
int paged_args(const uad_kv_pages* pages, const uad_kv_seqs* seqs, int n_rows, bool device, PagedArgs* out, bool eight = false);
// Tokens 0 .. n - 1 of a sequence, whose pages are table[0 ..] (device memory, checked), next to each other: k, v [n][n_kv][dh] of the
// pages' type, 16-byte aligned.
cudaError_t launch_kv_gather(const PagedArgs& p, const int* table, int n, void* k, void* v, cudaStream_t s);
inline bool bad_address(const void* p, int64_t stride, int es) {
  return reinterpret_cast<uintptr_t>(p) % 16 != 0 || stride < 0 || (stride * es) % 16 != 0;
}
// Whether p is memory of the current device.
bool on_current_device(const void* p);
// What an entry returns for its launches. Their error is this call's: the next one, which may ask for the last error, does not find it.
inline int launched(cudaError_t e) {
  if (e == cudaSuccess) return UAD_OK;
  cudaGetLastError();
  return UAD_ECUDA;
}

}  // namespace uad
