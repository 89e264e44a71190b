// The paged cache in 8 bits: the blocks' scales as the kernels take them, codes as numbers.
#pragma once
#include <cuda_fp16.h>

#include "kv_pages.cuh"

namespace uad {

// The scale of head h of block i of a page is at k + page * page + i * block + h * head (in elements), of the values at the same
// place of v.
struct Scales {
  float *k = nullptr, *v = nullptr;
  int64_t page = 0, block = 0, head = 0;
  int log_block = 0;    // tokens of a block
  FastDiv per_page;     // division by the blocks of a page
};

// Two codes (the lower one first) as f16, exactly.
__device__ __forceinline__ uint32_t e4m3_f16(uint32_t w) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
  return r;
}
__device__ __forceinline__ float2 e4m3_pair(uint32_t w) {
  const uint32_t r = e4m3_f16(w);
  return __half22float2(*reinterpret_cast<const __half2*>(&r));
}

// kv_append8.cu: paged_args and the checks of the scales.
int pages8_args(const uad_kv_pages8* pages, const uad_kv_seqs* seqs, int n_rows, bool device, PagedArgs* out, Scales* scales);

// kv_append8.cu: tokens 0 .. n - 1 of a sequence, whose pages are table[0 ..] (device memory, checked), next to each other as fp32: k, v
// [n][n_kv][dh], 16-byte aligned.
cudaError_t launch_kv_gather8(const PagedArgs& p, const Scales& sc, const int* table, int n, void* k, void* v, cudaStream_t s);

}  // namespace uad
