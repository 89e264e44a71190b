// Attention over a paged cache through a window that leaves the first tokens visible: bf16 and fp32 caches. Kernels of their own, so that
// those without sinks stay as they are.
#include "paged_attn_kernels.cuh"

cudaError_t uad::launch_paged_sinks(const PagedAttnArgs& a, cudaStream_t s) {
  return a.p.dh == 64 ? launch_dh<64, true>(a, s) : a.p.dh == 128 ? launch_dh<128, true>(a, s) : launch_dh<256, true>(a, s);
}
