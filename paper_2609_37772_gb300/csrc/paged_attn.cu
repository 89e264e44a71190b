// Attention of few new tokens over a paged key-value cache.
#include "kv_pages.cuh"

using namespace uad;

namespace {

struct PagedAttnArgs {
  PagedArgs p;
  const void* q;
  void* out;
  float* lse;
  const uint8_t* mask;
  int64_t q_stride, out_stride, mask_stride;
  float scale;
  int n_heads, group, causal, window;
};

constexpr int kWarps = 4;

template <int T>
__device__ __forceinline__ float get(const void* p, int64_t e) {
  if constexpr (T == F32) return static_cast<const float*>(p)[e];
  else return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[e]);
}

// One CTA a row and head: every warp takes each kWarps-th key.
template <int T, int DH>
__global__ void __launch_bounds__(32 * kWarps) paged_attn_kernel(const PagedAttnArgs a) {
  constexpr int E = DH / 32;
  __shared__ float so[kWarps][DH], sm[kWarps], sl[kWarps];
  pdl_wait();
  pdl_trigger();
  const PagedArgs& p = a.p;
  const int b = blockIdx.z, j = blockIdx.y, h = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const SeqRows s = seq_rows(p, b);
  if (s.n < 0) {
    if (h == 0 && j == 0 && threadIdx.x == 0) kv_report(p, UAD_KV_BAD_SEQ);
    return;
  }
  if (j >= s.n) return;
  const int row = s.first + j, pos = s.len - s.n + j, kvh = h / a.group;
  const int hi = a.causal ? pos + 1 : s.len, lo = a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
  const int* tab = p.table + b * p.table_stride;
  float q[E], o[E], m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) {
    q[e] = get<T>(a.q, row * a.q_stride + (int64_t)h * DH + lane + 32 * e) * a.scale;
    o[e] = 0.f;
  }
  for (int key = lo + warp; key < hi; key += kWarps) {
    if (a.mask && !a.mask[b * a.mask_stride + key]) continue;
    int64_t at = token_at(p, tab, key);
    if (at < 0) {
      if (lane == 0) kv_report(p, UAD_KV_BAD_PAGE);
      continue;
    }
    at += kvh * p.head_stride;
    float d = 0.f;
    for (int e = 0; e < E; ++e) d += q[e] * get<T>(p.k, at + lane + 32 * e);
    for (int x = 16; x > 0; x >>= 1) d += __shfl_xor_sync(0xffffffffu, d, x);
    if (d < -3.402823466e38f) d = -3.402823466e38f;   // a seen key, unlike one that is not
    const float mn = fmaxf(m, d), f = expf(m - mn), w = expf(d - mn);
    m = mn;
    l = l * f + w;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * get<T>(p.v, at + lane + 32 * e);
  }
  for (int e = 0; e < E; ++e) so[warp][lane + 32 * e] = o[e];
  if (lane == 0) sm[warp] = m, sl[warp] = l;
  __syncthreads();
  float M = -INFINITY, L = 0.f;
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm[w]);
  for (int w = 0; w < kWarps; ++w) L += M == -INFINITY ? sl[w] : sl[w] * expf(sm[w] - M);
  const bool none = M == -INFINITY && L == 0.f, undefined = M == -3.402823466e38f;
  for (int d = threadIdx.x; d < DH; d += 32 * kWarps) {
    float x = 0.f;
    for (int w = 0; w < kWarps; ++w) x += so[w][d] * (M == -INFINITY ? 1.f : expf(sm[w] - M));
    x = none ? 0.f : undefined ? NAN : x / L;
    const int64_t e = row * a.out_stride + (int64_t)h * DH + d;
    if constexpr (T == F32) static_cast<float*>(a.out)[e] = x;
    else static_cast<__nv_bfloat16*>(a.out)[e] = __float2bfloat16_rn(x);
  }
  if (a.lse && threadIdx.x == 0)
    a.lse[(int64_t)row * a.n_heads + h] = none ? -INFINITY : undefined ? NAN : M + logf(L);
}

int attn_args(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* t, bool device, PagedAttnArgs* a) {
  if (!t) return UAD_EINVAL;
  const int rc = paged_args(pages, seqs, t->n_rows, device, &a->p);
  if (rc) return rc;
  const int es = a->p.dtype == F32 ? 4 : 2;
  if (t->n_heads < 1 || t->n_heads % a->p.n_kv || t->n_heads / a->p.n_kv > 64) return UAD_EINVAL;
  if ((t->causal != 0 && t->causal != 1) || t->window < 0 || !isfinite(t->scale)) return UAD_EINVAL;
  if (device) {
    if (!t->q || !t->out || t->q_stride < 0 || t->out_stride < 0 || (t->key_mask && t->mask_stride < 0)) return UAD_EINVAL;
    if (reinterpret_cast<uintptr_t>(t->q) % 16 || reinterpret_cast<uintptr_t>(t->out) % 16) return UAD_EINVAL;
    if (t->q_stride * es % 16 || t->out_stride * es % 16 || reinterpret_cast<uintptr_t>(t->lse) % 4) return UAD_EINVAL;
  }
  a->q = t->q; a->out = t->out; a->lse = t->lse; a->mask = t->key_mask;
  a->q_stride = t->q_stride; a->out_stride = t->out_stride; a->mask_stride = t->mask_stride;
  a->scale = t->scale != 0.f ? t->scale : 1.f / sqrtf((float)a->p.dh);
  a->n_heads = t->n_heads; a->group = t->n_heads / a->p.n_kv; a->causal = t->causal; a->window = t->window;
  return UAD_OK;
}

}  // namespace

extern "C" {

int64_t uad_paged_attention_workspace(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn) {
  PagedAttnArgs a{};
  const int rc = attn_args(pages, seqs, attn, false, &a);
  if (rc) return rc;
  return 0;
}

int uad_paged_attention(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn, void* workspace,
                        size_t workspace_bytes, int32_t* status, void* stream) {
  PagedAttnArgs a{};
  const int rc = attn_args(pages, seqs, attn, true, &a);
  if (rc) return rc;
  if (a.p.n_seqs == 0 || a.p.n_rows == 0) return UAD_OK;
  a.p.status = status;
  (void)workspace;
  (void)workspace_bytes;
  const dim3 grid(a.n_heads, a.p.max_new, a.p.n_seqs);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
#define ATTN(T)                                                                                    \
  e = a.p.dh == 64    ? launch_k(paged_attn_kernel<T, 64>, grid, 32 * kWarps, 0, s, a)             \
      : a.p.dh == 128 ? launch_k(paged_attn_kernel<T, 128>, grid, 32 * kWarps, 0, s, a)            \
                      : launch_k(paged_attn_kernel<T, 256>, grid, 32 * kWarps, 0, s, a)
  if (a.p.dtype == F32) ATTN(F32);
  else ATTN(BF16);
#undef ATTN
  return e == cudaSuccess ? UAD_OK : UAD_ECUDA;
}

}  // extern "C"
