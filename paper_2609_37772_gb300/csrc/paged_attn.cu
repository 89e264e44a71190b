// Attention of few new tokens over a paged key-value cache: the split of the work, the checks of the arguments, and the kernels of
// bf16 and fp32 caches without sinks.
#include "paged_attn_kernels.cuh"

using namespace uad;

namespace {

// How many rows a CTA takes and how the keys are cut, from sizes alone (the workspace of a captured call holds for what its
// graph replays). A CTA costs about 5 us before and after its keys, so there are no more of them than the SMs hold at once
// (`slots`), and pieces are not shorter than 256 keys (fp32: 64) but where everything is one small wave. A cluster
// joins its pieces in 1 us, the workspace and a second kernel take 3; but clusters are placed as a whole, which leaves
// SMs idle once there are many of them or they are large. Long pieces are cut further, up to four waves, so that
// sequences of different lengths even out; but less than 1.75 waves cost more than one. In us, pieces with / without a
// cluster:
//   1 x 817 keys, 8 heads over 1 of 256:   13: 7.1 / 9.1,  7: 8.3 / 9.6
//   64 x 282..1129, the same:               4: 16.3 / 18.4,  8: 23.3 / 17.1
//   6 x 2001..8003, 5 new tokens:          12: 31.8 / 32.8,  16: 48.1 / 27.5
//   2 x 32768, 131071, 32 over 8 of 128:   28: - / 130,  80: - / 117
//   16 x 4000, 32 over 8 of 128:            3: - / 50,  4: - / 57
//   16 x 700, 8 new tokens, 24 of 64:       1: 16.5,  2: - / 22.6
//   64 x 4000, 4 new tokens, 8 over 1 of 256: 2: - / 75,  4: - / 86
// With more heads than the SMs hold CTAs and up to 512 keys, a CTA's warps may have a key/value head each, which needs no joining. Its
// queries then take four times the shared memory, so that fewer CTAs fit an SM (heads of 256: one and not two), and their number is a
// quarter. Both forms cost their rounds (about 4 us a round, 40000 / head_dim keys of a head, before and after the keys) and the keys
// of the fullest SM, an eighth more where warps have heads, half more where they have 32 rows and are alone on their SM. In us, one
// token, with / without, and what the costs choose:
//   51 x 5 keys, 24 heads of 64:                4.7 / 9.0, with         256 x 60, the same:     21.7 / 40.2, with
//   26 x 512, the same:                        22.7 / 18.9, without     64 x 300, the same:     23.8 / 25.5, with
//   64 x 60, 32 over 8 of 128:                  8.1 / 9.8, with         102 x 512, the same:    40.3 / 37.0, without
//   51 x 60, 8 of 256:                         10.5 / 11.4, with        38 x 300, the same:     28.9 / 19.1, without
//   102 x 60, 128 over 4 of 128:               13.8 / 14.8, with        76 x 512, the same:     49.1 / 20.4, without
// Keys past 512 gain nothing (64 x up to 2000 keys of 24 heads of 64: 106 / 86).
size_t warp_heads_smem(int dh, int row_tiles) {
  if (dh == 64) return row_tiles == 1 ? tc_smem<64, 1>(kWarps) : row_tiles == 2 ? tc_smem<64, 2>(kWarps) : tc_smem<64, 4>(kWarps);
  if (dh == 128) return row_tiles == 1 ? tc_smem<128, 1>(kWarps) : row_tiles == 2 ? tc_smem<128, 2>(kWarps) : tc_smem<128, 4>(kWarps);
  return row_tiles == 1 ? tc_smem<256, 1>(kWarps) : tc_smem<256, 2>(kWarps);
}
struct Split {
  int pieces, piece_keys, clustered;
};
// `keys` in at most n pieces.
Split cut_keys(int64_t keys, int64_t n, int64_t units, int64_t slots, int64_t round) {
  const int64_t piece = ((keys + n - 1) / n + round - 1) / round * round;
  Split c;
  c.piece_keys = (int)(piece < (1ll << 30) ? piece : 1ll << 30);
  c.pieces = (int)((keys + c.piece_keys - 1) / c.piece_keys);
  const int64_t ctas = units * c.pieces;
  c.clustered = c.pieces > 1 && ((c.pieces <= kMaxCluster && ctas <= kAttnSms) || (c.pieces <= 8 && ctas * 20 <= slots * 17));
  return c;
}
Split split_keys(int64_t keys, int64_t units, int64_t slots, int64_t least, int64_t round) {
  const auto most = [&](int64_t n) { return (keys + n - 1) / n; };   // pieces of at least n keys
  int64_t n;
  if (keys <= kMaxCluster * 256 && units * (most(round) < kMaxCluster ? most(round) : kMaxCluster) <= kAttnSms) {
    return cut_keys(keys, most(round) < kMaxCluster ? most(round) : kMaxCluster, units, slots, round);
  } else {
    n = units * 5 >= slots * 3 ? 1 : units * 2 > slots ? 2 : slots / units;
    if (n > 1 && n <= 8 && units * n * 20 > slots * 17) n = slots * 17 / (units * 20) > 1 ? slots * 17 / (units * 20) : n;
    if (n > most(least)) n = most(least);
    const int64_t waves = 4 * slots / units < most(1024) ? 4 * slots / units : most(1024);
    if (waves > n) n = waves;
    if (n > 2 && units * n > slots && units * n * 4 < slots * 7) n = slots / units > 1 ? slots / units : n;
  }
  return cut_keys(keys, n, units, slots, 64);
}
// warp_smem: shared memory of a CTA whose warps have heads of their own (0: there is no such form). round: keys that the warps of a CTA take at
// once, of which the pieces of a small call are multiples (8-bit caches, 128 / 64 in us: 1 x 817 of 8 heads over 1 of 256 7.1 / 7.5, 1 x 100 of 24
// heads of 64 4.0 / 5.0).
void attn_plan(const uad_kv_seqs* s, int ctas_per_sm, size_t warp_smem, int round, PagedAttnArgs* a) {
  const int64_t all = s->max_len > 0 && s->max_len < a->p.capacity ? s->max_len : a->p.capacity;
  const int64_t near = (int64_t)a->window + a->sinks + a->p.max_new - 1;
  const int64_t keys = a->window > 0 && near < all ? near : all;
  const int64_t units = (int64_t)a->p.n_seqs * a->p.n_kv * a->row_blocks, slots = kAttnSms * ctas_per_sm;
  const int64_t least = a->p.dtype == F32 ? 64 : 256;
  a->warp_heads = 0;
  if (warp_smem > 0 && a->p.n_kv % kWarps == 0 && keys <= 512) {
    const int64_t fit = 228 * 1024 / ((int64_t)warp_smem + 1024);   // an SM's, and what it keeps of each CTA's
    const int64_t ctas = units / kWarps, held = kAttnSms * (fit < ctas_per_sm ? fit : ctas_per_sm), lap = 8 * (40000 / a->p.dh);
    const int64_t with = (ctas + held - 1) / held * lap + (ctas + kAttnSms - 1) / kAttnSms * kWarps * keys * (a->row_tiles == 4 ? 12 : 9);
    const int64_t without = (units + slots - 1) / slots * lap + (units + kAttnSms - 1) / kAttnSms * keys * 8;
    a->warp_heads = with < without;
  }
  Split c = split_keys(keys, units, slots, least, round);
  if (keys < all && c.pieces > 1 && !c.clustered) {
    // Fewer keys can be more pieces, or as many that are no cluster: no more than there are without the window, so that what
    // a call without one needs is enough for every window. (What makes a cluster of so many pieces makes one of fewer.)
    const int most = split_keys(all, units, slots, least, round).pieces;
    if (most < c.pieces) c = cut_keys(keys, most, units, slots, 64);
  }
  a->pieces = c.pieces;
  a->piece_keys = c.piece_keys;
  a->clustered = c.clustered;
}

}  // namespace

int64_t uad::attn_bytes(const PagedAttnArgs& a) {
  return a.pieces > 1 && !a.clustered ? (int64_t)a.p.n_rows * a.n_heads * a.pieces * (a.p.dh + 2) * 4 : 0;
}

bool uad::attn_workspace(PagedAttnArgs* a, void* workspace, size_t bytes) {
  const int64_t need = attn_bytes(*a);
  if (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 || bytes < (size_t)need)) return false;
  a->part_o = static_cast<float*>(workspace);
  a->part_ml = reinterpret_cast<float2*>(a->part_o + (int64_t)a->p.n_rows * a->n_heads * a->pieces * a->p.dh);
  return true;
}

int uad::attn_args(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* t, int sinks, bool device, PagedAttnArgs* a) {
  if (!t) return UAD_EINVAL;
  const int rc = paged_args(pages, seqs, t->n_rows, device, &a->p);
  return rc ? rc : attn_split(seqs, t, sinks, device, nullptr, a);
}

int uad::attn_split(const uad_kv_seqs* seqs, const uad_attn* t, int sinks, bool device, const AttnFit8* eight, PagedAttnArgs* a) {
  const int es = a->p.dtype == F32 ? 4 : 2;   // of queries and outputs
  if (sinks < 0) return UAD_EINVAL;
  if (t->n_heads < 1 || t->n_heads % a->p.n_kv || t->n_heads / a->p.n_kv > 64) return UAD_EINVAL;
  if ((int64_t)t->n_heads * a->p.max_new >= (1ll << 31)) return UAD_EINVAL;
  if ((t->causal != 0 && t->causal != 1) || t->window < 0 || !isfinite(t->scale)) return UAD_EINVAL;
  if (device) {
    if (!t->q || !t->out || t->q_stride < 0 || t->out_stride < 0 || (t->key_mask && t->mask_stride < 0)) return UAD_EINVAL;
    if (reinterpret_cast<uintptr_t>(t->q) % 16 || reinterpret_cast<uintptr_t>(t->out) % 16) return UAD_EINVAL;
    if (t->q_stride * es % 16 || t->out_stride * es % 16 || reinterpret_cast<uintptr_t>(t->lse) % 4) return UAD_EINVAL;
  }
  a->q = t->q; a->out = t->out; a->lse = t->lse; a->mask = t->key_mask;
  a->q_stride = t->q_stride; a->out_stride = t->out_stride; a->mask_stride = t->mask_stride;
  a->scale = t->scale != 0.f ? t->scale : 1.f / sqrtf((float)a->p.dh);
  a->scale_log2 = a->scale * 1.4426950408889634f;
  a->n_heads = t->n_heads; a->group = t->n_heads / a->p.n_kv; a->causal = t->causal; a->window = t->window;
  a->sinks = t->window > 0 ? sinks : 0;
  if (a->p.n_seqs == 0 || a->p.n_rows == 0) return UAD_OK;   // nothing to split: no pieces, no workspace, no launch
  // rows of a CTA: 8, 16 or 32, as many as there are, within what the registers hold
  const int dh = a->p.dh, tiles = a->p.dtype == F32 ? 1 : dh == 256 ? 2 : 4;
  const int64_t rows = (int64_t)a->p.max_new * a->group;
  a->row_tiles = 1;
  while (a->row_tiles < tiles && 8 * a->row_tiles < rows) a->row_tiles *= 2;
  a->row_blocks = (int)((rows + 8 * a->row_tiles - 1) / (8 * a->row_tiles));
  // fp32, 64 dims: three CTAs an SM hide more, two have the registers that make a lone one faster (64 x 8000 keys of two heads 119 us
  // against 132, 33 x 600 with 4 new tokens 10.7 against 12.7; but 28.7 against 22.8 with 16, where two an SM are one wave)
  const int64_t units = (int64_t)a->p.n_seqs * a->p.n_kv * a->row_blocks;
  a->f32_ctas = dh == 64 && (units > 304 || units * 5 < 304 * 3) ? 3 : 2;
  const int log_tiles = a->row_tiles == 4 ? 2 : a->row_tiles - 1;
  if (eight) attn_plan(seqs, eight->ctas[log_tiles], eight->smem[log_tiles], eight->round[log_tiles], a);
  else if (a->p.dtype == F32) attn_plan(seqs, a->f32_ctas, 0, 64, a);
  else attn_plan(seqs, a->row_tiles == 4 || dh == 256 ? 2 : dh == 64 && a->row_tiles == 1 ? 4 : 3, warp_heads_smem(dh, a->row_tiles), 64, a);
  a->by_group = FastDiv((uint32_t)a->group);
  a->by_x = FastDiv((uint32_t)(a->clustered ? a->pieces : a->row_blocks));
  return UAD_OK;
}

extern "C" {

int64_t uad_paged_attention_workspace(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn) {
  return uad_paged_attention_sinks_workspace(pages, seqs, attn, 0);
}

int64_t uad_paged_attention_sinks_workspace(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn, int32_t sinks) {
  PagedAttnArgs a{};
  const int rc = attn_args(pages, seqs, attn, sinks, false, &a);
  return rc ? rc : attn_bytes(a);
}

int uad_paged_attention(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn, void* workspace,
                        size_t workspace_bytes, int32_t* status, void* stream) {
  return uad_paged_attention_sinks(pages, seqs, attn, 0, workspace, workspace_bytes, status, stream);
}

int uad_paged_attention_sinks(const uad_kv_pages* pages, const uad_kv_seqs* seqs, const uad_attn* attn, int32_t sinks, void* workspace,
                              size_t workspace_bytes, int32_t* status, void* stream) {
  PagedAttnArgs a{};
  const int rc = attn_args(pages, seqs, attn, sinks, true, &a);
  if (rc) return rc;
  if (a.p.n_seqs == 0 || a.p.n_rows == 0) return UAD_OK;
  a.p.status = status;
  if (!attn_workspace(&a, workspace, workspace_bytes)) return UAD_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.sinks > 0) return launched(launch_paged_sinks(a, s));
  return launched(a.p.dh == 64 ? launch_dh<64, false>(a, s) : a.p.dh == 128 ? launch_dh<128, false>(a, s) : launch_dh<256, false>(a, s));
}

}  // extern "C"
