// Attention of few new tokens over a paged cache that is held in 8 bits.
//
// out = sum_j p_j sv_j c_j with p = softmax(scale sk_j q c'_j): codes c', c of e4m3 and a scale of keys and one of values for each
// block of tokens and head. Half the bytes of a bf16 cache for the same products, so that the instructions of a key count: the tensor
// cores multiply f16 (e4m3 is emulated in mma.sync here), which every code is exactly, two codes an instruction. A warp takes a
// slice of 16 or 32 keys at a time out of a ring of its own, as with bf16 caches, but
// - keys: the 16 bytes of a row that ldmatrix hands out are 16 dims, four to a lane. Which of an MMA's dims they are called does not matter
//   as long as the queries agree: a lane's four bytes are its two registers of B, and the queries lie in shared memory in that order;
// - values: ldmatrix transposes bytes (16 keys by 16 dims), so a lane gets four keys of one dim, which are its two registers of A; the rows
//   that it is given in turn are the keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9 that the lane has as scores;
// - rows lie in shared memory without gaps, their 16-byte pieces exchanged by a number that differs between the eight keys of each
//   access (key_swap), the first eight or every second pair;
// - queries: f16 after a power of two that takes each row's largest value to 2^13..2^14: bf16 has fewer bits, and what falls below
//   f16's least is 2^-38 of the largest;
// - scales come through the ring beside the codes. A key's multiplies its scores; a value's multiplies the weights, 2^11 p sv / r:
//   r is a power of two of the row, the largest p sv so far, as m is its largest score so far (p is 2^(score - m)): keys that the row does
//   not see, or gives no weight, have no part in it, whatever their scale. A weight goes in as two f16, its upper 11 bits and the rest: a second MMA
//   for an error of 2^-21, and 2^-34 of the row's largest weight for small ones, where one f16 has 2^-11, an eighth of what the
//   output's own rounding to bf16 is (one / two, in us: 64 x 4000 keys of 32 heads over 8 of 128 93 / 95, of 8 over 1 of 256 28 / 29, with 4 new tokens
//   60 / 67; 16 x 4000 with 8 new tokens of 32 over 8 of 128 60 / 74, where the MMAs of four tiles of rows count).
//
// One new token: 64 x 4000 keys of 32 heads over 8 of 128 take 96 us (524 MB, 5.5 TB/s; 170 from a bf16 cache), 2 sequences of up to 131071 of
// the same 63 us (5.3 TB/s), 64 x 4000 of 8 over 1 of 256 29 us (4.5 TB/s). What bounds: the latencies of a warp's slice (about 860
// instructions for 32 keys of 128 dims, of which the conversions of codes are 190; 0.44 issued a cycle and scheduler) with the two to four
// warps a scheduler that registers allow. Slices of 16 keys with four CTAs an SM take 111 us for the first, four slots of the ring in place
// of three 97; of 256 dims, slices of 16 keys 31 us for the last.
#include "kv_pages8.cuh"
#include "paged_attn.cuh"

#include <algorithm>

namespace uad {
namespace {

struct PagedAttn8Args {
  PagedAttnArgs a;
  Scales sc;
  // Places in 32 bits: of codes in units of the largest power of two that divides all strides (at least 16, at most 2^31), of scales in elements.
  // 64-bit sums and shuffles take 1 to 4% longer with heads of 64 and 128.
  uint32_t unit, page_units, slot_units, head_units, scale_page, scale_block, scale_head;
  int parts;      // into how many the sequences' chunks are cut evenly; 0: as attn_plan has it
  int2* spans;    // [CTA] the sequence that begins in its part and ends in a later one, and that one; -1: there is none
};

constexpr float kLag = 4.f;            // how far (base 2) scores and weights may pass their running maximum before it follows: f16 holds 2^15
constexpr int kWeightBits = 11;        // weights are up to 2^kWeightBits where the running maximum follows
constexpr float kLeastUnit = 7.888609052210118e-31f;   // 2^-100, of a row's weights

__device__ __forceinline__ void mma16816h(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldm4(uint32_t* r, uint32_t s) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(s) : "memory");
}
// Two matrices of 16 rows (keys, the addresses of lanes 0..15 and 16..31) by 16 bytes (dims): lane (g, t) gets the rows 4 t .. 4 t + 3 of
// the columns g and g + 8 of each.
__device__ __forceinline__ void ldm_t8(uint32_t* r, uint32_t s) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(s) : "memory");
}
// Four codes as two pairs of f16.
__device__ __forceinline__ void e4m3_f16x4(uint32_t w, uint32_t* lo, uint32_t* hi) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}\n" : "=r"(*lo), "=r"(*hi) : "r"(w));
}
// The larger one; NaN where one is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 lds_f2(uint32_t s) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(s) : "memory");
  return v;
}
__device__ __forceinline__ float lds_f(uint32_t s) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(s) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t s) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(s) : "memory");
  return v;
}
__device__ __forceinline__ void sts_u32(uint32_t s, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(s), "r"(v) : "memory"); }
// 16 bytes to shared memory where ok is true.
__device__ __forceinline__ void cp16_if(uint32_t s, const void* g, bool ok) {
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n @p cp.async.cg.shared.global [%0], [%1], 16;\n}\n" ::"r"(s), "l"(g), "r"((uint32_t)ok) : "memory");
}
// 4 bytes to shared memory, zeros where ok is false.
__device__ __forceinline__ void cp4_or_zero(uint32_t s, const void* g, bool ok) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(s), "l"(g), "r"(ok ? 4 : 0) : "memory");
}
__device__ __forceinline__ void sts_zero16(uint32_t s) { asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(s), "r"(0) : "memory"); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Four codes: 0x80 in the bytes that are NaN; 0xff there.
__device__ __forceinline__ uint32_t nan_bits(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (nan_bits(w) >> 7) * 0xffu; }

template <int DH, int NR>
constexpr int slice_steps() { return NR == 4 || (DH == 256 && NR == 2) ? 1 : 2; }   // keys of a slice, in sixteens
template <int DH, int NR>   // K and V slices in turn
constexpr int ring_slots() { return DH == 256 ? (NR == 1 ? 3 : 4) : NR == 4 ? 8 : DH == 128 ? 3 : 4; }
// What the numbers of a key's 16-byte pieces are xored with. Eight keys of one access (0..7, 8..15, or pairs 0 1 8 9 2 3 10 11, 4 5 12 13 6 7 14 15)
// then lie in different banks, of which 128 bytes go around once: a row of 64 dims is half of that.
template <int DH>
__device__ __forceinline__ int key_swap(int key) {
  return DH == 64 ? (key >> 1 & 3) ^ (key >> 3 & 1) << 1 : (key & 7) ^ (key >> 3 & 1) << 2;
}
template <int DH>
constexpr int query_pitch() { return 2 * DH + 16; }
template <int DH, int NR>
constexpr int slot_bytes() { return slice_steps<DH, NR>() * 16 * DH + 128; }   // codes, then scales
template <int DH, int NR>
constexpr int ring8() { return kWarps * ring_slots<DH, NR>() * slot_bytes<DH, NR>(); }
// a set of queries: rows, then what their scores are multiplied by
template <int DH, int NR>
constexpr int query_bytes() { return 8 * NR * (query_pitch<DH>() + 4); }
template <int DH, int NR>
constexpr size_t smem8(int heads) {
  return (size_t)ring8<DH, NR>() + receive_extra<DH, 8 * NR>(ring8<DH, NR>()) + sizeof(EndShared<8 * NR>) + heads * query_bytes<DH, NR>();
}
template <int DH, int NR>
constexpr size_t even_smem(int seqs) { return smem8<DH, NR>(1) + (seqs + 1) * 4; }
template <int DH, int NR>
constexpr int ctas8() { return NR == 4 || DH == 256 ? 2 : DH == 64 && NR == 1 ? 4 : 3; }

// Where a key's codes and scale are in this head; kNowhere: no row sees it or its page is none.
constexpr uint32_t kNowhere = 0xffffffffu;
struct Place {
  uint32_t code, scale;
};
__device__ __forceinline__ Place place_of(const PagedAttn8Args& g, const Piece& c, const Found& f) {
  const PagedAttnArgs& a = g.a;
  if (f.key >= c.k1 || !f.shown) return {kNowhere, 0};
  if ((unsigned)f.page >= (unsigned)a.p.n_pages) {
    kv_report(a.p, UAD_KV_BAD_PAGE);
    return {kNowhere, 0};
  }
  const uint32_t slot = f.token - a.p.page.div(f.token) * a.p.page.d;
  return {f.page * g.page_units + slot * g.slot_units + c.kvh * g.head_units,
          f.page * g.scale_page + (slot >> g.sc.log_block) * g.scale_block + c.kvh * g.scale_head};
}

// Sharing evenly. A sequence's keys are chunks of four slices; the sequences' chunks one behind the other are cut into as many parts as
// there are CTAs for each key/value head and block of rows (blockIdx.x: the part, .y: the head, .z: the rows), whatever the
// lengths. Parts are the same for all heads, which so read a token's keys at about the same time: they lie next to each other in most caches, and
// reading one head's alone takes up to 1.6 times as long (64 x 1000 keys of 24 heads of 64: 75 us against 46, with one f16 a weight). A CTA takes the pieces of its part
// in turn. A sequence that lies in one part is done there. Otherwise its pieces go to the workspace (a CTA has two at most: one
// of a sequence that began before its part, one of a sequence that goes on behind it), and a second kernel joins them.
constexpr int kEvenSeqs = 1024;   // sequences that a CTA sums up

template <int DH, int NR>
constexpr int chunk_keys() { return kWarps * 16 * slice_steps<DH, NR>(); }

template <int DH, int NR>
__device__ __forceinline__ int chunks_of(const PagedAttnArgs& a, const SeqRows& s) {
  if (s.n <= 0) return 0;
  const int64_t near = (int64_t)a.window + s.n - 1 + a.sinks;   // no block of rows has more keys
  const int keys = a.window > 0 && near < s.len ? (int)near : s.len;
  return (keys + chunk_keys<DH, NR>() - 1) / chunk_keys<DH, NR>();
}
// This CTA's part of the chunks, and the sequence that it begins in.
struct EvenShare {
  int share, from, to, b;
  SeqRows s;
};
// Sums over the sequences: at[b] chunks before sequence b, at[n_seqs] all of them. By all threads; ends with a barrier.
template <int DH, int NR>
__device__ __forceinline__ EvenShare even_sums(const PagedAttnArgs& a, int* at) {
  __shared__ int before[kWarps];
  __shared__ int4 found;
  const int n = a.p.n_seqs, per = (n + kThreads - 1) / kThreads, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b0 = threadIdx.x * per;
  int sum = 0;
  SeqRows s{};
  for (int b = b0; b < min(n, b0 + per); ++b) {
    s = seq_rows(a.p, b);
    if (s.n < 0 && blockIdx.x + blockIdx.y + blockIdx.z == 0) kv_report(a.p, UAD_KV_BAD_SEQ);
    at[b] = sum;
    sum += chunks_of<DH, NR>(a, s);
  }
  int upto = sum;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int v = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 31) before[warp] = upto;
  __syncthreads();
  int add = upto - sum, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) add += before[w];
    all += before[w];
  }
  EvenShare e;
  e.share = max((all + (int)gridDim.x - 1) / (int)gridDim.x, 2);   // short ones cost more than they gain
  const int64_t from = (int64_t)e.share * blockIdx.x;
  e.from = (int)min(from, (int64_t)all);
  e.to = (int)min(from + e.share, (int64_t)all);
  for (int b = b0; b < min(n, b0 + per); ++b) at[b] += add;
  if (threadIdx.x == kThreads - 1) at[n] = all;
  if (per == 1 && e.from >= add && e.from < add + sum) found = make_int4(b0, s.first, s.n, s.len);
  __syncthreads();
  e.b = per == 1 ? found.x : -1;
  e.s = {found.y, found.z, found.w};
  return e;
}
// The sequence of chunk x: the last b with at[b] <= x.
__device__ __forceinline__ int even_seq(const int* at, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}
// A CTA's number, under which its spans and pieces lie.
__device__ __forceinline__ int even_cta(int part, int head, int rows) { return (part * gridDim.y + head) * gridDim.z + rows; }

template <int DH, int NR, bool EVEN>   // head dim; 8 NR query rows
__global__ void __launch_bounds__(kThreads, ctas8<DH, NR>()) paged_attn8_kernel(const PagedAttn8Args args) {
  constexpr int KT = slice_steps<DH, NR>(), KEYS = 16 * KT, SLOTS = ring_slots<DH, NR>(), AHEAD = (SLOTS + 1) / 2;
  constexpr int MT = (NR + 1) / 2, QPITCH = query_pitch<DH>(), SLOT = slot_bytes<DH, NR>(), SCALES = KEYS * DH;
  constexpr int STEPS = DH / 16, RING = ring8<DH, NR>(), CHUNK = chunk_keys<DH, NR>(), EXTRA = receive_extra<DH, 8 * NR>(RING);
  constexpr int LANES = DH >= 128 ? 8 : DH / 16, AT_ONCE = 32 / LANES;   // lanes that copy 16 bytes each of a key; keys at once
  using S = Sums<DH, 8 * NR>;
  static_assert(kWarps * S::kBytes <= RING, "the warps' sums fit the ring");
  static_assert(AHEAD * KEYS <= 64, "the bits of the keys ahead");
  static_assert(SLOT % 128 == 0, "rows' pieces are exchanged by xor within 128 bytes");
  constexpr int ODD = DH == 64 ? 32 : 64;   // what the addresses of keys 8..15 of sixteen are xored with
  extern __shared__ __align__(128) unsigned char smem[];
  const PagedAttnArgs& a = args.a;
  const uint32_t base = su32(smem);
  EndShared<8 * NR>* end = reinterpret_cast<EndShared<8 * NR>*>(smem + RING + EXTRA);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t sq = base + RING + EXTRA + sizeof(EndShared<8 * NR>) + (a.warp_heads ? warp * query_bytes<DH, NR>() : 0);
  const uint32_t sf = sq + 8 * NR * QPITCH;   // what each row's scores are multiplied by
  pdl_wait();
  pdl_trigger();
  const uint32_t ring = base + warp * (SLOTS * SLOT);
  // even: where this CTA's part begins and ends, in chunks of all units, and where it is
  int* const sums = reinterpret_cast<int*>(smem + RING + EXTRA + sizeof(EndShared<8 * NR>) + query_bytes<DH, NR>());
  int x = 0;
  EvenShare e;
  if constexpr (EVEN) {
    e = even_sums<DH, NR>(a, sums);
    x = e.from;
    if (threadIdx.x == 0) args.spans[even_cta(blockIdx.x, blockIdx.y, blockIdx.z)] = make_int2(-1, 0);
  }
  for (bool again = false;; again = true) {
  Piece c;
  Found first[AHEAD + 1], found;
  int part = 0;   // even: 0 the whole sequence, 1 of one from before, 2 of one that begins here
  if constexpr (EVEN) {
    if (again) __syncthreads();   // shared memory is free
    int b, c0, c1, chunks;
    do {   // the next sequence that has rows for this CTA
      if (x >= e.to) return;
      if (!again && x == e.from && e.b >= 0) {   // known from the sums
        b = e.b;
        c.s = e.s;
      } else {
        b = even_seq(sums, a.p.n_seqs, x);
        c.s = seq_rows(a.p, b);
      }
      chunks = sums[b + 1] - sums[b];
      c0 = x - sums[b];
      c1 = min(chunks, c0 + e.to - x);
      x += c1 - c0;
      c.r0 = blockIdx.z * 8 * NR;
      c.rows = min(8 * NR, c.s.n * a.group - c.r0);
    } while (c.rows <= 0);
    part = c0 > 0 ? 1 : c1 < chunks ? 2 : 0;
    if (part == 2 && threadIdx.x == 0) args.spans[even_cta(blockIdx.x, blockIdx.y, blockIdx.z)] = make_int2(b, (sums[b + 1] - 1) / e.share);
    c.b = b;
    c.kvh = blockIdx.y;
    c.piece = 0;
    c.kw = warp;
    c.wk = kWarps;
    const int before = c.s.len - c.s.n, at = before + (int)a.by_group.div(c.r0), lo = a.window > 0 ? max(0, at - a.window + 1) : 0;
    c.shift = max(0, lo - a.sinks);
    c.first_pos = at - c.shift;
    c.last_pos = before - c.shift + (int)a.by_group.div(c.r0 + c.rows - 1);
    const int hi = a.causal ? c.last_pos + 1 : c.s.len - c.shift;
    c.k0 = min(c0 * CHUNK, hi);
    c.k1 = c1 == chunks ? hi : min(c1 * CHUNK, hi);
#pragma unroll
    for (int i = 0; i < AHEAD + 1; ++i) first[i] = find_key<true>(a, b, c.shift, c.k0 + (i * kWarps + warp) * KEYS + lane % KEYS);
  } else {
    if (!find_piece<AHEAD + 1, true>(a, 8 * NR, KEYS, &c, first) || no_keys(a, c)) return;
  }
  // Queries: requested before anything that waits for a page, and put as f16, each row times a power of two; dims 4 t .. 4 t + 3 of
  // sixteen where an MMA has its 2 t, 2 t + 1, 2 t + 8, 2 t + 9.
  constexpr int W = DH / 64;   // pairs of a lane
  const auto get_query = [&](int r, uint32_t* w) {
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + (r < c.rows ? row_at(a, c, r, a.q_stride, DH) : 0) + 2 * W * lane;
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0;
    if (r >= c.rows) return;
    if constexpr (W == 1) w[0] = *reinterpret_cast<const uint32_t*>(src);
    else if constexpr (W == 2) { const uint2 v = *reinterpret_cast<const uint2*>(src); w[0] = v.x; w[1] = v.y; }
    else { const uint4 v = *reinterpret_cast<const uint4*>(src); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
  };
  const auto put_query = [&](int r, const uint32_t* w) {
    uint32_t top = 0;   // the largest exponent of a finite value
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const uint32_t e0 = w[i] >> 7 & 0xff, e1 = w[i] >> 23 & 0xff;
      top = max(top, max(e0 == 0xff ? 0u : e0, e1 == 0xff ? 0u : e1));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    const uint32_t e = min(127u + 13 + 127 - top, 253u);
    const float f = __uint_as_float(e << 23);
    if (lane == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(sf + 4 * r), "f"(a.scale_log2 * __uint_as_float((254 - e) << 23)) : "memory");
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int d = 2 * (W * lane + i), x = d & 15;
      sts_u32(sq + r * QPITCH + 2 * ((d & ~15) + (x >> 2) * 2 + (x & 2) * 4), pack_f16(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f));
    }
  };
  // a warp's share of the CTA's rows, or the first half of its own
  uint32_t qw[4 * NR][W];
#pragma unroll
  for (int i = 0; i < 4 * NR; ++i)
    if (i < 2 * NR || a.warp_heads) get_query(a.warp_heads ? i : warp + kWarps * i, qw[i]);
  const int slices = (c.k1 - c.k0 + KEYS - 1) / KEYS, mine = (slices - c.kw + c.wk - 1) / c.wk;
  const auto slice_key = [&](int i) { return c.k0 + (i * c.wk + c.kw) * KEYS; };

  uint64_t seen = 0;   // KEYS bits a slice, the next one lowest
  uint32_t at[KEYS / AT_ONCE], scale_at = kNowhere;
  bool whole = true;   // every key of the slice whose places are in `at` is seen
  int slot = 0;
  const uint32_t to = ring + lane / LANES * DH + (lane % LANES ^ key_swap<DH>(lane / LANES)) * 16;
  // of key AT_ONCE h + lane / LANES: half of a row of keys further on and every eight keys, another half is exchanged
  const auto place = [&](int h) { return (to ^ ((LANES == 8 ? (h ^ h >> 1) & 1 : h & 1) ? ODD : 0)) + slot * SLOT + AT_ONCE * h * DH; };
  // Keys that nobody sees are not copied: their scores are not looked at, their values are zeros.
  const auto copy = [&](int i, const void* pool, const float* scales, bool values) {
    if (i < mine) {
      const char* src = static_cast<const char*>(pool) + lane % LANES * 16;
#pragma unroll
      for (int h = 0; h < KEYS / AT_ONCE; ++h)
#pragma unroll
        for (int x = 0; x < DH / (16 * LANES); ++x)
          cp16_if(place(h) + x * 16 * LANES, src + (uint64_t)at[h] * args.unit + x * 16 * LANES, at[h] != kNowhere);
      if (values && !whole) {
#pragma unroll
        for (int h = 0; h < KEYS / AT_ONCE; ++h)
#pragma unroll
          for (int x = 0; x < DH / (16 * LANES); ++x)
            if (at[h] == kNowhere) sts_zero16(place(h) + x * 16 * LANES);
      }
      if (lane < KEYS) cp4_or_zero(ring + slot * SLOT + SCALES + 4 * lane, scales + (scale_at == kNowhere ? 0 : scale_at), scale_at != kNowhere);
    }
    cp_commit();
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
  };
  const auto copy_k = [&](int i, int ahead, const Found& fnd) {
    Place e{kNowhere, 0};
    if (i < mine) e = place_of(args, c, fnd);
    const uint32_t there = __ballot_sync(0xffffffffu, e.code != kNowhere) & (0xffffffffu >> (32 - KEYS));
    whole = there == 0xffffffffu >> (32 - KEYS);
    seen |= (uint64_t)there << (KEYS * ahead);
#pragma unroll
    for (int h = 0; h < KEYS / AT_ONCE; ++h) at[h] = __shfl_sync(0xffffffffu, e.code, AT_ONCE * h + lane / LANES);
    scale_at = e.code == kNowhere ? kNowhere : e.scale;
    copy(i, a.p.k, args.sc.k, false);
  };
  const auto next_k = [&](int i) {
    copy_k(i, AHEAD - 1, found);
    if (i + 1 < mine) found = find_key<true>(a, c.b, c.shift, slice_key(i + 1) + (lane & (KEYS - 1)));
  };
  const auto copy_v = [&](int i) { copy(i, a.p.v, args.sc.v, true); };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    if (i & 1) copy_v(i / 2);
    else copy_k(i / 2, i / 2, first[i / 2]);
  }
  found = first[AHEAD];

#pragma unroll
  for (int i = 0; i < 4 * NR; ++i)
    if (i < 2 * NR || a.warp_heads) put_query(a.warp_heads ? i : warp + kWarps * i, qw[i]);
  if (a.warp_heads) {
#pragma unroll
    for (int i = 0; i < 4 * NR; ++i) get_query(4 * NR + i, qw[i]);
#pragma unroll
    for (int i = 0; i < 4 * NR; ++i) put_query(4 * NR + i, qw[i]);
  }
  float o[STEPS][NR][4] = {}, m[2 * MT], l[2 * MT], rf[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) m[i] = -INFINITY, l[i] = 0.f;
  __syncthreads();   // the queries are there
#pragma unroll
  for (int j = 0; j < 2 * MT; ++j) rf[j] = j < NR ? lds_f(sf + 4 * (8 * j + g)) : 0.f;
  uint32_t q[NR == 1 ? STEPS : 1][4];   // one tile of rows stays in registers
  const uint32_t qa = sq + ((lane & 7) + (NR > 1 ? 8 * (lane >> 3 & 1) : 0)) * QPITCH + (NR > 1 ? lane >> 4 : lane >> 3 & 1) * 16;
  if constexpr (NR == 1) {
#pragma unroll
    for (int x = 0; x < STEPS; x += 2) {
      uint32_t r[4];   // dims 16 x .. + 31 of rows 0..7
      ldm4(r, sq + (lane & 7) * QPITCH + (lane >> 3) * 16 + x * 32);
      q[x][0] = r[0]; q[x][2] = r[1]; q[x + 1][0] = r[2]; q[x + 1][2] = r[3];
      q[x][1] = q[x][3] = q[x + 1][1] = q[x + 1][3] = 0;
    }
  }
  float unit[2 * MT];   // of the rows' weights p sv: powers of two that no weight has passed by more than 2^kLag
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) unit[i] = kLeastUnit;
  const uint32_t ka = ring + (lane & 7) * DH + ((lane >> 3) ^ key_swap<DH>(lane & 7)) * 16;             // 8 keys, 64 dims
  const int vk = (lane >> 2 & 3) * 2 + (lane & 1) + (lane >> 1 & 1) * 8;
  const uint32_t va = ring + vk * DH + ((lane >> 4) ^ key_swap<DH>(vk)) * 16;                           // 16 keys, 32 dims
  int use = 0;       // slot of the slice at hand
  for (int i = 0; i < mine; ++i) {
    cp_wait<SLOTS - 1>();
    __syncwarp();
    float s[MT][2 * KT][4] = {};
#pragma unroll
    for (int x = 0; x < STEPS; x += 4) {
      uint32_t kk[2 * KT][4];
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n) ldm4(kk[n], (ka ^ ((x * 16 & 64) ^ (n & 1 ? ODD : 0))) + use * SLOT + n * 8 * DH + (x * 16 & ~127));
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        uint32_t qq[MT][4];
        if constexpr (NR > 1)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) ldm4(qq[mt], qa + mt * 16 * QPITCH + (x + y) * 32);
#pragma unroll
        for (int n = 0; n < 2 * KT; ++n) {
          uint32_t b0, b1;
          e4m3_f16x4(kk[n][y], &b0, &b1);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) mma16816h(s[mt][n], NR > 1 ? qq[mt] : q[NR == 1 ? x + y : 0], b0, b1);
        }
      }
    }
    float2 ks[2 * KT];   // the keys' scales
#pragma unroll
    for (int n = 0; n < 2 * KT; ++n) ks[n] = lds_f2(ring + use * SLOT + SCALES + 32 * n + 8 * t);
    use = use + 1 == SLOTS ? 0 : use + 1;
    const uint32_t bits = (uint32_t)seen & (0xffffffffu >> (32 - KEYS));
    seen >>= KEYS;
    __syncwarp();   // read by all: the slot may be filled again
    if constexpr (SLOTS & 1) copy_v(i + AHEAD - 1);
    else next_k(i + AHEAD);

    // scores, base 2; hidden keys
    const int key = slice_key(i);
    const bool mixed = (a.causal && key + KEYS - 1 > c.first_pos) || (a.window > 0 && key <= c.last_pos - a.window);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n)
#pragma unroll
        for (int e = 0; e < (NR > 1 ? 4 : 2); ++e) {
          const float v = s[mt][n][e] * (rf[2 * mt + (e >> 1)] * (e & 1 ? ks[n].y : ks[n].x));   // a large query's factor and a small scale first
          s[mt][n][e] = max_nan(v, kLeast);
        }
    if (mixed || bits != (0xffffffffu >> (32 - KEYS))) {
#pragma unroll
      for (int j = 0; j < (NR > 1 ? 2 * MT : 1); ++j) {   // rows g + 8 j
        int from = 0, end_key = c.k1;
        if (mixed) {
          const int pos = c.s.len - c.s.n - c.shift + (int)a.by_group.div(c.r0 + 8 * j + g);
          if (a.causal) end_key = pos + 1;
          if (a.window > 0) from = pos - a.window + 1;
        }
#pragma unroll
        for (int n = 0; n < 2 * KT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int k = 8 * n + 2 * t + e;
            if (!(bits >> k & 1) || (key + k < from && key + k >= a.sinks) || key + k >= end_key) s[j >> 1][n][2 * (j & 1) + e] = -INFINITY;
          }
      }
    }
    float f[2 * MT];
    bool grew = false;
#pragma unroll
    for (int j = 0; j < (NR > 1 ? 2 * MT : 1); ++j) {
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n) top = fmaxf(top, fmaxf(s[j >> 1][n][2 * (j & 1)], s[j >> 1][n][2 * (j & 1) + 1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      f[j] = 1.f;
      if (top > m[j] + kLag) {
        f[j] = ex2_approx(m[j] - top);
        m[j] = top;
        grew = true;
      }
      const float mm = m[j] == -INFINITY ? 0.f : m[j];
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < 2 * KT; ++n) {
        float* v = s[j >> 1][n] + 2 * (j & 1);
        v[0] = ex2_approx(v[0] - mm);
        v[1] = ex2_approx(v[1] - mm);
        sum += v[0] + v[1];
      }
      l[j] = l[j] * f[j] + sum;
    }

    cp_wait<SLOTS - 1>();
    __syncwarp();
    // weights p sv, of which a power of two, the row's unit, goes before the sums
#pragma unroll
    for (int k = 0; k < 2 * KT; ++k) {
      const float2 w = lds_f2(ring + use * SLOT + SCALES + 32 * k + 8 * t);
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        float* v = s[n >> 1][k] + 2 * (n & 1);   // 0 times what a row does not see is 0
        v[0] = v[0] == 0.f ? 0.f : v[0] * w.x;
        v[1] = v[1] == 0.f ? 0.f : v[1] * w.y;
      }
    }
    float most[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      most[n] = 0.f;
#pragma unroll
      for (int k = 0; k < 2 * KT; ++k) most[n] = fmaxf(most[n], fmaxf(s[n >> 1][k][2 * (n & 1)], s[n >> 1][k][2 * (n & 1) + 1]));
      grew |= most[n] > unit[n] * (1 << (int)kLag);
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        float top = most[n];
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float held = unit[n] * f[n], all = fmaxf(fmaxf(top, held), kLeastUnit);   // in the new maximum's terms
        const float now = __uint_as_float(min((__float_as_uint(all) + 0x7fffffu) & 0xff800000u, 254u << 23)), kept = held / now;
        unit[n] = now;
        const float f0 = __shfl_sync(0xffffffffu, kept, 8 * t), f1 = __shfl_sync(0xffffffffu, kept, 8 * t + 4);
#pragma unroll
        for (int y = 0; y < STEPS; ++y) {
          o[y][n][0] *= f0;
          o[y][n][1] *= f1;
          o[y][n][2] *= f0;
          o[y][n][3] *= f1;
        }
      }
    }
    // as two f16: the upper 11 bits and the rest
    uint32_t hi[NR][2 * KT], lo[NR][2 * KT];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const float per_unit = __uint_as_float(((254u + kWeightBits) << 23) - __float_as_uint(unit[n]));   // 2^kWeightBits / unit
#pragma unroll
      for (int k = 0; k < 2 * KT; ++k) {
        const float p0 = s[n >> 1][k][2 * (n & 1)] * per_unit, p1 = s[n >> 1][k][2 * (n & 1) + 1] * per_unit;
        const float h0 = __uint_as_float(__float_as_uint(p0) & 0xffffe000u), h1 = __uint_as_float(__float_as_uint(p1) & 0xffffe000u);
        hi[n][k] = pack_f16(h0, h1);
        lo[n][k] = pack_f16(p0 - h0, p1 - h1);
      }
    }
    // Where rows see different keys, a value that one of them does not see must not reach it, not even as 0 times NaN:
    // NaN codes of such a slice are left out here and added row by row below.
    bool odd = false;
    if (mixed) {
      uint32_t any = 0;
#pragma unroll 4
      for (int x = lane; x < KEYS * DH / 16; x += 32) {
        const uint4 w = lds16(ring + use * SLOT + x * 16);
        any |= nan_bits(w.x) | nan_bits(w.y) | nan_bits(w.z) | nan_bits(w.w);
      }
      odd = __any_sync(0xffffffffu, any != 0);
    }
#pragma unroll
    for (int x = 0; x < STEPS; x += 2)
#pragma unroll
      for (int u = 0; u < KT; ++u) {
        uint32_t v[4];   // dims 16 x + g, 16 x + g + 8; the next sixteen dims
        ldm_t8(v, (va ^ (x * 16 & (DH == 64 ? 32 : 96))) + use * SLOT + u * 16 * DH + (DH == 64 ? 0 : x * 16 & ~127));
        if (odd) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] &= ~nan_bytes(v[j]);
        }
        uint32_t fr[2][4];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          e4m3_f16x4(v[2 * y], &fr[y][0], &fr[y][2]);
          e4m3_f16x4(v[2 * y + 1], &fr[y][1], &fr[y][3]);
#pragma unroll
          for (int n = 0; n < NR; ++n) mma16816h(o[x + y][n], fr[y], hi[n][2 * u], hi[n][2 * u + 1]);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int n = 0; n < NR; ++n) mma16816h(o[x + y][n], fr[y], lo[n][2 * u], lo[n][2 * u + 1]);
      }
    if (odd) {
#pragma unroll 1
      for (int k = 0; k < KEYS; ++k) {
        if (!(bits >> k & 1)) continue;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const int r = 8 * n + 2 * t;
          const bool see0 = row_sees<true>(a, c, r, key + k), see1 = row_sees<true>(a, c, r + 1, key + k);
          const uint32_t from = ring + use * SLOT + k * DH + g;
#pragma unroll
          for (int x = 0; x < STEPS; ++x) {
            const uint32_t at = from + (x ^ key_swap<DH>(k)) * 16;
            const bool bad0 = (lds_u8(at) & 0x7f) == 0x7f, bad1 = (lds_u8(at + 8) & 0x7f) == 0x7f;
            if (bad0 && see0) o[x][n][0] = NAN;
            if (bad0 && see1) o[x][n][1] = NAN;
            if (bad1 && see0) o[x][n][2] = NAN;
            if (bad1 && see1) o[x][n][3] = NAN;
          }
        }
      }
    }
    use = use + 1 == SLOTS ? 0 : use + 1;
    __syncwarp();   // read by all: the slot may be filled again
    if constexpr (SLOTS & 1) next_k(i + AHEAD);
    else copy_v(i + AHEAD);
  }

  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    l[j] += __shfl_xor_sync(0xffffffffu, l[j], 1);
    l[j] += __shfl_xor_sync(0xffffffffu, l[j], 2);
  }
  // the warps' sums, scaled to common maxima, to where the ring was
  if (t == 0) {
#pragma unroll
    for (int j = 0; j < NR; ++j) end->m[warp][8 * j + g] = m[j], end->l[warp][8 * j + g] = l[j];
  }
  __syncthreads();
  if (!EVEN && a.clustered) cluster_arrive();   // the ring is free: others may send their shares
  const bool alone = !EVEN && a.warp_heads;
  if (!alone) common_rows(end);
  float* so = reinterpret_cast<float*>(smem) + warp * (S::kBytes / 4);
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int r = 8 * n + 2 * t;
    const float u = unit[n] * (1.f / (1 << kWeightBits)), u0 = __shfl_sync(0xffffffffu, u, 8 * t), u1 = __shfl_sync(0xffffffffu, u, 8 * t + 4);
    const float f0 = alone ? u0 : u0 * weight(end->m[warp][r], common_max(end, r));
    const float f1 = alone ? u1 : u1 * weight(end->m[warp][r + 1], common_max(end, r + 1));
    float* dst = so + r * S::kPitch + g;
#pragma unroll
    for (int x = 0; x < STEPS; ++x) {
      dst[16 * x] = o[x][n][0] * f0;
      dst[16 * x + S::kPitch] = o[x][n][1] * f1;
      dst[16 * x + 8] = o[x][n][2] * f0;
      dst[16 * x + 8 + S::kPitch] = o[x][n][3] * f1;
    }
  }
  if (alone) {   // the warp's rows are its own
    __syncwarp();
    for (int gr = 0; gr < S::kGroups; ++gr) {
      const int r = S::row(gr, lane), d = S::dim(gr, lane);
      if (r < c.rows) put_row<BF16>(a, c, r, d, *reinterpret_cast<const float4*>(so + r * S::kPitch + d), end->m[warp][r], end->l[warp][r], true);
    }
    return;
  }
  __syncthreads();
  if constexpr (!EVEN) {
    finish<BF16, DH, 8 * NR>(a, c, reinterpret_cast<const float*>(smem), end, reinterpret_cast<float4*>(smem + (EXTRA ? RING : kWarps * S::kBytes)));
    return;
  } else {
#pragma unroll 2
    for (int gr = warp; gr < S::kGroups; gr += kWarps) {
      const int r = S::row(gr, lane), d = S::dim(gr, lane);
      const float* from = reinterpret_cast<const float*>(smem) + r * S::kPitch + d;
      float4 y = *reinterpret_cast<const float4*>(from);
#pragma unroll
      for (int w = 1; w < kWarps; ++w) {
        const float4 z = *reinterpret_cast<const float4*>(from + w * (S::kBytes / 4));
        y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
      }
      if (r >= c.rows) continue;
      const float2 ml = end->ml[r];
      if (part == 0) {
        put_row<BF16>(a, c, r, d, y, ml.x, ml.y, true);
      } else {
        const int64_t row = (int64_t)(2 * even_cta(blockIdx.x, blockIdx.y, blockIdx.z) + part - 1) * (8 * NR) + r;
        *reinterpret_cast<float4*>(a.part_o + row * DH + d) = y;
        if (d == 0) a.part_ml[row] = ml;
      }
    }
  }
  }
}

// Joins the rows of the sequence that begins in part blockIdx.x and goes on behind it: one warp 64 dims of a row, its halves the pieces in turn, eight of
// them requested together. A CTA's first piece of two is of the sequence from before, its second of the one that begins with it.
// blockIdx.z: the block of rows and four rows of it.
template <int DH, int NR>
__global__ void __launch_bounds__(kThreads) paged_join8_kernel(const PagedAttn8Args args) {
  const PagedAttnArgs& a = args.a;
  // No early start for the kernel behind it: where this one's CTAs are still there, an SM does not take as many of the next attention's as it
  // could, and the one wave of those becomes two (64 x 4000 keys of 32 heads over 8 of 128, call after call: 137 us against 96 with one f16 a weight).
  pdl_wait();
  constexpr int FOURS = 8 * NR / kWarps;
  const int head = blockIdx.y / (DH / 64), column = blockIdx.y % (DH / 64), block = blockIdx.z / FOURS;
  const auto cta = [&](int part) { return (part * a.p.n_kv + head) * a.row_blocks + block; };
  const int2 span = args.spans[cta(blockIdx.x)];
  if (span.x < 0) return;
  Piece c;
  c.s = seq_rows(a.p, span.x);
  c.kvh = head;
  c.r0 = block * 8 * NR;
  c.rows = min(8 * NR, c.s.n * a.group - c.r0);
  const int r = blockIdx.z % FOURS * kWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (r >= c.rows) return;
  const int from = blockIdx.x, n = span.y - from + 1, d = lane % 16 * 4 + 64 * column;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  float top = -INFINITY, sum = 0.f;
  constexpr int AT_ONCE = 8;
  for (int i0 = lane / 16; i0 < n; i0 += 2 * AT_ONCE) {
    float2 ml[AT_ONCE];
    float4 y[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int i = i0 + 2 * k;
      ml[k] = make_float2(-INFINITY, 0.f);
      y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < n) {
        const int64_t row = (int64_t)(2 * cta(from + i) + (i == 0 ? 1 : 0)) * (8 * NR) + r;
        ml[k] = a.part_ml[row];
        y[k] = *reinterpret_cast<const float4*>(a.part_o + row * DH + d);
      }
    }
    float now = top;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) now = fmaxf(now, ml[k].x);
    const float f = weight(top, now);
    top = now;
    sum *= f;
    x.x *= f; x.y *= f; x.z *= f; x.w *= f;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const float w = weight(ml[k].x, top);
      sum += ml[k].y * w;
      x.x += y[k].x * w; x.y += y[k].y * w; x.z += y[k].z * w; x.w += y[k].w * w;
    }
  }
  __syncwarp();
  const float other = __shfl_xor_sync(0xffffffffu, top, 16), most = fmaxf(top, other), f = weight(top, most);
  sum *= f;
  x.x *= f; x.y *= f; x.z *= f; x.w *= f;
  sum += __shfl_xor_sync(0xffffffffu, sum, 16);
  x.x += __shfl_xor_sync(0xffffffffu, x.x, 16);
  x.y += __shfl_xor_sync(0xffffffffu, x.y, 16);
  x.z += __shfl_xor_sync(0xffffffffu, x.z, 16);
  x.w += __shfl_xor_sync(0xffffffffu, x.w, 16);
  if (lane < 16) put_row<BF16>(a, c, r, d, x, most, sum, true);
}

template <int DH, int NR>
cudaError_t launch8(const PagedAttn8Args& a, cudaStream_t s) {
  static OncePerDevice once, once_even;
  if (!a.parts) {
    const cudaError_t e = launch_attn(once, paged_attn8_kernel<DH, NR, false>, smem8<DH, NR>(a.a.warp_heads ? kWarps : 1), smem8<DH, NR>(kWarps), a.a, a, s);
    if (e != cudaSuccess || a.a.pieces == 1 || a.a.clustered) return e;
    const dim3 grid((unsigned)a.a.n_heads * a.a.p.max_new, DH / 64, a.a.p.n_seqs);
    return launch_k(paged_join_kernel<BF16, DH>, grid, kThreads, 0, s, a.a);
  }
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const auto kernel = paged_attn8_kernel<DH, NR, true>;
  e = (cudaError_t)once_even.run(dev, [&] {
    return (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)even_smem<DH, NR>(kEvenSeqs));
  });
  if (e != cudaSuccess) return e;
  const dim3 grid(a.parts, a.a.p.n_kv, a.a.row_blocks);
  e = launch_k(kernel, grid, dim3(kThreads), even_smem<DH, NR>(a.a.p.n_seqs), s, a);
  return e != cudaSuccess ? e : launch_k(paged_join8_kernel<DH, NR>, dim3(a.parts, a.a.p.n_kv * (DH / 64), a.a.row_blocks * (8 * NR / kWarps)), kThreads, 0, s, a);
}

template <int DH>
AttnFit8 fit8() {
  if constexpr (DH == 256)
    return {{ctas8<DH, 1>(), ctas8<DH, 2>(), 0}, {smem8<DH, 1>(kWarps), smem8<DH, 2>(kWarps), 0}, {chunk_keys<DH, 1>(), chunk_keys<DH, 2>(), 0}};
  else
    return {{ctas8<DH, 1>(), ctas8<DH, 2>(), ctas8<DH, 4>()}, {smem8<DH, 1>(kWarps), smem8<DH, 2>(kWarps), smem8<DH, 4>(kWarps)},
            {chunk_keys<DH, 1>(), chunk_keys<DH, 2>(), chunk_keys<DH, 4>()}};
}

template <int DH>
cudaError_t launch_dh8(const PagedAttn8Args& a, cudaStream_t s) {
  if (a.a.row_tiles == 1) return launch8<DH, 1>(a, s);
  if constexpr (DH == 256) return launch8<DH, 2>(a, s);   // 16 rows at most
  else return a.a.row_tiles == 2 ? launch8<DH, 2>(a, s) : launch8<DH, 4>(a, s);
}

int64_t even_ctas(const PagedAttn8Args& a) { return (int64_t)a.parts * a.a.p.n_kv * a.a.row_blocks; }
// Bytes of the two pieces that each CTA can have: values, maxima and sums; and of the spans.
int64_t attn8_bytes(const PagedAttn8Args& a) {
  return a.parts ? even_ctas(a) * (2 * 8 * a.a.row_tiles * (a.a.p.dh + 2) * 4 + 8) + 8 : attn_bytes(a.a);
}

// Into how many parts the chunks are cut; 0: not evenly. Evenly, a call costs about 6 us more (the sums, a second kernel) and a CTA about 4 us for each further sequence, and it gains what SMs idle otherwise: pieces in waves of which the last
// is part-filled, and lengths that differ. So the CTAs' shares have to last some 24 us at the rates (keys a microsecond and CTA) at
// which they come, and to be half a sequence long at least. In us, evenly / as attn_plan has it, for equal lengths and for a
// quarter of the longest and more (which of the two the host cannot know: batches of several new tokens pay 6 to 7% where lengths are
// equal for 20% where they are not):
//   64 x 4000 keys, 32 heads over 8 of 128:  96 / 111 and 67 / 79      64 x 2000, the same:            54 / 67 and 42 / 47
//   64 x 4000, 4 new tokens, 8 over 1 of 256: 67 / 63 and 50 / 64      16 x 4000, 8 new, 32 / 8 of 128: 74 / 70 and 55 / 69
//   32768 and 131071, 32 over 8 of 128:      67 / 80                   64 x 1000, 24 heads of 64:      53 / 48 and 41 / 38
//   64 x 4000, 8 over 1 of 256:              34 / 29 and 29 / 27       16 x 1000, 32 / 8 of 128:       19 / 13 and 17 / 12
int even_parts(const PagedAttnArgs& a, const uad_kv_seqs* s, int ctas) {
  const int64_t all = s->max_len > 0 && s->max_len < a.p.capacity ? s->max_len : a.p.capacity;
  const int64_t near = (int64_t)a.window + a.sinks + a.p.max_new - 1, keys = a.window > 0 && near < all ? near : all;
  const int64_t each = (int64_t)a.p.n_kv * a.row_blocks, slots = (int64_t)kAttnSms * ctas, parts = slots / each;
  const int rate = a.p.dh == 256 ? (a.row_tiles == 1 ? 36 : 24) : a.p.dh == 128 ? (a.row_tiles == 1 ? 48 : a.row_tiles == 2 ? 30 : 14)
                                                                                : (a.row_tiles == 1 ? 72 : a.row_tiles == 2 ? 50 : 30);
  if (a.warp_heads || a.p.n_seqs > kEvenSeqs || a.p.n_seqs > 2 * parts) return 0;
  if (((int64_t)a.p.capacity / 64 + 1) * a.p.n_seqs >= (1ll << 30)) return 0;   // the sums stay within 31 bits
  return each * a.p.n_seqs * keys >= slots * 24 * rate ? (int)parts : 0;
}

int attn8_args(const uad_kv_pages8* pages, const uad_kv_seqs* seqs, const uad_attn* t, int sinks, bool device, PagedAttn8Args* a) {
  if (!t) return UAD_EINVAL;
  int rc = pages8_args(pages, seqs, t->n_rows, device, &a->a.p, &a->sc);
  if (rc) return rc;
  const uad_kv_pages& g = pages->pages;
  // offsets in 32 bits: of codes in units of the strides (which are 32 bits themselves), of scales in elements
  const int64_t any = g.page_stride | g.slot_stride | g.head_stride, unit = std::min<int64_t>(any & -any, 1ll << 31), top = 0xffffffffll;
  const int blocks = (g.page_size + pages->block - 1) / pages->block;
  if (g.page_stride / unit > top || g.slot_stride / unit > top || g.head_stride / unit > top || pages->scale_page_stride > top ||
      pages->scale_block_stride > top || pages->scale_head_stride > top)
    return UAD_EINVAL;
  const auto last = [&](int64_t page, int64_t inner, int n, int64_t head) {   // below 2^31 2^32 each
    return (double)(g.n_pages - 1) * page + (double)(n - 1) * inner + (double)(g.n_kv_heads - 1) * head;
  };
  if (last(g.page_stride / unit, g.slot_stride / unit, g.page_size, g.head_stride / unit) >= (double)top ||
      last(pages->scale_page_stride, pages->scale_block_stride, blocks, pages->scale_head_stride) >= (double)top)
    return UAD_EINVAL;
  a->unit = (uint32_t)unit;
  a->page_units = (uint32_t)(g.page_stride / unit); a->slot_units = (uint32_t)(g.slot_stride / unit); a->head_units = (uint32_t)(g.head_stride / unit);
  a->scale_page = (uint32_t)pages->scale_page_stride; a->scale_block = (uint32_t)pages->scale_block_stride;
  a->scale_head = (uint32_t)pages->scale_head_stride;
  const int dh = a->a.p.dh;
  const AttnFit8 fit = dh == 64 ? fit8<64>() : dh == 128 ? fit8<128>() : fit8<256>();
  rc = attn_split(seqs, t, sinks, device, &fit, &a->a);
  if (rc || a->a.p.n_seqs == 0 || a->a.p.n_rows == 0) return rc;
  const int ctas = fit.ctas[a->a.row_tiles == 4 ? 2 : a->a.row_tiles - 1];
  a->parts = even_parts(a->a, seqs, ctas);
  if (a->parts && a->a.window > 0) {   // only where a call without the window does, whose workspace is to be enough
    PagedAttnArgs all = a->a;
    uad_attn u = *t;
    u.window = 0;
    attn_split(seqs, &u, 0, false, &fit, &all);
    a->parts = even_parts(all, seqs, ctas) ? a->parts : 0;
  }
  return UAD_OK;
}

}  // namespace
}  // namespace uad

using namespace uad;

extern "C" {

int64_t uad_paged_attention8_workspace(const uad_kv_pages8* pages, const uad_kv_seqs* seqs, const uad_attn* attn, int32_t sinks) {
  PagedAttn8Args a{};
  const int rc = attn8_args(pages, seqs, attn, sinks, false, &a);
  // What a call with a window needs may be what pieces of attn_plan's need: the larger one, so that one without is enough.
  return rc ? rc : std::max(attn8_bytes(a), attn_bytes(a.a));
}

int uad_paged_attention8(const uad_kv_pages8* pages, const uad_kv_seqs* seqs, const uad_attn* attn, int32_t sinks, void* workspace,
                         size_t workspace_bytes, int32_t* status, void* stream) {
  PagedAttn8Args a{};
  const int rc = attn8_args(pages, seqs, attn, sinks, true, &a);
  if (rc) return rc;
  if (a.a.p.n_seqs == 0 || a.a.p.n_rows == 0) return UAD_OK;
  a.a.p.status = status;
  const int64_t need = attn8_bytes(a);
  if (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 || workspace_bytes < (size_t)need)) return UAD_EINVAL;
  if (a.parts) {
    a.a.part_o = static_cast<float*>(workspace);
    a.a.part_ml = reinterpret_cast<float2*>(a.a.part_o + even_ctas(a) * 2 * 8 * a.a.row_tiles * a.a.p.dh);
    a.spans = reinterpret_cast<int2*>(a.a.part_ml + even_ctas(a) * 2 * 8 * a.a.row_tiles);
  } else if (!attn_workspace(&a.a, workspace, workspace_bytes)) {
    return UAD_EINVAL;
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return launched(a.a.p.dh == 64 ? launch_dh8<64>(a, s) : a.a.p.dh == 128 ? launch_dh8<128>(a, s) : launch_dh8<256>(a, s));
}

}  // extern "C"
