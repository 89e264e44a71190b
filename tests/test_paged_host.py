"""CPU checks of the paged cache's and the 4-bit projection's host side: structures, frequencies, weight rounding, page
division, and the refusals of the C entries and of the binding (no GPU is touched)."""
import ctypes as C
import os
import shutil
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_37772_gb300", "csrc")


def test_structures_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = ["uad_kv_pages", "uad_kv_seqs", "uad_rope", "uad_kv_rows", "uad_attn"]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "uad.h"', "int main(void) {"]
    for s in names:
        lines.append(f'  printf("{s} size %zu\\n", sizeof({s}));')
        lines += [f'  printf("{s} {f} %zu\\n", offsetof({s}, {f}));' for f, _ in getattr(uad, s)._fields_]
    lines += [f'  printf("const {k} %d\\n", (int)({k}));' for k in ("UAD_KV_BAD_PAGE", "UAD_KV_BAD_SEQ", "UAD_W4_MAX_ROWS")]
    (tmp_path / "p.c").write_text("\n".join(lines) + "\n  return 0;\n}\n")
    subprocess.run([cc, "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(tmp_path / "p.c"), "-o", str(tmp_path / "p")], check=True)
    for line in subprocess.run([str(tmp_path / "p")], check=True, capture_output=True, text=True).stdout.splitlines():
        s, f, n = line.split()
        want = getattr(uad, f) if s == "const" else C.sizeof(getattr(uad, s)) if f == "size" else getattr(getattr(uad, s), f).offset
        assert int(n) == want, line


def test_page_division(tmp_path):
    """Every page size up to 70000 at the borders of its pages, near 2^31 too, and small positions one by one."""
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no host compiler")
    (tmp_path / "t.cc").write_text(r"""
#include "fast_div.h"
#include <cstdio>
#include <initializer_list>
int main() {
  for (uint32_t d = 1; d <= 70000; ++d) {
    const uad::FastDiv f(d);
    const uint32_t top = 0x7fffffffu, last = top / d;
    for (uint32_t q : {0u, 1u, 2u, last / 3, last / 2, last - (last > 0), last})
      for (int i = -1; i <= 1; ++i) {
        const int64_t n = (int64_t)q * d + i;
        if (n >= 0 && n <= top && f.div((uint32_t)n) != (uint32_t)n / d) return printf("%u / %u\n", (uint32_t)n, d), 1;
      }
    if (f.div(top) != top / d) return printf("top / %u\n", d), 1;
    if (d < 300)
      for (uint32_t n = 0; n < 5000; ++n)
        if (f.div(n) != n / d) return printf("%u / %u\n", n, d), 1;
  }
  return 0;
}
""")
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", CSRC, "-o", str(tmp_path / "t"), str(tmp_path / "t.cc")], check=True)
    r = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("theta,dim", [(10000.0, 256), (500000.0, 64), (1.0, 16), (0.5, 32)])
def test_rope_frequencies_are_fractions_of_a_turn(theta, dim):
    r = uad.rope(theta, dim)
    assert r.dim == dim
    for i in range(dim // 2):
        turns = theta ** (-2.0 * i / dim) / (2 * np.pi)
        got = r.turn[i] / 2.0 ** 64
        assert abs(got - turns % 1.0) <= 4 * 2.0 ** -53 * max(1.0, turns)
    assert all(t == 0 for t in r.turn[dim // 2:])


@pytest.mark.parametrize("theta,dim", [(10000.0, 0), (10000.0, 24), (10000.0, 272), (0.0, 64), (-1.0, 64), (float("inf"), 64), (float("nan"), 64)])
def test_rope_refusals(theta, dim):
    with pytest.raises(uad.UADError):
        uad.rope(theta, dim)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("symmetric", [False, True])
def test_quantize_w4(group, symmetric):
    rng = np.random.default_rng(group)
    w = (rng.normal(size=(256, 11)) * 0.02).astype(np.float32)
    w[:group, 0] = 0            # a group of zeros
    w[:group, 1] = 0.25         # of one value
    w[group:, 2] = np.abs(w[group:, 2])
    q, s, z = uad.quantize_w4(w, group, symmetric)
    scale = (s.astype(np.uint32) << 16).view(np.float32)
    back = paged.dequantize(q, scale, z).T
    step = np.repeat(scale.T, group, axis=0)
    assert np.all(back[:group, 0] == 0)
    # half a step of the nearest multiple; a bf16 scale that was rounded down by up to 2^-8 leaves the ends of the range up to
    # 15 * 2^-8 < 0.06 steps outside; the zero point's own rounding moves the range by half a step
    assert np.all(np.abs(back - w) <= step * (0.5 + 0.06 + (0 if symmetric else 0.5)))
    if symmetric:
        assert z is None and (q & 15).min() >= 1 and (q >> 4).min() >= 1
    else:
        assert z.max() <= 15


def test_quantize_w4_refusals():
    for w, group in [(np.zeros((64, 3)), 16), (np.zeros((96, 3)), 64), (np.full((64, 3), np.nan), 64), (np.full((64, 3), np.inf), 64)]:
        with pytest.raises(uad.UADError):
            uad.quantize_w4(w, group)


# ---- refusals of the C entries: nothing is dereferenced -------------------------------------------------------------------

P = 1 << 20   # an aligned address that no call may look at


def pages(**kw):
    return uad.uad_kv_pages(**(dict(k=P, v=P, page_stride=16 * 128, slot_stride=128, head_stride=64, dtype=1, n_pages=4, page_size=16,
                                    n_kv_heads=2, head_dim=64) | kw))


def seqs(**kw):
    return uad.uad_kv_seqs(**(dict(table=P, len=P, start=P, table_stride=8, n_seqs=3, table_width=8, max_new=1, max_len=0) | kw))


def rows(**kw):
    return uad.uad_kv_rows(**(dict(q=P, k=P, v=P, q_stride=256, k_stride=128, v_stride=128, q_out=P, q_out_stride=256, dtype=1, n_heads=4,
                                   n_rows=3) | kw))


def attn(**kw):
    return uad.uad_attn(**(dict(q=P, out=P, lse=P, q_stride=256, out_stride=256, n_heads=4, n_rows=3, causal=1) | kw))


BAD_PAGES = [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(dtype=2), dict(dtype=-1), dict(head_dim=32), dict(head_dim=96),
             dict(head_dim=512), dict(n_pages=0), dict(page_size=0), dict(page_size=65537), dict(n_kv_heads=0), dict(n_kv_heads=1025),
             dict(page_stride=0), dict(slot_stride=-128), dict(head_stride=0), dict(page_stride=1028), dict(slot_stride=132), dict(head_stride=66)]
BAD_SEQS = [dict(n_seqs=-1), dict(n_seqs=65536), dict(max_new=0), dict(max_len=-1), dict(table_width=0), dict(table_stride=7),
            dict(table_width=1 << 27, table_stride=1 << 27), dict(table=None), dict(len=None), dict(start=None, n_seqs=4)]
BAD_ROWS = [dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(q=None, n_heads=0, k=None, v=None), dict(n_heads=0), dict(n_heads=-1),
            dict(dtype=2), dict(q=P + 4), dict(k=P + 4), dict(v=P + 4), dict(q_out=P + 4), dict(q_stride=257), dict(k_stride=-128), dict(v_stride=129),
            dict(q_out_stride=260), dict(n_rows=-1)]
BAD_ATTN = [dict(q=None), dict(out=None), dict(q=P + 2), dict(out=P + 8), dict(lse=P + 2), dict(q_stride=-8), dict(out_stride=260), dict(n_heads=0),
            dict(n_heads=3), dict(n_heads=130), dict(causal=2), dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(n_rows=-1),
            dict(key_mask=P, mask_stride=-1)]


def call_append(p, s, r, rope=None):
    return uad.uad_kv_append(p, s, r, rope, None, None)


def call_attention(p, s, a, ws=None, n=0):
    return uad.uad_paged_attention(p, s, a, ws, n, None, None)


@pytest.mark.parametrize("kw", BAD_PAGES)
def test_bad_pages_are_refused(kw):
    assert call_append(pages(**kw), seqs(), rows()) == uad.UAD_EINVAL
    assert call_attention(pages(**kw), seqs(), attn()) == uad.UAD_EINVAL
    assert uad.uad_paged_attention_workspace(pages(**kw), seqs(), attn()) == uad.UAD_EINVAL


@pytest.mark.parametrize("kw", BAD_SEQS)
def test_bad_sequences_are_refused(kw):
    assert call_append(pages(), seqs(**kw), rows()) == uad.UAD_EINVAL
    assert call_attention(pages(), seqs(**kw), attn()) == uad.UAD_EINVAL


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_bad_rows_are_refused(kw):
    assert call_append(pages(), seqs(), rows(**kw)) == uad.UAD_EINVAL


@pytest.mark.parametrize("kw", BAD_ATTN)
def test_bad_attention_arguments_are_refused(kw):
    assert call_attention(pages(), seqs(), attn(**kw)) == uad.UAD_EINVAL


def test_null_structures_and_pages_that_are_no_gpu_memory():
    for a in ((None, seqs(), rows()), (pages(), None, rows()), (pages(), seqs(), None)):
        assert call_append(*a) == uad.UAD_EINVAL
    for a in ((None, seqs(), attn()), (pages(), None, attn()), (pages(), seqs(), None)):
        assert call_attention(*a) == uad.UAD_EINVAL
    host = np.zeros(1 << 16, np.uint8)
    at = (host.ctypes.data + 63) // 64 * 64
    assert call_append(pages(k=at, v=at), seqs(), rows()) == uad.UAD_EINVAL
    assert call_attention(pages(k=at, v=at), seqs(), attn()) == uad.UAD_EINVAL
    assert call_append(pages(), seqs(), rows(), uad.uad_rope(dim=128)) == uad.UAD_EINVAL   # wider than a head
    assert call_append(pages(), seqs(), rows(), uad.uad_rope(dim=0)) == uad.UAD_EINVAL


def test_empty_batches_are_answered_without_a_launch():
    assert call_append(pages(), seqs(n_seqs=0), rows()) == uad.UAD_OK
    assert call_append(pages(), seqs(), rows(n_rows=0)) == uad.UAD_OK
    assert call_attention(pages(), seqs(n_seqs=0), attn()) == uad.UAD_OK
    assert call_attention(pages(), seqs(), attn(n_rows=0)) == uad.UAD_OK


def test_workspace_sizes():
    """Host only, without tables; enough for what it grows with, and nothing per cached token."""
    s = seqs(table=None, len=None, start=None, table_width=100000, table_stride=100000, max_new=4)
    n = uad.uad_paged_attention_workspace(pages(), s, attn(n_rows=12))
    assert 0 <= n <= 64 << 20
    for kw in (dict(n_seqs=65535), dict(n_seqs=65535, max_new=16), dict(max_len=5)):
        big = seqs(table=None, len=None, start=None, table_width=100000, table_stride=100000, **kw)
        assert 0 <= uad.uad_paged_attention_workspace(pages(), big, attn(n_rows=70000)) <= 64 << 20


BAD_W4 = [dict(x=None), dict(q=None), dict(scale=None), dict(out=None), dict(M=0), dict(N=0), dict(K=0), dict(group=16), dict(group=256), dict(K=96),
          dict(x=P + 2), dict(q=P + 8), dict(scale=P + 1), dict(bias=P + 2), dict(out=P + 1), dict(N=1 << 30, K=1 << 11), dict(K=-64), dict(N=-1)]


def call_w4(x=P, q=P, scale=P, zero=None, bias=None, out=P, M=1, N=16, K=128, group=64):
    return uad.uad_linear_w4(x, q, scale, zero, bias, out, M, N, K, group, None)


@pytest.mark.parametrize("kw", BAD_W4)
def test_bad_projections_are_refused(kw):
    assert call_w4(**kw) == uad.UAD_EINVAL


def test_too_many_rows_and_weights_that_are_no_gpu_memory():
    assert call_w4(M=uad.UAD_W4_MAX_ROWS + 1) == uad.UAD_ETOOBIG
    assert call_w4(N=1, K=(1 << 30) + 128) == uad.UAD_EINVAL
    host = np.zeros(4096, np.uint8)
    assert call_w4(q=(host.ctypes.data + 63) // 64 * 64) == uad.UAD_EINVAL


def test_prefix_from_pages_needs_a_context():
    assert uad.uad_set_prefix_paged(None, 0, (uad.uad_kv_pages * 1)(), 1, None, 0) == uad.UAD_EINVAL


# ---- the binding stops malformed tensors before the call ----------------------------------------------------------------------


def test_binding_refuses_malformed_tensors():
    k = torch.zeros(4, 16, 2, 64)
    with pytest.raises(ValueError, match="one type"):
        uad.PagedCache(k, k[:3])
    with pytest.raises(ValueError, match="one type"):
        uad.PagedCache(k, k.double())
    with pytest.raises(ValueError, match="strides"):
        uad.PagedCache(k, torch.zeros(4, 2, 16, 64).transpose(1, 2))
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        uad.PagedCache(k.half(), k.half())
    with pytest.raises(ValueError, match="last dimension"):
        uad.PagedCache(torch.zeros(4, 16, 64, 2).transpose(2, 3), torch.zeros(4, 16, 64, 2).transpose(2, 3))
    with pytest.raises(ValueError, match="on the GPU"):
        uad.PagedCache(k, k)
    table, length = torch.zeros(3, 8, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="table: expected int32"):
        uad.Sequences(table.long(), length)
    with pytest.raises(ValueError, match="shape"):
        uad.Sequences(table[:2], length)
    with pytest.raises(ValueError, match="contiguous"):
        uad.Sequences(torch.zeros(8, 3, dtype=torch.int32).t(), length)
    with pytest.raises(ValueError, match="on the GPU"):
        uad.Sequences(table, length)
    x, q, s, out = torch.zeros(2, 128, dtype=torch.bfloat16), torch.zeros(5, 64, dtype=torch.uint8), torch.zeros(5, 2, dtype=torch.bfloat16), torch.zeros(2, 5)
    for bad in (dict(x=x.float()), dict(x=x[0]), dict(q=q[:, :32]), dict(q=q.char()), dict(scale=s.float()), dict(out=out.t()), dict(zero=s),
                dict(bias=torch.zeros(4)), dict()):
        with pytest.raises(ValueError):
            uad.linear_w4(**(dict(x=x, q=q, scale=s, out=out) | bad))


# ---- empty batches of long caches ---------------------------------------------------------------------------------------------


@pytest.mark.parametrize("max_len", [0, 5000])
@pytest.mark.parametrize("width", [256, 257, 313, 1 << 20])
def test_empty_batches_of_long_caches(width, max_len):
    """No sequences or no rows, over tables of 4096 tokens and more: no work to split, so no workspace and no launch. In a process of
    its own, which a division by zero would end."""
    code = f"""
import paper_2609_37772_gb300 as uad
P = 1 << 20
pages = uad.uad_kv_pages(k=P, v=P, page_stride=2048, slot_stride=128, head_stride=64, dtype=1, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64)
for dtype in (0, 1):
    pages.dtype = dtype
    for n_seqs, n_rows in ((0, 3), (0, 0), (3, 0)):
        for window in (0, 9000):
            seqs = uad.uad_kv_seqs(table=P, len=P, start=P, table_stride={width}, n_seqs=n_seqs, table_width={width}, max_new=2, max_len={max_len})
            attn = uad.uad_attn(q=P, out=P, lse=P, q_stride=256, out_stride=256, n_heads=4, n_rows=n_rows, causal=1, window=window)
            assert uad.uad_paged_attention_workspace(pages, seqs, attn) == 0
            assert uad.uad_paged_attention(pages, seqs, attn, None, 0, None, None) == 0
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr)


# ---- one workspace for layers with and without a window ------------------------------------------------------------------------


def workspace(heads, dtype, n_seqs, new, max_len, window, width=4096):
    hq, hkv, dh = heads
    p = pages(dtype=dtype, n_kv_heads=hkv, head_dim=dh, head_stride=dh, slot_stride=hkv * dh, page_stride=16 * hkv * dh)
    s = seqs(table=None, len=None, start=None, table_width=width, table_stride=width, n_seqs=n_seqs, max_new=new, max_len=max_len)
    return uad.uad_paged_attention_workspace(p, s, attn(n_heads=hq, n_rows=n_seqs * new, q_stride=hq * dh, out_stride=hq * dh, window=window))


def test_a_workspace_without_a_window_holds_for_every_window():
    """Fewer keys may be cut into more pieces: what they need stays within what all keys need."""
    assert workspace((8, 2, 64), 1, 32, 1, 2400, 2100) <= workspace((8, 2, 64), 1, 32, 1, 2400, 0)
    assert workspace((8, 1, 256), 0, 8, 4, 2350, 1714) <= workspace((8, 1, 256), 0, 8, 4, 2350, 0)
    rng = np.random.default_rng(0)
    heads = [(8, 1, 256), (4, 1, 128), (8, 2, 64), (24, 24, 64), (32, 8, 128), (4, 2, 64)]
    for _ in range(4000):
        h, dtype = heads[rng.integers(len(heads))], int(rng.integers(2))
        n_seqs, new = int(np.exp(rng.uniform(0, 6))), int(np.exp(rng.uniform(0, 4)))
        max_len = int(np.exp(rng.uniform(0, 11))) if rng.integers(4) else 0
        most = workspace(h, dtype, n_seqs, new, max_len, 0)
        for w in np.exp(rng.uniform(0, np.log(max_len or 65536), 6)).astype(int):
            assert 0 <= workspace(h, dtype, n_seqs, new, max_len, int(w)) <= most, (h, dtype, n_seqs, new, max_len, w)


# ---- queries rotated in place -----------------------------------------------------------------------------------------------


def test_queries_in_place_need_one_type_and_stride():
    """With another element size or stride a thread's output lies on what another thread has yet to read. (Without
    sequences a call whose arguments are sound is answered, and reaches no GPU.)"""
    for cache, row, out_stride, sound in ((1, 1, 256, True), (0, 0, 256, True), (1, 0, 256, False), (0, 1, 256, False), (1, 1, 512, False), (0, 0, 264, False)):
        r = rows(dtype=row, q=P, q_out=P, q_out_stride=out_stride)
        assert call_append(pages(dtype=cache), seqs(n_seqs=0), r) == (uad.UAD_OK if sound else uad.UAD_EINVAL)
        assert call_append(pages(dtype=cache), seqs(n_seqs=0), rows(dtype=row, q=P, q_out=P + (1 << 16), q_out_stride=out_stride)) == uad.UAD_OK
    assert call_append(pages(), seqs(n_seqs=0), rows(dtype=1, n_rows=1, q_out_stride=512)) == uad.UAD_OK   # the stride of one row says nothing
