"""CPU checks of the 8-bit cache, of windows with sinks and of the pages' bookkeeping: structures, the oracle's codes, refusals of the C
entries and of the binding (no GPU is touched)."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged8
from test_paged_host import BAD_ATTN, BAD_PAGES, BAD_ROWS, BAD_SEQS, P, attn, pages, rows, seqs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_structures_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "uad.h"', "int main(void) {"]
    for s in ("uad_kv_pages8", "uad_page_pool", "uad_kv_wanted"):
        lines.append(f'  printf("{s} size %zu\\n", sizeof({s}));')
        lines += [f'  printf("{s} {f} %zu\\n", offsetof({s}, {f}));' for f, _ in getattr(uad, s)._fields_]
    lines += [f'  printf("const {k} %d\\n", (int)({k}));' for k in ("UAD_DTYPE_E4M3", "UAD_KV_NO_ROOM", "UAD_KV_BAD_POOL")]
    (tmp_path / "p.c").write_text("\n".join(lines) + "\n  return 0;\n}\n")
    subprocess.run([cc, "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(tmp_path / "p.c"), "-o", str(tmp_path / "p")], check=True)
    for line in subprocess.run([str(tmp_path / "p")], check=True, capture_output=True, text=True).stdout.splitlines():
        s, f, n = line.split()
        want = getattr(uad, f) if s == "const" else C.sizeof(getattr(uad, s)) if f == "size" else getattr(getattr(uad, s), f).offset
        assert int(n) == want, line


def test_the_oracles_codes_are_those_of_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).double().numpy(), paged8.VALUES, equal_nan=True)
    x = torch.cat([torch.randn(20000, generator=torch.Generator().manual_seed(0)) * s for s in (1e-3, 0.02, 1.0, 90.0)]).clamp(-448, 448)
    finite = torch.from_numpy(paged8.VALUES[np.isfinite(paged8.VALUES)]).float()
    ties = (finite[:126] + finite[1:127]) / 2
    x = torch.cat([x, finite, ties, -ties])
    assert np.array_equal(paged8.encode(x.numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_the_oracles_scales():
    for top in (448.0, 448.0001, 447.9, 1.75, 1.7500001, 3.0, 1e-20, 3e38, 2.0 ** -90):
        s = paged8.scale_of(top)
        assert top <= 448 * s and (top > 448 * s / 2 or s == 2.0 ** -100)
    assert paged8.scale_of(0.0) == paged8.scale_of(1e-40) == 2.0 ** -100


def pages8(inner=None, **kw):
    p = pages(**(dict(dtype=2) | (inner or {})))
    return uad.uad_kv_pages8(**(dict(pages=p, k_scale=P, v_scale=P, scale_page_stride=2, scale_block_stride=2, scale_head_stride=1, block=16) | kw))


BAD_SCALES = [dict(k_scale=None), dict(v_scale=None), dict(k_scale=P + 2), dict(v_scale=P + 1), dict(block=0), dict(block=8), dict(block=48),
              dict(block=128), dict(scale_page_stride=0), dict(scale_block_stride=-1), dict(scale_head_stride=0)]


def call_append(p, s, r, rope=None):
    return uad.uad_kv_append8(p, s, r, rope, None, None)


def call_attention(p, s, a, sinks=0):
    return uad.uad_paged_attention8(p, s, a, sinks, None, 0, None, None)


@pytest.mark.parametrize("kw", BAD_SCALES)
def test_bad_scales_are_refused(kw):
    assert call_append(pages8(**kw), seqs(), rows()) == uad.UAD_EINVAL
    assert call_attention(pages8(**kw), seqs(), attn()) == uad.UAD_EINVAL
    assert uad.uad_paged_attention8_workspace(pages8(**kw), seqs(), attn(), 0) == uad.UAD_EINVAL


@pytest.mark.parametrize("kw", [kw for kw in BAD_PAGES if kw != dict(dtype=2)] + [dict(dtype=0), dict(dtype=1), dict(dtype=3)])
def test_bad_pages_are_refused(kw):
    # strides count bytes here: what breaks the rule of 16 bytes in bf16 breaks it in bytes too
    assert call_append(pages8(kw), seqs(), rows()) == uad.UAD_EINVAL
    assert call_attention(pages8(kw), seqs(), attn()) == uad.UAD_EINVAL


def test_other_types_do_not_take_codes():
    assert uad.uad_kv_append(pages(dtype=2), seqs(), rows(), None, None, None) == uad.UAD_EINVAL
    assert uad.uad_paged_attention_sinks(pages(dtype=2), seqs(), attn(window=3), 2, None, 0, None, None) == uad.UAD_EINVAL
    assert uad.uad_set_prefix_paged(None, 0, (uad.uad_kv_pages * 1)(pages(dtype=2)), 1, None, 0) == uad.UAD_EINVAL


@pytest.mark.parametrize("kw", BAD_SEQS)
def test_bad_sequences_are_refused(kw):
    assert call_append(pages8(), seqs(**kw), rows()) == uad.UAD_EINVAL
    assert call_attention(pages8(), seqs(**kw), attn()) == uad.UAD_EINVAL


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_bad_rows_are_refused(kw):
    assert call_append(pages8(), seqs(), rows(**kw)) == uad.UAD_EINVAL


@pytest.mark.parametrize("kw", BAD_ATTN)
def test_bad_attention_arguments_are_refused(kw):
    assert call_attention(pages8(), seqs(), attn(**kw)) == uad.UAD_EINVAL
    assert uad.uad_paged_attention_sinks(pages(), seqs(), attn(**kw), 2, None, 0, None, None) == uad.UAD_EINVAL


def test_sinks_are_not_negative():
    assert call_attention(pages8(), seqs(n_seqs=0), attn(window=4), -1) == uad.UAD_EINVAL
    assert uad.uad_paged_attention_sinks(pages(), seqs(n_seqs=0), attn(window=4), -1, None, 0, None, None) == uad.UAD_EINVAL
    assert uad.uad_paged_attention_sinks_workspace(pages(), seqs(), attn(window=4), -1) == uad.UAD_EINVAL


def test_null_structures_host_memory_and_ropes():
    for a in ((None, seqs(), rows()), (pages8(), None, rows()), (pages8(), seqs(), None)):
        assert call_append(*a) == uad.UAD_EINVAL
    for a in ((None, seqs(), attn()), (pages8(), None, attn()), (pages8(), seqs(), None)):
        assert call_attention(*a) == uad.UAD_EINVAL
    host = np.zeros(1 << 16, np.uint8)
    at = (host.ctypes.data + 63) // 64 * 64
    assert call_append(pages8(dict(k=at, v=at)), seqs(), rows()) == uad.UAD_EINVAL
    assert call_attention(pages8(dict(k=at, v=at)), seqs(), attn()) == uad.UAD_EINVAL
    for dim in (128, 0, 24):
        assert call_append(pages8(), seqs(n_seqs=0), rows(), uad.uad_rope(dim=dim)) == uad.UAD_EINVAL


def test_empty_batches_are_answered_without_a_launch():
    assert call_append(pages8(), seqs(n_seqs=0), rows()) == uad.UAD_OK
    assert call_append(pages8(), seqs(), rows(n_rows=0)) == uad.UAD_OK
    for sinks in (0, 5):
        assert call_attention(pages8(), seqs(n_seqs=0), attn(window=9), sinks) == uad.UAD_OK
        assert call_attention(pages8(), seqs(), attn(n_rows=0), sinks) == uad.UAD_OK
        assert uad.uad_paged_attention8_workspace(pages8(), seqs(n_seqs=0), attn(), sinks) == 0


def test_queries_in_place_need_bf16_rows_of_one_stride():
    for row, out_stride, sound in ((1, 256, True), (0, 256, False), (1, 512, False)):
        r = rows(dtype=row, q=P, q_out=P, q_out_stride=out_stride)
        assert call_append(pages8(), seqs(n_seqs=0), r) == (uad.UAD_OK if sound else uad.UAD_EINVAL)


def test_offsets_of_32_bits():
    """Codes in units of the strides' common power of two, scales in elements; what lies beyond is refused by the attention."""
    def need(inner=None, **kw):
        return uad.uad_paged_attention8_workspace(pages8(inner, **kw), seqs(), attn(), 0)

    assert need(dict(n_pages=1 << 24, page_stride=16 * 1024, slot_stride=1024, head_stride=64)) >= 0            # 256 GiB in units of 64 bytes
    assert need(dict(n_pages=(1 << 24) + 1, page_stride=16 * 1024, slot_stride=1024, head_stride=64)) == uad.UAD_EINVAL
    assert need(dict(n_pages=1 << 21, page_stride=16 * 2000, slot_stride=2000, head_stride=80)) >= 0            # 62.5 GiB in units of 16
    assert need(dict(n_pages=1 << 22, page_stride=16 * 2000, slot_stride=2000, head_stride=80)) == uad.UAD_EINVAL
    for kw in (dict(page_stride=1 << 62), dict(slot_stride=1 << 62), dict(head_stride=1 << 62), dict(page_stride=1 << 62, n_pages=(1 << 31) - 1)):
        assert need(dict(dict(n_pages=4), **kw)) in (0, uad.UAD_EINVAL)   # counted without overflow
    for kw in (dict(scale_page_stride=1 << 33), dict(scale_block_stride=1 << 32), dict(scale_head_stride=1 << 40)):
        assert need(**kw) == uad.UAD_EINVAL
    assert need(dict(n_pages=1 << 20), scale_page_stride=1 << 11) >= 0
    assert need(dict(n_pages=1 << 21), scale_page_stride=1 << 12) == uad.UAD_EINVAL


def test_units_of_offsets_are_32_bits_themselves():
    """Strides that share a power of two past 2^31: places are counted in units of 2^31, and what those do not hold is refused."""
    def need(n_pages, stride):
        return uad.uad_paged_attention8_workspace(pages8(dict(n_pages=n_pages, page_size=1, n_kv_heads=1, page_stride=stride, slot_stride=stride, head_stride=stride)),
                                                  seqs(), attn(n_heads=4), 0)

    assert need((1 << 31) - 1, 1 << 31) == 0
    for shift in (33, 34, 40, 47):
        assert need(1 << 63 - shift, 1 << shift) == 0   # the last page's place is 2^32 - 2^(shift - 31)
        assert need((1 << 63 - shift) + 1, 1 << shift) == uad.UAD_EINVAL
    assert need(2, 1 << 62) == 0
    assert need(3, 1 << 62) == uad.UAD_EINVAL


def test_a_workspace_without_a_window_holds_for_every_window_and_sinks():
    rng = np.random.default_rng(0)
    heads = [(8, 1, 256), (4, 1, 128), (8, 2, 64), (24, 24, 64), (32, 8, 128), (4, 2, 64)]
    for _ in range(3000):
        hq, hkv, dh = heads[rng.integers(len(heads))]
        kind = int(rng.integers(3))
        n_seqs, new = int(np.exp(rng.uniform(0, 6))), int(np.exp(rng.uniform(0, 4)))
        max_len = int(np.exp(rng.uniform(0, 11))) if rng.integers(4) else 0
        inner = dict(n_kv_heads=hkv, head_dim=dh, head_stride=dh, slot_stride=hkv * dh, page_stride=16 * hkv * dh)
        s = seqs(table=None, len=None, start=None, table_width=4096, table_stride=4096, n_seqs=n_seqs, max_new=new, max_len=max_len)

        def need(window, sinks):
            t = attn(n_heads=hq, n_rows=n_seqs * new, q_stride=hq * dh, out_stride=hq * dh, window=window)
            if kind == 2:
                return uad.uad_paged_attention8_workspace(pages8(inner), s, t, sinks)
            return uad.uad_paged_attention_sinks_workspace(pages(dtype=kind, **inner), s, t, sinks)

        most = need(0, 0)
        for w in np.exp(rng.uniform(0, np.log(max_len or 65536), 4)).astype(int):
            assert 0 <= need(int(w), int(rng.integers(0, 2000))) <= most


# ---- the pages' bookkeeping ---------------------------------------------------------------------------------------------------


def pool(**kw):
    return uad.uad_page_pool(**(dict(ring=P, state=P, state_out=P, n_pages=10, page_size=16) | kw))


def wanted(**kw):
    return uad.uad_kv_wanted(**(dict(table=P, len=P, want=P, len_out=P, start=P, slot=P, row_seq=P, row_pos=P, table_stride=4, n_seqs=2, table_width=4,
                                     n_rows=8) | kw))


@pytest.mark.parametrize("kw", [dict(ring=None), dict(state=None), dict(state_out=None), dict(n_pages=0), dict(n_pages=(1 << 30) + 1), dict(page_size=0),
                                dict(page_size=65537)])
def test_bad_pools_are_refused(kw):
    assert uad.uad_kv_resize(pool(**kw), wanted(), None, None) == uad.UAD_EINVAL


@pytest.mark.parametrize("kw", [dict(table=None), dict(len=None), dict(want=None), dict(len_out=None), dict(start=None), dict(table_stride=3), dict(n_seqs=-1),
                                dict(n_seqs=65536), dict(table_width=0), dict(n_rows=-1), dict(table_width=1 << 27, table_stride=1 << 27)])
def test_bad_requests_are_refused(kw):
    assert uad.uad_kv_resize(pool(), wanted(**kw), None, None) == uad.UAD_EINVAL


def test_null_structures_and_rings_that_are_no_gpu_memory():
    assert uad.uad_kv_resize(None, wanted(), None, None) == uad.UAD_EINVAL
    assert uad.uad_kv_resize(pool(), None, None, None) == uad.UAD_EINVAL
    host = np.zeros(64, np.int32)
    assert uad.uad_kv_resize(pool(ring=host.ctypes.data), wanted(), None, None) == uad.UAD_EINVAL


# ---- the binding stops malformed tensors before the call ------------------------------------------------------------------------


def test_binding_refuses_malformed_tensors():
    k = torch.zeros(4, 20, 2, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.zeros(4, 2, 2)
    for args, match in (((k, k), "goes with"), ((k, k, s), "goes with"), ((k.float(), k.float(), s, s), "goes with"), ((k, k, s, s, 20), "16, 32 or 64"),
                        ((k, k, s, s, 32), "k_scale"), ((k, k, s.double(), s, 16), "k_scale"), ((k, k, s, s[:, :1], 16), "v_scale"),
                        ((k, k, s, s.permute(1, 0, 2).contiguous().permute(1, 0, 2), 16), "v_scale"), ((k, k, s, s, 16), "on the GPU"),
                        ((k.view(torch.uint8), k.view(torch.uint8), s, s, 16), "float32 or bfloat16")):
        with pytest.raises(ValueError, match=match):
            uad.PagedCache(*args[:4], **(dict(block=args[4]) if len(args) > 4 else {}))
    whole = torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError, match="ring: must be on the GPU"):
        uad.PagePool(whole, whole[:2], 16)
    with pytest.raises(ValueError, match="ring: expected int32"):
        uad.PagePool(whole.long(), whole[:2], 16)
    with pytest.raises(ValueError, match="ring"):
        uad.PagePool(whole[:0], whole[:2], 16)
