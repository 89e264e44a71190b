"""Caches of which a part is no memory of the current device are refused by the C entries, before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad

pytestmark = pytest.mark.gpu


def entries(kind):
    """A sound cache of one page and the calls on it: (its structure, append, attention)."""
    dtype = {"e4m3": torch.uint8, "bf16": torch.bfloat16, "f32": torch.float32}[kind]
    k, v = (torch.zeros(1, 16, 1, 64, device="cuda", dtype=dtype) for _ in range(2))
    whole = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    seqs = uad.Sequences(whole(0).view(1, 1), whole(1), max_new=1)
    out = torch.full((1, 64), 7.5, device="cuda", dtype=torch.float32 if kind == "f32" else torch.bfloat16)
    x = torch.zeros(1, 192, device="cuda")
    q = torch.zeros_like(out)
    rows = uad.uad_kv_rows(k=x.data_ptr(), v=x.data_ptr() + 256, k_stride=192, v_stride=192, dtype=0, n_rows=1)
    attn = uad.uad_attn(q=q.data_ptr(), out=out.data_ptr(), q_stride=64, out_stride=64, n_heads=1, n_rows=1)
    keep = [k, v, seqs, x, q, rows, attn]
    if kind == "e4m3":
        scales = torch.ones(2, 1, 1, 1, device="cuda")
        cache = uad.PagedCache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), scales[0], scales[1])
        keep.append(scales)
        return cache.pages8, lambda p: uad.uad_kv_append8(p, seqs.seqs, rows, None, None, None), \
            lambda p: uad.uad_paged_attention8(p, seqs.seqs, attn, 0, None, 0, None, None), out, keep
    return uad.PagedCache(k, v).pages, lambda p: uad.uad_kv_append(p, seqs.seqs, rows, None, None, None), \
        lambda p: uad.uad_paged_attention(p, seqs.seqs, attn, None, 0, None, None), out, keep


@pytest.mark.parametrize("kind,part", [("e4m3", "k"), ("e4m3", "v"), ("e4m3", "k_scale"), ("e4m3", "v_scale"), ("bf16", "k"), ("bf16", "v"), ("f32", "v")])
def test_parts_on_the_host_are_refused(kind, part):
    sound, append, attention, out, keep = entries(kind)
    host = np.zeros(1 << 14, np.uint8)
    at = (host.ctypes.data + 63) // 64 * 64
    pages = type(sound).from_buffer_copy(sound)
    setattr(pages.pages if kind == "e4m3" and part in ("k", "v") else pages, part, at)
    assert append(C.byref(pages)) == attention(C.byref(pages)) == uad.UAD_EINVAL
    torch.cuda.synchronize()
    assert bool((out == 7.5).all())
    assert append(C.byref(sound)) == attention(C.byref(sound)) == uad.UAD_OK
    torch.cuda.synchronize()
    assert bool((out == 0).all())
