"""GPU parity of attention through a window that leaves the first tokens visible, over bf16 and fp32 caches, against the 64-bit oracle. The
cases and tolerances are those of the attention without sinks (test_gpu_paged.py), which takes away a mask's worth of keys here."""
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from test_gpu_paged import Case, check_attention

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


def run(c, window, sinks, causal=True, mask=None, max_len=0, stream=None):
    width = c.hq * c.dh
    q = c.randn(c.rows, width)
    out = torch.full((c.rows, width), 7.5, device="cuda", dtype=c.dtype)
    lse = torch.full((c.rows, c.hq), 7.5, device="cuda")
    s, cache = c.sequences(max_len), uad.PagedCache(c.k, c.v)
    need = cache.attention_workspace(s, c.rows, c.hq, window, sinks)
    assert need <= cache.attention_workspace(s, c.rows, c.hq)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    cache.attention(s, q, out, ws[:-64], causal=causal, window=window, sinks=sinks, key_mask=mask, lse=lse, status=status, stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[-64:] == 255).all()) and int(status) == 0
    used = int(c.start[-1])
    assert bool((out[used:] == 7.5).all()) and bool((lse[used:] == 7.5).all())
    return q, out, lse


class Row:
    """One row of a case as a case, with what the window hides from it as a mask: test_gpu_paged's check does the rest."""

    def __init__(self, c, t, b, pos, window, sinks, causal, mask):
        self.hq, self.hkv, self.dh, self.dtype, self.n = c.hq, c.hkv, c.dh, c.dtype, 1
        self.lens, self.start, self.keys, self.values = [c.lens[b]], [0, 1], [c.keys[b]], [c.values[b]]
        j = np.arange(c.lens[b])
        seen = (j > pos - window) | (j < sinks)
        if causal:
            seen &= j <= pos
        if mask is not None:
            seen &= mask[b, :c.lens[b]].cpu().numpy() != 0
        self.mask = torch.from_numpy(seen[None])


def check(c, q, out, lse, window, sinks, causal=True, mask=None):
    for b in range(c.n):
        for t in range(int(c.start[b]), int(c.start[b + 1])):
            pos = c.lens[b] - (int(c.start[b + 1]) - t)
            r = Row(c, t, b, pos, window, sinks, causal, mask)
            check_attention(r, q[t:t + 1], out[t:t + 1], lse[t:t + 1], causal=False, mask=r.mask)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(20, 4), (1, 1), (16, 16), (5, 100), (64, 33), (300, 1), (7, 0)])
def test_windows_and_sinks(window, sinks, dtype):
    """Windows that begin before, in, at the end of and behind the sinks; sequences shorter than either; no sinks."""
    c = Case((8, 2, 64), 16, [1, 5, 23, 24, 25, 40, 90, 400, 0], [1, 2, 1, 1, 4, 16, 3, 1, 0], dtype, seed=window)
    for causal in (True, False):
        q, out, lse = run(c, window, sinks, causal)
        check(c, q, out, lse, window, sinks, causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,page", [((8, 1, 256), 16), ((4, 1, 128), 5), ((24, 24, 64), 100), ((32, 8, 128), 64), ((40, 2, 64), 1), ((3, 3, 256), 12)],
                         ids=lambda h: str(h))
def test_heads_and_pages(heads, page, dtype):
    c = Case(heads, page, [700, 33, 260, 131], [1, 2, 5, 1], dtype, "phsd", seed=page)
    q, out, lse = run(c, 50, 6)
    check(c, q, out, lse, 50, 6)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("max_len", [0, 100, 9000])
def test_what_lies_between_is_not_looked_at(max_len, dtype):
    """Pages between the sinks and the window are given back (-1), their tokens NaN; one that a sink and one that the window needs stay."""
    c = Case((8, 1, 128), 16, [9000, 5000, 600], [2, 1, 8], dtype, seed=3)
    window, sinks = 2000, 20
    for b in range(3):
        lo = c.lens[b] - c.new[b] - window + 1
        for i in range(2, max(0, lo) // 16):
            pg = int(c.table[b, i])
            c.k[pg], c.v[pg] = math.nan, math.nan
            c.keys[b][16 * i:16 * i + 16] = c.values[b][16 * i:16 * i + 16] = math.nan
            c.table[b, i] = -1
    q, out, lse = run(c, window, sinks, max_len=max_len)
    check(c, q, out, lse, window, sinks)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_sinks(dtype):
    """A mask over sinks and window; rows that are left with a single sink, with the first key of their window, with nothing."""
    c = Case((4, 2, 64), 16, [100, 100, 100], [1, 1, 2], dtype, seed=4)
    mask = torch.ones((3, c.width * 16), dtype=torch.uint8, device="cuda")
    mask[0, 1:3] = 0
    mask[1, :] = 0
    mask[1, 2] = 1
    mask[1, 50] = 1   # neither sink nor window
    mask[2, :4] = 0
    mask[2, 80:] = 0
    q, out, lse = run(c, 20, 4, mask=mask)
    check(c, q, out, lse, 20, 4, mask=mask)
    assert bool((out[3] == 0).all()) and torch.equal(out[2].double().cpu(), torch.from_numpy(c.values[2][79].repeat(2, axis=0).reshape(-1)))


def test_no_sinks_is_the_call_without():
    c = Case((8, 2, 64), 16, [400, 90], [1, 3], seed=5)
    s, cache = c.sequences(), uad.PagedCache(c.k, c.v)
    q = c.randn(c.rows, 512)
    ws = torch.empty(cache.attention_workspace(s, c.rows, 8), dtype=torch.uint8, device="cuda")
    for window, sinks in ((50, 0), (0, 7)):
        a, b = torch.zeros_like(q), torch.zeros_like(q)
        cache.attention(s, q, a, ws, window=window)
        cache.attention(s, q, b, ws, window=window, sinks=sinks)
        torch.cuda.synchronize()
        assert torch.equal(a, b)


@pytest.mark.parametrize("sinks", [-1, 1 << 31, (1 << 32) + 4])
def test_sinks_past_32_bits_are_refused(sinks):
    k = torch.zeros(2, 16, 1, 64, device="cuda")
    whole = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, out = torch.zeros(1, 64, device="cuda"), torch.full((1, 64), 7.5, device="cuda")
    seqs, cache = uad.Sequences(whole(0, 1).view(1, 2), whole(20), max_new=1), uad.PagedCache(k, k)
    with pytest.raises(ValueError, match="sinks"):
        cache.attention_workspace(seqs, 1, 1, 4, sinks)
    with pytest.raises(ValueError, match="sinks"):
        cache.attention(seqs, q, out, window=4, sinks=sinks)
    torch.cuda.synchronize()
    assert bool((out == 7.5).all())
