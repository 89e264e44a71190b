"""GPU parity of the paged key-value cache's append and attention against the 64-bit oracle, at the sizes, layouts and
masks where they can go wrong, and their behaviour on streams, in graphs and with bad tables.

Tolerances. Rotation: cos and sin are off by at most 2^-23 (an angle known to 2^-28 turns, a correctly reduced function
to one ulp), two products and a sum round by 2^-24 each: (|a| + |b|) 2^-22, then the type's half step.
Attention: a score of dh products in fp32 is off by at most dh 2^-23 scale sum |q k| (the tensor cores truncate, an ulp a
step; the scaling rounds once): d. Probabilities then are off by a factor e^d at most, twice (numerator and
denominator), by exp's own error (2^-20 with the scores' magnitudes here) and by 2^-16 where they are the sum of two bf16;
sums of n terms by n 2^-23. The output is off by that much of sum p |v|, then by the type's half step.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TINY = 1e-30


class Case:
    """A batch: pools with NaN in every slot that no sequence holds, tables in a random order."""

    def __init__(self, heads, page, lens, new, dtype=torch.bfloat16, layout="pshd", seed=0, rows_behind=2, width=None, spare=5):
        self.hq, self.hkv, self.dh = heads
        self.page, self.dtype = page, dtype
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.lens, self.new = list(lens), list(new)
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.n = len(self.lens)
        self.rows = int(self.start[-1]) + rows_behind
        self.width = width or max(1, max((n + page - 1) // page for n in self.lens))
        used = [(n + page - 1) // page for n in self.lens]
        self.pages = sum(used) + spare
        ids = torch.randperm(self.pages, generator=self.g, device="cuda").tolist()
        self.table = np.full((self.n, self.width), -1, np.int32)
        for b, u in enumerate(used):
            self.table[b, :u] = [ids.pop() for _ in range(u)]
        shape = (2, self.pages, page, self.hkv, self.dh) if layout == "pshd" else (2, self.pages, self.hkv, page, self.dh)
        if layout == "joint":   # keys and values of a page next to each other
            shape = (self.pages, 2, page, self.hkv, self.dh)
        pool = torch.full(shape, float("nan"), device="cuda", dtype=dtype)
        if layout == "joint":
            pool = pool.transpose(0, 1)
        elif layout == "phsd":
            pool = pool.transpose(2, 3)
        self.k, self.v = pool[0], pool[1]
        # what the sequences hold
        self.keys, self.values = [], []
        for b, n in enumerate(self.lens):
            at = np.arange(n)
            k = self.randn(n, self.hkv, self.dh)
            v = self.randn(n, self.hkv, self.dh)
            pg = torch.from_numpy(self.table[b, at // page].astype(np.int64)).cuda()
            sl = torch.from_numpy(at % page).cuda()
            self.k[pg, sl], self.v[pg, sl] = k, v
            self.keys.append(k.double().cpu().numpy())
            self.values.append(v.double().cpu().numpy())

    def randn(self, *shape, dtype=None):
        return torch.randn(shape, generator=self.g, device="cuda").to(dtype or self.dtype)

    def sequences(self, max_len=0, max_new=None):
        self.dev = [torch.from_numpy(x).cuda() for x in (self.table, np.array(self.lens, np.int32), self.start)]
        return uad.Sequences(*self.dev, max_len=max_len, max_new=max_new or max(1, max(self.new)))

    def put(self, b, pos, k=None, v=None):
        """Overwrite one cached token's keys / values of a sequence (every head)."""
        pg, sl = int(self.table[b, pos // self.page]), pos % self.page
        for x, pool, held in ((k, self.k, self.keys), (v, self.v, self.values)):
            if x is not None:
                pool[pg, sl] = torch.as_tensor(x, dtype=torch.float64, device="cuda").to(self.dtype)
                held[b][pos] = x


def run_attention(c, causal=True, window=0, mask=None, scale=None, max_len=0, fused=False, stream=None, max_new=None):
    width = c.hq * c.dh
    q = c.randn(c.rows, width + 16)[:, :width] if fused else c.randn(c.rows, width)
    out = torch.full((c.rows, width + (8 if fused else 0)), 7.5, device="cuda", dtype=c.dtype)[:, :width]
    lse = torch.full((c.rows, c.hq), 7.5, device="cuda")
    s = c.sequences(max_len, max_new)
    cache = uad.PagedCache(c.k, c.v)
    ws = torch.full((cache.attention_workspace(s, c.rows, c.hq, window) + 64,), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    cache.attention(s, q, out, ws[:-64], scale=scale, causal=causal, window=window, key_mask=mask, lse=lse, status=status, stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[-64:] == 255).all())
    return q, out, lse, int(status)


def check_attention(c, q, out, lse, causal=True, window=0, mask=None, scale=None):
    scale = scale or 1 / math.sqrt(c.dh)
    qn, on, ln = q.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    mn = None if mask is None else mask.cpu().numpy()
    group, worst = c.hq // c.hkv, 0.0
    for t, at in enumerate(paged.rows_of(c.lens, c.start)):
        b, pos = at
        j = np.arange(c.lens[b])
        seen = np.ones(c.lens[b], bool)
        if causal:
            seen &= j <= pos
        if window:
            seen &= j > pos - window
        if mn is not None:
            seen &= mn[b, :c.lens[b]] != 0
        n = int(seen.sum())
        for h in range(c.hkv):
            rows = qn[t].reshape(c.hq, c.dh)[h * group:(h + 1) * group]
            k, v = c.keys[b][:, h], c.values[b][:, h]
            want, wl = paged.attend(rows, k, v, seen, scale)
            got, gl = on[t].reshape(c.hq, c.dh)[h * group:(h + 1) * group], ln[t, h * group:(h + 1) * group]
            if n == 0:
                assert np.all(got == 0) and np.all(np.isneginf(gl)), (t, h)
                continue
            bad = np.isnan(want)
            assert np.array_equal(np.isnan(got), bad) and np.array_equal(np.isnan(gl), np.isnan(wl)), (t, h)
            if bad.all():
                continue
            with np.errstate(all="ignore"):
                z = scale * rows @ k[seen].T
                p = np.exp(z - z.max(axis=1, keepdims=True))
                p /= p.sum(axis=1, keepdims=True)
                d = c.dh * 2.0 ** -23 * scale * (np.abs(rows) @ np.abs(k[seen]).T).max(axis=1, keepdims=True)
                rel = 2 * (2 * d + 2.0 ** -20 + 2.0 ** -16 + n * 2.0 ** -23)
                tol = rel * (p @ np.abs(v[seen])) + HALF[c.dtype] * np.abs(want) + TINY
                err = np.abs(got - want)
                assert np.all((err <= tol) | bad), (t, h, float(np.nanmax(err / tol)))
                assert np.all((np.abs(gl - wl) <= d[:, 0] + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -22 * np.abs(wl)) | np.isnan(wl)), (t, h, gl, wl)
            worst = max(worst, float(np.nanmax(err / tol)))
    return worst


HEADS = [(8, 1, 256), (4, 1, 128), (8, 2, 64), (24, 24, 64), (32, 8, 128), (3, 3, 256), (21, 1, 64), (128, 2, 128)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_attention_of_one_token(heads, dtype):
    """Lengths of one token and around the pages, tiles and pieces; a sequence without new tokens; one token that is all."""
    c = Case(heads, 16, [1, 2, 15, 16, 17, 63, 64, 65, 200, 0, 333, 40], [1, 1, 1, 1, 1, 1, 1, 1, 1, 0, 1, 0], dtype, seed=sum(heads))
    q, out, lse, status = run_attention(c)
    assert status == 0
    check_attention(c, q, out, lse)
    used = int(c.start[-1])
    assert bool((out[used:] == 7.5).all()) and bool((lse[used:] == 7.5).all())   # rows of nobody


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,layout", [(1, "pshd"), (5, "phsd"), (12, "joint"), (100, "pshd"), (128, "phsd"), (16, "joint")])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 37), (False, 70)])
def test_attention_of_a_few_tokens(page, layout, causal, window, dtype):
    """Drafts and chunks of different lengths, ends of pages inside of tiles, windows, fused rows, every layout."""
    c = Case((8, 2, 64), page, [3, 40, 129, 700, 64, 9], [3, 5, 1, 16, 0, 9], dtype, layout, seed=page)
    q, out, lse, status = run_attention(c, causal, window, fused=True)
    assert status == 0
    check_attention(c, q, out, lse, causal, window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(8, 1, 256), (16, 2, 128), (5, 1, 64)], ids=lambda h: "x".join(map(str, h)))
def test_attention_with_key_masks(heads, dtype):
    """Masked cameras, single keys left, and rows that see nothing at all (output 0, lse -inf)."""
    c = Case(heads, 16, [90, 300, 33, 64, 5], [4, 2, 1, 3, 5], dtype, seed=7)
    mask = torch.ones((c.n, c.width * c.page + 3), dtype=torch.uint8, device="cuda")[:, :c.width * c.page]
    mask[0, 10:70] = 0
    mask[1] = 0
    mask[1, 299] = 255      # the last token alone sees anything
    mask[2] = 0             # nothing
    mask[3, :60] = 0
    mask[4, ::2] = 0
    for causal in (True, False):
        q, out, lse, status = run_attention(c, causal, mask=mask)
        assert status == 0
        check_attention(c, q, out, lse, causal, mask=mask)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(8, 1, 256), (4, 2, 128), (8, 8, 64)], ids=lambda h: "x".join(map(str, h)))
def test_what_a_token_does_not_see_has_no_influence(heads, dtype):
    """NaN and infinities in keys and values of later tokens, before the window, and in masked places."""
    for causal, window in ((True, 0), (True, 20)):
        c = Case(heads, 16, [37, 80], [6, 3], dtype, seed=11)
        for pos, x in ((33, math.nan), (34, math.inf), (36, -math.inf)):   # tokens of the call itself
            c.put(0, pos, k=x, v=x)
        mask = torch.ones((c.n, c.width * c.page), dtype=torch.uint8, device="cuda")
        for pos in (3, 50, 78):
            c.put(1, pos, k=math.nan, v=math.inf)
            mask[1, pos] = 0
        if window:
            c.put(1, 58, k=math.nan, v=math.nan)   # the first of the three rows sees 58 to 77, the others do not
        q, out, lse, status = run_attention(c, causal, window, mask)
        assert status == 0
        check_attention(c, q, out, lse, causal, window, mask)
        assert bool(torch.isfinite(out[:2].float()).all())   # rows 0 and 1 of the first draft see nothing of it


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_special_scores(dtype):
    """Scores far apart (one key takes all), +inf and NaN (undefined), -inf (no weight; undefined where there is nothing else)."""
    c = Case((4, 2, 64), 16, [50, 50, 50, 50, 20], [1, 1, 1, 1, 1], dtype, seed=3)
    c.put(0, 17, k=100.0)
    c.put(1, 4, k=np.array([math.nan] + [0.0] * 63))
    q, out, lse, status = run_attention(c, scale=3.0)
    check_attention(c, q, out, lse, scale=3.0)
    c.put(2, 9, v=math.inf)      # seen, with a weight above 0: infinite
    c.put(3, 49, v=-math.inf)
    q, out, lse, status = run_attention(c)
    assert bool((out[2] == math.inf).all()) and bool((out[3] == -math.inf).all())
    assert bool(torch.isfinite(out[0].float()).all()) and bool(torch.isnan(out[1]).all())
    c2 = Case((1, 1, 64), 4, [6, 6, 6], [1, 1, 1], dtype, seed=4)
    one = torch.zeros(c2.rows, 64, device="cuda", dtype=dtype)
    one[:, 0] = 1.0
    e = np.zeros(64)
    for pos in range(6):
        c2.put(0, pos, k=np.concatenate([[-math.inf], e[1:]]))                       # all -inf: undefined
        c2.put(1, pos, k=np.concatenate([[-math.inf if pos else 2.0], e[1:]]))       # one key left
        c2.put(2, pos, k=np.concatenate([[math.inf if pos == 3 else 0.5], e[1:]]))   # +inf: undefined
    out = torch.empty(c2.rows, 64, device="cuda", dtype=dtype)
    lse = torch.empty(c2.rows, 1, device="cuda")
    s, cache = c2.sequences(), uad.PagedCache(c2.k, c2.v)
    ws = torch.empty(cache.attention_workspace(s, c2.rows, 1), dtype=torch.uint8, device="cuda")
    cache.attention(s, one, out, ws, scale=1.0, lse=lse)
    torch.cuda.synchronize()
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(out[2]).all()) and bool(torch.isnan(lse[0])) and bool(torch.isnan(lse[2]))
    assert np.array_equal(out[1].double().cpu().numpy(), c2.values[1][0, 0]) and abs(float(lse[1]) - 2.0) < 1e-6


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("max_len", [0, 1, 100, 5000])
def test_long_caches_are_split_and_joined(dtype, max_len):
    """The work's split follows max_len, right or wrong; shorter and longer sequences beside each other."""
    c = Case((8, 1, 256), 64, [5000, 3, 1900, 4097, 64], [2, 1, 1, 4, 1], dtype, seed=5)
    q, out, lse, status = run_attention(c, max_len=max_len)
    assert status == 0
    check_attention(c, q, out, lse)


def test_many_sequences():
    c = Case((8, 1, 64), 16, [1 + 7 * i % 90 for i in range(300)], [1] * 300, seed=6)
    q, out, lse, status = run_attention(c)
    assert status == 0
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("heads,n,longest,new", [((24, 24, 64), 40, 90, 2), ((32, 8, 128), 60, 70, 1), ((16, 16, 256), 20, 80, 1),
                                                 ((24, 24, 64), 26, 2300, 1), ((12, 4, 64), 152, 60, 17)],
                         ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else str(x))
def test_more_heads_than_ctas(heads, n, longest, new):
    """Every warp of a CTA has a head of its own, with the pieces of long sequences too."""
    lens = [max(new, 1 + (37 * i) % longest) for i in range(n)]
    lens[1] = longest
    c = Case(heads, 16, lens, [min(new, 1 + i % new) for i in range(n)], seed=n)
    q, out, lse, status = run_attention(c)
    assert status == 0
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("heads,n,longest,new", [((24, 24, 64), 30, 700, 1), ((32, 8, 128), 58, 530, 1), ((8, 4, 64), 160, 600, 1), ((24, 24, 64), 17, 650, 8),
                                                 ((32, 8, 128), 16, 4100, 1)])
def test_many_heads_and_longer_caches(heads, n, longest, new):
    """More heads than CTAs whose keys are many, a wave that is nearly full, one that would be barely more than one."""
    lens = [longest if b < 2 else max(new, longest * (b % 7) // 7) for b in range(n)]
    c = Case(heads, 16, lens, [new] * n, seed=n)
    q, out, lse, status = run_attention(c, max_len=longest)
    assert status == 0
    check_attention(c, q, out, lse)


def test_offsets_past_32_bits():
    """Pages 2^30 elements apart: element offsets up to 3 * 2^30 + ..., bytes past 2^32."""
    buf = torch.zeros((3 << 30) + (1 << 21), dtype=torch.bfloat16, device="cuda")
    c = Case((8, 1, 256), 16, [64], [3], seed=8, spare=0)
    k = buf.as_strided((4, 16, 1, 256), (1 << 30, 256, 256, 1), 0)
    v = buf.as_strided((4, 16, 1, 256), (1 << 30, 256, 256, 1), 1 << 20)
    k.copy_(c.k)
    v.copy_(c.v)
    c.k, c.v = k, v
    q, out, lse, status = run_attention(c)
    assert status == 0
    check_attention(c, q, out, lse)
    r = uad.rope(10000.0, 256)
    new_k, new_v = c.randn(c.rows, 256), c.randn(c.rows, 256)
    uad.PagedCache(k, v).append(c.sequences(), new_k, new_v, rope=r)
    torch.cuda.synchronize()
    for j in range(3):
        pg, sl = int(c.table[0, (61 + j) // 16]), (61 + j) % 16
        assert torch.equal(v[pg, sl, 0], new_v[j])


def test_attention_leaves_bad_pages_and_sequences_out():
    c = Case((8, 2, 64), 16, [100, 64, 50, 30, 20], [2, 1, 1, 1, 1], seed=9)
    good = c.table.copy()
    c.table[0, 3] = c.pages          # past the last page: tokens 48..63 are left out
    c.table[1, 1] = -1
    mask = torch.ones((c.n, c.width * c.page), dtype=torch.uint8, device="cuda")
    q, out, lse, status = run_attention(c)
    assert status == uad.UAD_KV_BAD_PAGE
    mask[0, 48:64] = 0
    mask[1, 16:32] = 0
    check_attention(c, q, out, lse, mask=mask)
    q, out, lse, status = run_attention(c, mask=mask)   # not seen: not looked at
    assert status == 0
    check_attention(c, q, out, lse, mask=mask)
    c.table = good
    lens, start = c.lens, c.start
    for bad_lens, bad_start in (([100, -1, 50, 30, 20], start), ([100, c.width * 16 + 1, 50, 30, 20], start), ([100, 0, 50, 30, 20], start),
                                (lens, np.array([0, 2, 3, 4, 5, 99], np.int32)), (lens, np.array([-1, 2, 3, 4, 5, 6], np.int32)),
                                (lens, np.array([0, 2, 1, 4, 5, 6], np.int32))):
        c.lens, c.start = bad_lens, bad_start
        q, out, lse, status = run_attention(c, max_new=2)
        assert status == uad.UAD_KV_BAD_SEQ
        c.lens, c.start = lens, start
        assert bool(torch.isfinite(out.float()).all())
        # sequences that are whole are served: the fourth is in every one of these
        assert bool((out[4] != 7.5).any()) if bad_start is start else True
    c.new = [2, 1, 1, 1, 1]
    q, out, lse, status = run_attention(c, max_new=1)   # the first has two new tokens
    assert status == uad.UAD_KV_BAD_SEQ and bool((out[:2] == 7.5).all()) and bool((out[2:6] != 7.5).any(dim=1).all())


def test_without_start_every_row_is_a_sequence():
    c = Case((8, 1, 256), 16, [30, 1, 77], [1, 1, 1], seed=10, rows_behind=0)
    q = c.randn(3, 2048)
    table, lens, _ = [torch.from_numpy(x).cuda() for x in (c.table, np.array(c.lens, np.int32), c.start)]
    s = uad.Sequences(table, lens)
    cache = uad.PagedCache(c.k, c.v)
    out, lse = torch.empty_like(q), torch.empty(3, 8, device="cuda")
    ws = torch.empty(cache.attention_workspace(s, 3, 8), dtype=torch.uint8, device="cuda")
    cache.attention(s, q, out, ws, lse=lse)
    torch.cuda.synchronize()
    check_attention(c, q, out, lse)


def test_attention_is_the_same_every_time():
    c = Case((8, 1, 256), 16, [4000, 17, 900], [3, 1, 2], seed=12)
    s, cache = c.sequences(), uad.PagedCache(c.k, c.v)
    q = c.randn(c.rows, 2048)
    ws = torch.empty(cache.attention_workspace(s, c.rows, 8), dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(4):
        out = torch.empty_like(q)
        cache.attention(s, q, out, ws)
        outs.append(out)
    torch.cuda.synchronize()
    used = int(c.start[-1])
    assert all(torch.equal(outs[0][:used], o[:used]) for o in outs[1:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_in_stream_order_and_in_graphs(dtype):
    """Keys appended just before on the same side stream; a captured call that is replayed as the sequences grow; two graphs,
    each with a workspace of its own, at the same time."""
    c = Case((8, 1, 128), 16, [400, 9], [1, 1], dtype, seed=13, rows_behind=0, width=40, spare=40)
    free = sorted(set(range(c.pages)) - set(c.table[c.table >= 0].tolist()))
    for b in range(2):
        for i in range(40):
            if c.table[b, i] < 0 and free:
                c.table[b, i] = free.pop()
    s, cache = c.sequences(max_len=400), uad.PagedCache(c.k, c.v)
    length = c.dev[1]
    st = torch.cuda.Stream()
    rope = uad.rope(10000.0, 128)
    qkv = c.randn(2, 8 * 128 + 2 * 128)
    q_out, outs = torch.empty(2, 1024, device="cuda", dtype=dtype), [torch.empty(2, 1024, device="cuda", dtype=dtype) for _ in range(2)]
    lse = [torch.empty(2, 8, device="cuda") for _ in range(2)]
    n = cache.attention_workspace(s, 2, 8)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(i, stream):
        cache.append(s, qkv[:, 1024:1152], qkv[:, 1152:], q=qkv[:, :1024], q_out=q_out, rope=rope, stream=stream)
        cache.attention(s, q_out, outs[i], ws[i], lse=lse[i], stream=stream)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step(0, st)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            step(i, st)
        graphs.append(g)
    for turn in range(6):
        c.lens = [c.lens[0] + 7, c.lens[1] + 1]
        length.copy_(torch.tensor(c.lens, dtype=torch.int32))
        # tokens between are left from before or NaN: give the reference what the cache holds
        qkv.copy_(c.randn(*qkv.shape))
        for b in range(2):
            at = np.arange(c.lens[b])
            pg, sl = torch.from_numpy(c.table[b, at // 16].astype(np.int64)).cuda(), torch.from_numpy(at % 16).cuda()
            k, v = c.k[pg, sl].nan_to_num(0.25), c.v[pg, sl].nan_to_num(0.25)
            c.k[pg, sl], c.v[pg, sl] = k, v
        torch.cuda.synchronize()
        graphs[0].replay()
        torch.cuda.synchronize()
        for b in range(2):
            at = np.arange(c.lens[b])
            pg, sl = torch.from_numpy(c.table[b, at // 16].astype(np.int64)).cuda(), torch.from_numpy(at % 16).cuda()
            c.keys[b], c.values[b] = (x[pg, sl].double().cpu().numpy() for x in (c.k, c.v))
        check_attention(c, q_out, outs[0], lse[0])
    # both at once, attention alone (they write the same slots with the same values)
    outs[0].zero_()
    outs[1].zero_()
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        graphs[0].replay()
    with torch.cuda.stream(other):
        graphs[1].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    check_attention(c, q_out, outs[1], lse[1])


# ---- append -----------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("cache_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("row_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,rot", [((8, 1, 256), 256), ((4, 1, 128), 64), ((8, 2, 64), 64), ((6, 3, 64), 16), ((2, 2, 256), 240), ((24, 24, 64), 0)],
                         ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else str(x))
def test_append(heads, rot, row_type, cache_type):
    """Fused rows, ragged new tokens at near and far positions; every other slot and row stays as it was."""
    for page, layout in ((16, "pshd"), (5, "phsd"), (1, "joint")):
        c = Case(heads, page, [1, 60, 33, 0, 200], [1, 7, 0, 0, 65], cache_type, layout, seed=page)
        hq, hkv, dh = heads
        qkv = c.randn(c.rows, (hq + 2 * hkv) * dh, dtype=row_type)
        q, k, v = qkv.split([hq * dh, hkv * dh, hkv * dh], dim=1)
        q_out = torch.full((c.rows, hq * dh), 7.5, device="cuda", dtype=cache_type)
        before_k, before_v = c.k.clone(), c.v.clone()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        uad.PagedCache(c.k, c.v).append(c.sequences(), k, v, q=q, q_out=q_out, rope=uad.rope(10000.0, rot) if rot else None, status=status)
        torch.cuda.synchronize()
        assert int(status) == 0
        qn, kn, vn = (x.double().cpu().numpy().reshape(c.rows, -1, dh) for x in (q, k, v))
        got_q = q_out.double().cpu().numpy().reshape(c.rows, hq, dh)
        touched = torch.zeros(c.k.shape[:2], dtype=torch.bool, device="cuda")
        for t, (b, pos) in enumerate(paged.rows_of(c.lens, c.start)):
            pg, sl = int(c.table[b, pos // page]), pos % page
            touched[pg, sl] = True
            for got, x in ((got_q[t], qn[t]), (c.k[pg, sl].double().cpu().numpy(), kn[t])):
                want = paged.rotate(x, pos, 10000.0, rot)
                size = np.abs(x).copy()
                size[:, :rot // 2] += np.abs(x[:, rot // 2:rot])
                size[:, rot // 2:rot] = size[:, :rot // 2]
                tol = size * 2.0 ** -22 * (rot > 0) + HALF[cache_type] * (np.abs(want) + size * 2.0 ** -22)
                assert np.all(np.abs(got - want) <= tol), (t, np.max(np.abs(got - want) - tol))
            assert torch.equal(c.v[pg, sl], v[t].reshape(hkv, dh).to(cache_type))
        for now, then in ((c.k, before_k), (c.v, before_v)):
            assert torch.equal(torch.nan_to_num(now[~touched], 9.0), torch.nan_to_num(then[~touched], 9.0))
        assert bool((q_out[int(c.start[-1]):] == 7.5).all())


@pytest.mark.parametrize("heads,rot,tokens", [((8, 1, 256), 256, 700), ((8, 1, 256), 240, 2000), ((6, 3, 64), 16, 9000), ((32, 8, 128), 128, 800), ((3, 1, 128), 0, 5000)],
                         ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else str(x))
@pytest.mark.parametrize("row_type,cache_type", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
def test_append_of_many_tokens(heads, rot, tokens, row_type, cache_type):
    """Whole prompts in one call: the bits of the same tokens appended few at a time; tokens of a bad page are left out, their
    queries are not."""
    hq, hkv, dh = heads
    new = [tokens - tokens // 3, 1, tokens // 3]
    c = Case(heads, 16, [new[0] + 5, 1, new[2]], new, cache_type, "phsd", seed=tokens)
    bad = 3   # a page's place in the first sequence, which holds none
    c.table[0, bad] = c.pages + 7
    q, k, v = (c.randn(c.rows, n * dh, dtype=row_type) for n in (hq, hkv, hkv))
    rope = uad.rope(10000.0, rot) if rot else None
    once = torch.full((c.rows, hq * dh), 7.5, device="cuda", dtype=cache_type)
    few = once.clone()
    k2, v2 = c.k.clone(), c.v.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    uad.PagedCache(c.k, c.v).append(c.sequences(), k, v, q=q, q_out=once, rope=rope, status=status)
    table = torch.from_numpy(c.table).cuda()
    for b in range(3):
        for i in range(0, new[b], 16):
            n = min(16, new[b] - i)
            at = slice(int(c.start[b]) + i, int(c.start[b]) + i + n)
            length = torch.tensor([c.lens[b] - new[b] + i + n], dtype=torch.int32, device="cuda")
            start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
            uad.PagedCache(k2, v2).append(uad.Sequences(table[b:b + 1], length, start, max_new=16), k[at], v[at], q=q[at], q_out=few[at], rope=rope)
    torch.cuda.synchronize()
    assert int(status) == uad.UAD_KV_BAD_PAGE
    assert torch.equal(once, few) and not bool((once[:-2] == 7.5).all(dim=1).any()) and bool((once[-2:] == 7.5).all())
    for a, b in ((c.k, k2), (c.v, v2)):
        assert torch.equal(torch.nan_to_num(a, 9.0), torch.nan_to_num(b, 9.0))
    pg, sl = int(c.table[0, (c.lens[0] - 1) // 16]), (c.lens[0] - 1) % 16
    want = paged.rotate(k[new[0] - 1].double().cpu().numpy().reshape(hkv, dh), c.lens[0] - 1, 10000.0, rot)
    x = np.abs(k[new[0] - 1].double().cpu().numpy().reshape(hkv, dh))
    size = x + 0
    size[:, :rot // 2] += x[:, rot // 2:rot]
    size[:, rot // 2:rot] = size[:, :rot // 2]
    tol = size * 2.0 ** -22 * (rot > 0) + HALF[cache_type] * (np.abs(want) + size * 2.0 ** -22)
    assert np.all(np.abs(c.k[pg, sl].double().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("pos", [0, 1, 816, 65535, 1 << 20, 2_000_000_000])
def test_rotation_of_far_positions(pos):
    """fp32 rows at positions whose angles 32 bits do not hold."""
    page, dh = 64, 256
    table = torch.full((1, pos // page + 1), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 0
    pool = torch.zeros(2, 1, page, 1, dh, device="cuda")
    s = uad.Sequences(table, torch.tensor([pos + 1], dtype=torch.int32, device="cuda"))
    g = torch.Generator(device="cuda")
    g.manual_seed(pos)
    k = torch.randn(1, dh, generator=g, device="cuda")
    uad.PagedCache(pool[0], pool[1]).append(s, k, k, rope=uad.rope(10000.0, dh))
    torch.cuda.synchronize()
    x = k.double().cpu().numpy().reshape(1, dh)
    # both sides have their frequencies from a long double of 64 bits or more: power (an ulp), constant, product, and what is
    # cut off at 2^-64 of a turn are below 2^-60 of a position's radians each
    extra = 8 * (pos + 1) * 2.0 ** -60
    size = np.abs(x[:, :dh // 2]) + np.abs(x[:, dh // 2:])
    size = np.concatenate([size, size], axis=1)
    err = np.abs(pool[0, 0, pos % page].double().cpu().numpy() - paged.rotate(x, pos, 10000.0, dh))
    assert np.all(err <= size * (2.0 ** -22 + extra) + 2.0 ** -24 * size)


def test_append_of_queries_or_keys_alone_and_in_place():
    c = Case((8, 1, 256), 16, [20, 40], [2, 1], seed=2)
    s, cache, r = c.sequences(), uad.PagedCache(c.k, c.v), uad.rope(10000.0, 256)
    q, k, v = c.randn(c.rows, 2048), c.randn(c.rows, 256), c.randn(c.rows, 256)
    both = torch.empty_like(q)
    cache.append(s, k, v, q=q, q_out=both, rope=r)
    kept = c.k.clone()
    alone = q.clone()
    cache.append(s, q=alone, q_out=alone, rope=r)      # in place, keys untouched
    torch.cuda.synchronize()
    used = int(c.start[-1])
    assert torch.equal(alone[:used], both[:used]) and torch.equal(alone[used:], q[used:])
    assert torch.equal(kept.nan_to_num(1.0), c.k.nan_to_num(1.0))
    c.k.zero_()
    cache.append(s, k, v, rope=r)
    torch.cuda.synchronize()
    for b, pos in paged.rows_of(c.lens, c.start):
        pg, sl = int(c.table[b, pos // 16]), pos % 16
        assert torch.equal(c.k[pg, sl], kept[pg, sl])


def test_append_leaves_bad_pages_and_sequences_out():
    c = Case((8, 2, 64), 16, [40, 64, 50], [10, 4, 2], seed=14)
    c.table[0, 2] = c.pages + 5      # tokens 32..39
    lens = list(c.lens)
    k, v = c.randn(c.rows, 128), c.randn(c.rows, 128)
    for bad, want in ((None, uad.UAD_KV_BAD_PAGE), (3, uad.UAD_KV_BAD_PAGE | uad.UAD_KV_BAD_SEQ), (1 << 30, uad.UAD_KV_BAD_PAGE | uad.UAD_KV_BAD_SEQ)):
        c.lens = lens if bad is None else [lens[0], bad, lens[2]]
        before = c.v.clone().nan_to_num(9.0)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        uad.PagedCache(c.k, c.v).append(c.sequences(), k, v, status=status)
        torch.cuda.synchronize()
        assert int(status) == want
        changed = (c.v.nan_to_num(9.0) != before).any(dim=-1).any(dim=-1)
        allowed = torch.zeros_like(changed)
        for b, pos in [(0, 30), (0, 31), (1, 60), (1, 61), (1, 62), (1, 63), (2, 48), (2, 49)]:
            if not (b == 1 and bad is not None):
                allowed[int(c.table[b, pos // 16]), pos % 16] = True
        assert not bool((changed & ~allowed).any())
        if bad is None:
            assert bool((changed == allowed).all())


def test_calls_that_the_binding_refuses_on_the_gpu():
    c = Case((8, 2, 64), 16, [40], [1], seed=15, rows_behind=0)
    s, cache = c.sequences(), uad.PagedCache(c.k, c.v)
    q = c.randn(1, 512)
    out = torch.empty_like(q)
    for bad in (dict(q=q.float()), dict(q=q[:, :100]), dict(out=out[:, :64]), dict(out=out.cpu()), dict(lse=torch.empty(1, 8)),
                dict(lse=torch.empty(1, 9, device="cuda")), dict(key_mask=torch.ones(1, 47, dtype=torch.uint8, device="cuda")),
                dict(key_mask=torch.ones(1, 48, device="cuda")), dict(workspace=torch.empty(64, device="cuda"))):
        with pytest.raises(ValueError):
            cache.attention(s, **(dict(q=q, out=out) | bad))
    with pytest.raises(uad.UADError):
        cache.attention(s, q[:, :192].contiguous(), out[:, :192].contiguous())   # 3 heads over 2
    k = c.randn(1, 128)
    for bad in (dict(v=None), dict(q=q), dict(k=k[:, :64]), dict(v=k.float()), dict(k=None, v=None), dict(k=k.half(), v=k.half()),
                dict(q=q, q_out=out.float()), dict(status=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            cache.append(s, **(dict(k=k, v=k) | bad))
    with pytest.raises(uad.UADError):
        cache.append(s, k, k, rope=uad.rope(10000.0, 128))   # wider than a head
    big = Case((8, 1, 256), 16, [5000], [1], seed=16)
    bs, bc = big.sequences(), uad.PagedCache(big.k, big.v)
    n = bc.attention_workspace(bs, big.rows, 8)
    if n:
        bq = big.randn(big.rows, 2048)
        with pytest.raises(uad.UADError):
            bc.attention(bs, bq, torch.empty_like(bq), torch.empty(n - 1, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("heads,dtype,lens,new,window", [((8, 2, 64), torch.bfloat16, [2400] * 32, 1, 2100), ((8, 1, 256), torch.float32, [2350] * 8, 4, 1714)],
                         ids=["bf16", "f32"])
def test_a_window_takes_the_workspace_of_the_call_without_one(heads, dtype, lens, new, window):
    """One workspace for a model's layers with and without a window, where fewer keys would be cut into more pieces."""
    c = Case(heads, 16, lens, [new] * len(lens), dtype, seed=17, rows_behind=0)
    s, cache = c.sequences(max_len=max(lens)), uad.PagedCache(c.k, c.v)
    q = c.randn(c.rows, c.hq * c.dh)
    ws = torch.full((cache.attention_workspace(s, c.rows, c.hq) + 64,), 255, dtype=torch.uint8, device="cuda")
    for w in (window, 0):
        out, lse = torch.empty_like(q), torch.empty(c.rows, c.hq, device="cuda")
        cache.attention(s, q, out, ws[:-64], window=w, lse=lse)
        torch.cuda.synchronize()
        assert bool((ws[-64:] == 255).all())
        check_attention(c, q, out, lse, window=w)


@pytest.mark.parametrize("heads,n,longest,new", [((8, 8, 256), 38, 60, 1), ((8, 8, 256), 51, 60, 1), ((16, 16, 256), 51, 70, 1), ((16, 4, 256), 76, 50, 3), ((128, 4, 128), 76, 40, 1),
                                                 ((128, 4, 128), 102, 40, 1), ((32, 8, 128), 102, 60, 1), ((64, 8, 128), 60, 50, 1), ((32, 8, 64), 76, 130, 1), ((64, 4, 64), 130, 40, 2)],
                         ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else str(x))
def test_heads_to_warps_or_to_ctas(heads, n, longest, new):
    """Sizes on both sides of where a CTA's warps get heads of their own, every head size, 8 to 32 rows."""
    lens = [max(new, 1 + (41 * i) % longest) for i in range(n)]
    lens[-1] = longest
    c = Case(heads, 16, lens, [new] * n, seed=n + heads[2])
    q, out, lse, status = run_attention(c, max_len=longest)
    assert status == 0
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [0.0, -0.0, 0, 1e-60])
def test_a_scale_of_zero_is_not_the_default(scale, dtype):
    """Every seen key has the same weight: the mean of the values, and the logarithm of their number. (The scores, below 2^10,
    vanish beside 1 with fp32's least scale, so the errors are those of the sum, as for any scale.)"""
    c = Case((8, 2, 64), 16, [40, 700, 1, 65], [3, 1, 1, 9], dtype, seed=18)
    mask = torch.ones((c.n, c.width * c.page), dtype=torch.uint8, device="cuda")
    mask[1, 100:650] = 0
    q, out, lse, status = run_attention(c, mask=mask, scale=scale)
    assert status == 0
    mn = mask.cpu().numpy()
    for t, (b, pos) in enumerate(paged.rows_of(c.lens, c.start)):
        seen = np.flatnonzero(mn[b, :pos + 1])
        for h in range(c.hq):
            v = c.values[b][seen, h // 4]
            want, size, n = v.mean(axis=0), np.abs(v).mean(axis=0), len(seen)
            tol = 2 * (2.0 ** -20 + 2.0 ** -16 + n * 2.0 ** -23) * size + HALF[dtype] * np.abs(want) + TINY
            assert np.all(np.abs(out[t, h * 64:(h + 1) * 64].double().cpu().numpy() - want) <= tol)
            assert abs(float(lse[t, h]) - math.log(n)) <= 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -22 * math.log(n)


def test_a_call_that_cannot_be_launched_leaves_no_error_behind():
    """A call on the legacy stream while a stream that it waits for is captured is refused by the runtime. The error is that call's alone: uad_linear,
    which asks for the last error, does not find it."""
    rt = C.CDLL(next(m.split()[-1] for m in open("/proc/self/maps") if "libcudart.so" in m))   # the runtime that torch has loaded
    c = Case((8, 2, 64), 16, [40], [1], seed=19, rows_behind=0)
    s, cache, rope = c.sequences(), uad.PagedCache(c.k, c.v), uad.rope(10000.0, 64)
    q, k = c.randn(1, 512), c.randn(1, 128)
    out = torch.empty_like(q)
    ws = torch.empty(max(1, cache.attention_workspace(s, 1, 8)), dtype=torch.uint8, device="cuda")
    w, scale, y = torch.zeros(32, 256, dtype=torch.uint8, device="cuda"), torch.ones(32, 8, device="cuda").bfloat16(), torch.empty(1, 32, device="cuda")
    tiled = torch.from_numpy(uad.tile_weight(np.zeros((512, 128), np.float32)).view(np.int16)).cuda()
    z = torch.full((1, 128), 7.5, device="cuda")
    st, graph = C.c_void_p(), C.c_void_p()
    assert rt.cudaStreamCreate(C.byref(st)) == 0   # a blocking stream: the legacy stream waits for it, which a capture cannot have
    calls = [lambda: cache.append(s, k, k, q=q, q_out=out, rope=rope), lambda: cache.attention(s, q, out, ws), lambda: uad.linear_w4(q, w, scale, y)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    for call in calls:
        assert rt.cudaStreamBeginCapture(st, 0) == 0
        try:
            with pytest.raises(uad.UADError) as e:
                call()
            assert e.value.code == uad.UAD_ECUDA
        finally:
            rt.cudaStreamEndCapture(st, C.byref(graph))
            rt.cudaGetLastError()
        assert uad.uad_linear(q.data_ptr(), tiled.data_ptr(), None, z.fill_(7.5).data_ptr(), 1, 128, 512, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert bool((z == 0).all())
    assert rt.cudaStreamDestroy(st) == 0
