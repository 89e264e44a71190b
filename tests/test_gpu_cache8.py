"""GPU parity of the paged cache held in 8 bits (append and attention) against the 64-bit oracle.

Tolerances. Scales are compared exactly: they come from the largest raw value by its bits. Codes of values that are not rotated are the
nearest ones, exactly. A rotated value is off by (|a| + |b|) 2^-22 before it is rounded (cos and sin by 2^-23, two products and a
sum by 2^-24 each); its code is then within half a step of e4m3 of that: 2^(e - 4) for a value of exponent e, 2^(-10) of the scale
at the least.
Attention: as for bf16 caches a score is off by d = dh 2^-23 scale sum |q k| (products of f16 are exact, the tensor cores truncate), and by
three more roundings for the scales: 2^-22 of it. Probabilities are off by e^d twice, by 2^-20 of exp, sums of n terms by n 2^-23; the weights are the sum of
two f16, 2^-21 relative and 2^-34 of the row's largest where they are small; allowed are 2^-11 and 2^-36 of the values' sum (test_gpu_cache8_weights has the
closer bounds). The output is off by that much of sum p |v|, then by bf16's half step.
"""
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged, paged8

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
CODES = torch.float8_e4m3fn


class Case8:
    """A batch over pools whose every slot and scale that no sequence holds is NaN; scales of any size."""

    def __init__(self, heads, page, lens, new, block=16, layout="pshd", seed=0, rows_behind=2, width=None, spare=5, powers=False):
        self.hq, self.hkv, self.dh = heads
        self.page, self.block = page, block
        self.rng = np.random.default_rng(seed)
        self.lens, self.new = list(lens), list(new)
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.n = len(self.lens)
        self.rows = int(self.start[-1]) + rows_behind
        used = [(n + page - 1) // page for n in self.lens]
        self.width = width or max(1, max(used))
        self.pages = sum(used) + spare
        ids = self.rng.permutation(self.pages).tolist()
        self.table = np.full((self.n, self.width), -1, np.int32)
        for b, u in enumerate(used):
            self.table[b, :u] = [ids.pop() for _ in range(u)]
        self.blocks = (page + block - 1) // block
        self.codes = [np.full((self.pages, page, self.hkv, self.dh), 0x7f, np.uint8) for _ in range(2)]
        self.scales = [np.full((self.pages, self.blocks, self.hkv), np.nan) for _ in range(2)]
        for b, n in enumerate(self.lens):
            for codes, scales in zip(self.codes, self.scales):
                for i in range(used[b]):
                    pg, held = self.table[b, i], min(page, n - i * page)
                    nb = (held + block - 1) // block
                    s = 2.0 ** self.rng.integers(-9, -3, (nb, self.hkv)) * (1 if powers else self.rng.uniform(0.6, 1.9, (nb, self.hkv)))
                    scales[pg, :nb] = s.astype(np.float32)
                    x = self.rng.normal(size=(held, self.hkv, self.dh))
                    codes[pg, :held] = paged8.encode((x * 100).clip(-448, 448))
        self.layout = layout

    def on_gpu(self):
        def put(x):
            t = torch.from_numpy(x).cuda()
            if self.layout == "phsd":
                t = t.transpose(1, 2).contiguous().transpose(1, 2)
            return t.view(CODES)
        k, v = put(self.codes[0]), put(self.codes[1])
        if self.layout == "joint":   # keys and values of a page next to each other
            both = torch.stack([k.view(torch.uint8), v.view(torch.uint8)], dim=1).view(CODES)
            k, v = both[:, 0], both[:, 1]
        ks, vs = (torch.from_numpy(s.astype(np.float32)).cuda() for s in self.scales)
        if self.layout != "pshd":   # scales of a head next to each other
            ks, vs = (s.permute(2, 0, 1).contiguous().permute(1, 2, 0) for s in (ks, vs))
        self.pools = k, v, ks, vs
        self.cache = uad.PagedCache(k, v, ks, vs, block=self.block)
        return self.cache

    def sequences(self, max_len=0, max_new=None):
        self.dev = [torch.from_numpy(x).cuda() for x in (self.table, np.array(self.lens, np.int32), self.start)]
        return uad.Sequences(*self.dev, max_len=max_len, max_new=max_new or max(1, max(self.new)))

    def token(self, b, pos):
        """(page, slot, block) of a token."""
        return int(self.table[b, pos // self.page]), pos % self.page, pos % self.page // self.block

    def held(self, b, which):
        """What a sequence's tokens stand for, [len][heads][dh]."""
        pos = np.arange(self.lens[b])
        pg, sl = self.table[b, pos // self.page], pos % self.page
        return paged8.VALUES[self.codes[which][pg, sl]] * self.scales[which].astype(np.float32).astype(np.float64)[pg, sl // self.block][..., None]

    def fetch(self):
        """The pools as they are on the GPU."""
        torch.cuda.synchronize()
        k, v, ks, vs = self.pools
        return [x.contiguous().view(torch.uint8).cpu().numpy() for x in (k, v)], [x.cpu().numpy().astype(np.float64) for x in (ks, vs)]


# ---- append ---------------------------------------------------------------------------------------------------------------


def make_rows(c, dtype, q=True, scale=None):
    width = (c.hq if q else 0) * c.dh
    x = c.rng.normal(size=(c.rows, width + 2 * c.hkv * c.dh))
    if scale is not None:
        x *= scale
    t = torch.from_numpy(x).cuda().to(dtype)
    return t[:, :width], t[:, width:width + c.hkv * c.dh], t[:, width + c.hkv * c.dh:]


def half_step(x, s):
    """Half a step of the codes around the values x of scale s."""
    e = np.floor(np.log2(np.maximum(np.abs(x) / s, 2.0 ** -30)))
    return s * 2.0 ** (np.maximum(e, -6) - 4)


def check_append(c, q, k, v, q_out, rope, dim, before):
    codes, scales = c.fetch()
    theta = 10000.0 if rope else None
    used = int(c.start[-1])
    where = paged.rows_of(c.lens, c.start)
    for which, (rows, turned) in enumerate(((k, theta), (v, None))):
        if rows is None:
            assert np.array_equal(codes[which], before[0][which]) and np.array_equal(scales[which], before[1][which], equal_nan=True)
            continue
        rows = rows.double().cpu().numpy()[:used].reshape(used, c.hkv, c.dh)
        want, ws = before[0][which].copy(), before[1][which].copy()
        exact, s = paged8.append(want, ws, c.table, c.lens, c.start, c.page, c.block, rows, turned, dim)
        assert np.array_equal(scales[which], ws, equal_nan=True), which
        if turned is None:
            same = codes[which] == want
            assert np.all(same | ((codes[which] & 127 == 127) & (want & 127 == 127))), which
            continue
        # tokens of the call by tolerance, everything else exactly
        near = np.zeros(codes[which].shape[:2], bool)
        for t, (b, pos) in enumerate(where):
            pg, sl, _ = c.token(b, pos)
            near[pg, sl] = True
            got = paged8.VALUES[codes[which][pg, sl]] * s[t][:, None]
            h = dim // 2
            mag = np.abs(rows[t]).copy()
            mag[..., :h] = mag[..., h:dim] = np.abs(rows[t][..., :h]) + np.abs(rows[t][..., h:dim])
            mag[..., dim:] = 0
            bad = ~np.isfinite(exact[t])
            assert np.array_equal(np.isnan(got), bad), (t, b, pos)
            err, off = np.abs(got - exact[t]), mag * 2.0 ** -22
            tol = half_step(np.abs(np.where(bad, 0, exact[t])) + off, s[t][:, None]) + off
            assert np.all((err <= tol) | bad), (t, b, pos, float(np.nanmax(err / tol)))
        assert np.array_equal(codes[which][~near], want[~near])
    if q is not None:
        qn, got = q.double().cpu().numpy(), q_out.double().cpu().numpy()
        for t, (b, pos) in enumerate(where):
            x = qn[t].reshape(c.hq, c.dh)
            want = x if theta is None else paged.rotate(x, pos, theta, dim)
            mag = np.abs(x).copy()
            if theta is not None:
                h = dim // 2
                mag[..., :h] = mag[..., h:dim] = np.abs(x[..., :h]) + np.abs(x[..., h:dim])
            assert np.all(np.abs(got[t].reshape(c.hq, c.dh) - want) <= mag * 2.0 ** -22 + HALF * np.abs(want)), t
        assert bool((q_out[used:] == 7.5).all())


def run_append(c, dtype, rope=True, dim=None, q=True, kv=True, rows=None, stream=None):
    cache = c.on_gpu()
    qt, kt, vt = rows or make_rows(c, dtype, q)
    dim = dim or c.dh
    q_out = torch.full((c.rows, c.hq * c.dh), 7.5, device="cuda", dtype=torch.bfloat16) if q else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = c.fetch()
    cache.append(c.sequences(), kt if kv else None, vt if kv else None, q=qt if q else None, q_out=q_out,
                 rope=uad.rope(10000.0, dim) if rope else None, status=status, stream=stream)
    check_append(c, qt if q else None, kt if kv else None, vt if kv else None, q_out, rope, dim, before)
    return int(status)


HEADS = [(8, 1, 256), (4, 1, 128), (8, 2, 64), (24, 24, 64), (32, 8, 128), (3, 3, 256), (6, 5, 128)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_append(heads, block, dtype):
    """Whole prompts, single tokens that open a block, end one, join one and pass from one to the next; a sequence without any."""
    c = Case8(heads, 64, [70, 1, 65, 64, 40, 17, 0, 130, 33], [70, 1, 1, 1, 3, 16, 0, 67, 0], block, seed=sum(heads) + block)
    assert run_append(c, dtype) == 0


@pytest.mark.parametrize("page,layout,block", [(1, "pshd", 16), (5, "phsd", 16), (12, "joint", 32), (100, "pshd", 64), (100, "phsd", 16), (128, "joint", 64),
                                               (48, "phsd", 32)])
def test_append_to_blocks_that_end_with_odd_pages(page, layout, block):
    c = Case8((4, 2, 64), page, [3, 150, 101, 260, 90], [3, 7, 1, 120, 0], block, layout, seed=page)
    assert run_append(c, torch.bfloat16) == 0


@pytest.mark.parametrize("dim,rope,q,kv", [(32, True, True, True), (48, True, True, True), (128, False, True, True), (128, True, False, True),
                                           (128, True, True, False), (16, True, False, True)])
def test_append_of_parts(dim, rope, q, kv):
    """Part of each head rotated, nothing rotated, without queries, queries alone."""
    c = Case8((5, 3, 128), 16, [9, 40, 35], [9, 2, 20], 16, seed=dim)
    assert run_append(c, torch.float32, rope, dim, q, kv) == 0


def test_scales_grow_and_earlier_tokens_follow():
    """A block's earlier tokens keep their scale where the new ones are smaller and are rounded to the new one where they are larger,
    by powers of two and by other ratios (a cache that was rounded elsewhere)."""
    for powers in (True, False):
        for factor in (1e-3, 1.0, 40.0, 3e5):
            c = Case8((2, 2, 64), 32, [20, 45, 31, 64], [3, 1, 11, 16], 32, seed=1, powers=powers)
            rows = make_rows(c, torch.float32, True, factor)
            assert run_append(c, torch.float32, rows=rows) == 0


def test_borders_of_the_scales():
    """Largest values at and next to 448 times a power of two, zeros, subnormal and huge ones, infinities and NaN, which do not count."""
    c = Case8((1, 1, 64), 16, [16] * 14, [16] * 14, 16, seed=2, rows_behind=0)
    x = np.zeros((c.rows, 64), np.float32)
    top = np.float32(448)
    for b, value in enumerate([448.0, np.nextafter(top, np.float32(500)), np.nextafter(top, np.float32(0)), 449.0, 0.0, 1e-40, 3e38, 1.75 * 2.0 ** -60,
                               2.0 ** -92, 1e-33, 3.5, -7.0, 1e4, 2.0 ** -133]):
        x[16 * b + 5, 7] = value
        x[16 * b + 9, 3] = value / 3
    x[16 * 10 + 2, 0], x[16 * 11, 63], x[16 * 12, 1] = np.inf, np.nan, -np.inf
    t = torch.from_numpy(x).cuda()
    empty = t[:, :64]
    assert run_append(c, torch.float32, rope=False, q=False, rows=(empty, t, t.clone())) == 0


def test_a_cache_hardly_depends_on_how_it_was_written():
    """Token by token, in drafts and at once: the same scales, and the same values where they are normal numbers of the last scale."""
    heads, n = (1, 2, 128), 100
    rows = torch.randn(n, 3 * 128 * 2, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    rows *= torch.exp2(torch.randint(-6, 7, (n, 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).float())
    k, v = rows[:, :256], rows[:, 256:512]
    rope = uad.rope(10000.0, 128)
    got = []
    for steps in ([n], [1] * n, [7] * 14 + [2], [33, 1, 1, 40, 25]):
        c = Case8(heads, 24, [n], [n], 16, seed=4)
        cache, at = c.on_gpu(), 0
        for s in steps:
            at += s
            seqs = uad.Sequences(torch.from_numpy(c.table).cuda(), torch.tensor([at], dtype=torch.int32, device="cuda"),
                                 torch.tensor([0, s], dtype=torch.int32, device="cuda"), max_new=s)
            cache.append(seqs, k[at - s:at], v[at - s:at], rope=rope)
        got.append(c.fetch())
    for which in range(2):
        pos = np.arange(n)
        pg, sl = c.table[0, pos // 24], pos % 24
        codes, scales = got[0][0][which][pg, sl], got[0][1][which][pg, sl // 16]
        for other in got[1:]:
            assert np.array_equal(other[1][which][pg, sl // 16], scales)
            theirs = other[0][which][pg, sl]
            normal = codes & 0x78 != 0
            assert np.array_equal(theirs[normal], codes[normal])
            # a subnormal is rounded again by each growth: half a step of the last scale each, of which there are few
            assert np.abs(paged8.VALUES[theirs] - paged8.VALUES[codes]).max() <= 4 * 2.0 ** -9


def test_append_leaves_out_bad_pages_and_sequences():
    c = Case8((2, 1, 64), 16, [20, 40, 33, 64], [4, 4, 4, 4], 16, seed=5)
    good = c.table.copy()
    for bad_table, bad_len, bit in (({(0, 1): -1, (2, 2): c.pages}, {}, uad.UAD_KV_BAD_PAGE), ({}, {1: 4 * 16 + 1, 3: 3}, uad.UAD_KV_BAD_SEQ)):
        cache = c.on_gpu()
        before = c.fetch()
        c.table = good.copy()
        for at, x in bad_table.items():
            c.table[at] = x
        lens = list(c.lens)
        for b, x in bad_len.items():
            lens[b] = x
        q, k, v = make_rows(c, torch.float32)
        q_out = torch.full((c.rows, 128), 7.5, device="cuda", dtype=torch.bfloat16)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        seqs = uad.Sequences(torch.from_numpy(c.table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.from_numpy(c.start).cuda(), max_new=4)
        cache.append(seqs, k, v, q=q, q_out=q_out, status=status)
        codes, scales = c.fetch()
        assert int(status) == bit
        want, ws = [x.copy() for x in before[0]], [x.copy() for x in before[1]]
        left_out = [0, 2] if bad_table else [1, 3]
        for which, rows in enumerate((k, v)):
            r = rows.double().cpu().numpy().reshape(c.rows, 1, 64)
            for b in set(range(4)) - set(left_out):
                paged8.append(want[which], ws[which], good[b:b + 1], [c.lens[b]], [0, 4], 16, 16, r[c.start[b]:c.start[b + 1]])
            if bad_table:   # of the third sequence's tokens 29 to 32 the last one alone is on the bad page
                paged8.append(want[which], ws[which], good[2:3], [32], [0, 3], 16, 16, r[c.start[2]:c.start[2] + 3])
            assert np.array_equal(codes[which], want[which]) and np.array_equal(scales[which], ws[which], equal_nan=True)
        for b in range(4):
            assert bool((q_out[c.start[b]:c.start[b + 1]] == 7.5).all()) == (b in left_out and not bad_table)
        c.table = good


# ---- attention --------------------------------------------------------------------------------------------------------------


def run_attention(c, causal=True, window=0, sinks=0, mask=None, scale=None, max_len=0, fused=False, stream=None, q=None):
    width = c.hq * c.dh
    if q is None:
        q = torch.from_numpy(c.rng.normal(size=(c.rows, width + 16))).cuda().bfloat16()
        q = q[:, :width] if fused else q[:, :width].contiguous()
    out = torch.full((c.rows, width + (8 if fused else 0)), 7.5, device="cuda", dtype=torch.bfloat16)[:, :width]
    lse = torch.full((c.rows, c.hq), 7.5, device="cuda")
    s, cache = c.sequences(max_len), c.on_gpu()
    ws = torch.full((cache.attention_workspace(s, c.rows, c.hq, window, sinks) + 64,), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    cache.attention(s, q, out, ws[:-64], scale=scale, causal=causal, window=window, sinks=sinks, key_mask=mask, lse=lse, status=status, stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[-64:] == 255).all())
    used = int(c.start[-1])
    assert bool((out[used:] == 7.5).all()) and bool((lse[used:] == 7.5).all())   # rows of nobody
    return q, out, lse, int(status)


def check_attention(c, q, out, lse, causal=True, window=0, sinks=0, mask=None, scale=None):
    scale = 1 / math.sqrt(c.dh) if scale is None else scale
    qn, on, ln = q.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    mn = None if mask is None else mask.cpu().numpy()
    group, worst = c.hq // c.hkv, 0.0
    held = [(c.held(b, 0), c.held(b, 1)) for b in range(c.n)]
    for t, (b, pos) in enumerate(paged.rows_of(c.lens, c.start)):
        j = np.arange(c.lens[b])
        seen = np.ones(c.lens[b], bool)
        if causal:
            seen &= j <= pos
        if window:
            seen &= (j > pos - window) | (j < sinks)
        if mn is not None:
            seen &= mn[b, :c.lens[b]] != 0
        n = int(seen.sum())
        for h in range(c.hkv):
            rows = qn[t].reshape(c.hq, c.dh)[h * group:(h + 1) * group]
            k, v = held[b][0][:, h], held[b][1][:, h]
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
                d = (c.dh * 2.0 ** -23 + 2.0 ** -22) * abs(scale) * (np.abs(rows) @ np.abs(k[seen]).T).max(axis=1, keepdims=True)
                rel = 2 * (2 * d + 2.0 ** -20 + n * 2.0 ** -23) + 2.0 ** -11
                tol = rel * (p @ np.abs(v[seen])) + HALF * np.abs(want) + 2.0 ** -36 * np.abs(v[seen]).sum(axis=0) + 1e-30
                err = np.abs(got - want)
                assert np.all((err <= tol) | bad), (t, h, float(np.nanmax(err / tol)))
                assert np.all((np.abs(gl - wl) <= d[:, 0] + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -22 * np.abs(wl)) | np.isnan(wl)), (t, h, gl, wl)
            worst = max(worst, float(np.nanmax(err / tol)))
    return worst


MORE = HEADS[:-1] + [(10, 5, 128), (21, 1, 64), (128, 2, 128), (40, 2, 256)]


@pytest.mark.parametrize("heads", MORE, ids=lambda h: "x".join(map(str, h)))
def test_attention_of_one_token(heads):
    """Lengths of one token and around the pages, tiles and pieces; a sequence without new tokens; one token that is all."""
    c = Case8(heads, 16, [1, 2, 15, 16, 17, 63, 64, 65, 200, 0, 333, 40], [1, 1, 1, 1, 1, 1, 1, 1, 1, 0, 1, 0], seed=sum(heads))
    q, out, lse, status = run_attention(c)
    assert status == 0
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("page,layout,block", [(1, "pshd", 16), (5, "phsd", 16), (12, "joint", 16), (100, "pshd", 64), (128, "phsd", 32), (16, "joint", 64),
                                               (40, "pshd", 32)])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 37, 0), (False, 70, 9), (True, 30, 4)])
def test_attention_of_a_few_tokens(page, layout, block, causal, window, sinks):
    """Drafts and chunks of different lengths, ends of pages and blocks inside of tiles, windows, fused rows, every layout."""
    c = Case8((8, 2, 64), page, [3, 40, 129, 700, 64, 9], [3, 5, 1, 16, 0, 9], block, layout, seed=page)
    q, out, lse, status = run_attention(c, causal, window, sinks, fused=True)
    assert status == 0
    check_attention(c, q, out, lse, causal, window, sinks)


@pytest.mark.parametrize("heads,new", [((8, 1, 256), 1), ((8, 1, 256), 5), ((16, 2, 128), 1), ((16, 2, 128), 3), ((16, 2, 128), 7), ((8, 8, 64), 4), ((20, 4, 128), 2)],
                         ids=lambda h: str(h))
def test_attention_with_key_masks(heads, new):
    """Masked cameras, single keys left, and rows that see nothing at all (output 0, lse -inf)."""
    c = Case8(heads, 16, [90, 300, 33, 64, 5 + new], [new] * 5, seed=7)
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


@pytest.mark.parametrize("heads", [(8, 1, 256), (4, 2, 128), (8, 8, 64), (16, 4, 64)], ids=lambda h: "x".join(map(str, h)))
def test_what_a_token_does_not_see_has_no_influence(heads):
    """NaN codes of later tokens of the call, before the window, in masked places; what sees them is NaN."""
    for window, sinks in ((0, 0), (20, 0), (20, 3)):
        c = Case8(heads, 16, [37, 80], [6, 3], seed=11)

        def put(b, pos, which, code):
            pg, sl, _ = c.token(b, pos)
            c.codes[which][pg, sl] = code

        for pos in (33, 34, 36):   # tokens of the call itself
            put(0, pos, 0, 0x7f)
            put(0, pos, 1, 0xff)
        put(0, 32, 1, 0x7f) if heads[2] == 64 else None   # values alone: the scores are sound
        mask = torch.ones((c.n, c.width * c.page), dtype=torch.uint8, device="cuda")
        for pos in (3, 50, 78):
            put(1, pos, 0, 0x7f)
            put(1, pos, 1, 0x7f)
            mask[1, pos] = 0
        if window:
            put(1, 58, 1, 0x7f)   # the first of the three rows sees 58 to 77, the others do not
            pg, sl, _ = c.token(1, 59)
            c.codes[1][pg, sl, 0, 5] = 0xff   # one dim of one head: rows 0 and 1 see it
        q, out, lse, status = run_attention(c, True, window, sinks, mask)
        assert status == 0
        check_attention(c, q, out, lse, True, window, sinks, mask)


def test_scales_and_scores_far_apart():
    """Values' scales that grow and fall by 2^20 along a sequence, a key that takes all, keys' scales of 2^-90, queries of 1e-20 and 1e20."""
    c = Case8((4, 2, 64), 16, [300, 300, 300, 300], [1, 1, 2, 1], seed=8)
    used = [c.table[b, :19] for b in range(4)]
    for i in range(19):
        c.scales[1][used[0][i]] = np.float32(2.0 ** (i * 2 - 20) * 1.3)
        c.scales[1][used[1][i]] = np.float32(2.0 ** (20 - i * 2))
    pg, sl, _ = c.token(2, 250)
    c.codes[0][pg, sl] = 0x7e   # 448 everywhere
    c.scales[0][used[3]] = 2.0 ** -90
    q = torch.from_numpy(c.rng.normal(size=(c.rows, 256))).cuda().bfloat16()
    q[3] *= 2.0 ** 20
    q, out, lse, status = run_attention(c, q=q)
    assert status == 0
    check_attention(c, q, out, lse)
    for factor, scale in ((2.0 ** 66, 2.0 ** -69), (2.0 ** -70, 2.0 ** 67)):
        x = q * factor
        x, out, lse, status = run_attention(c, q=x, scale=scale)
        check_attention(c, x, out, lse, scale=scale)


def test_queries_that_are_not_finite_and_zero():
    c = Case8((2, 1, 128), 16, [40, 40, 40], [1, 1, 1], seed=9)
    q = torch.from_numpy(c.rng.normal(size=(c.rows, 256))).cuda().bfloat16()
    q[0, 3] = math.nan
    q[1, :] = 0
    q[2, 130] = math.nan
    q, out, lse, status = run_attention(c, q=q)
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("max_len", [0, 1, 100, 5000])
@pytest.mark.parametrize("heads", [(8, 1, 256), (8, 2, 64), (32, 8, 128)], ids=lambda h: "x".join(map(str, h)))
def test_long_caches_are_split_and_joined(heads, max_len):
    """The work's split follows max_len, right or wrong; shorter and longer sequences beside each other."""
    c = Case8(heads, 64, [5000, 3, 1900, 4097, 64], [2, 1, 1, 4, 1], 64, seed=5)
    q, out, lse, status = run_attention(c, max_len=max_len)
    assert status == 0
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("heads,new", [((8, 1, 256), 1), ((8, 1, 256), 3), ((32, 8, 128), 1), ((8, 2, 128), 4), ((8, 2, 128), 8), ((24, 24, 64), 1), ((8, 2, 64), 3),
                                       ((16, 2, 64), 4), ((21, 1, 64), 5)], ids=lambda h: str(h))
@pytest.mark.parametrize("causal,window,sinks,masked", [(True, 0, 0, False), (False, 0, 0, True), (True, 90, 5, False), (True, 300, 0, True)])
def test_keys_that_are_shared_evenly(heads, new, causal, window, sinks, masked):
    """Tables so wide that the work is split for long sequences: parts that end inside of sequences, at their ends and behind the last one, sequences
    without new tokens, with fewer rows than others, shorter than a chunk, and one that several parts share."""
    c = Case8(heads, 16, [1500, 40, 0, 128, 257, 1, 700, 64, 33, 2900], [new, 1, 0, new, 0, 1, new, 1, new, new], seed=new, width=60000)
    mask = None
    if masked:
        mask = torch.ones((c.n, c.width * c.page), dtype=torch.uint8, device="cuda")
        mask[0, 100:1400] = 0
        mask[3] = 0
        mask[9, ::3] = 0
    q, out, lse, status = run_attention(c, causal, window, sinks, mask, max_len=900000)
    assert status == 0
    check_attention(c, q, out, lse, causal, window, sinks, mask)


def test_keys_that_are_shared_evenly_with_bad_sequences():
    """Many sequences, one of which has a length that its table does not hold: it is left out, the others are served."""
    lens = [1 + 37 * i % 400 for i in range(140)]
    c = Case8((8, 4, 64), 16, lens, [1] * 140, seed=3, width=30000)
    s, cache = c.sequences(400000), c.on_gpu()
    c.dev[1][77] = -5
    q = torch.from_numpy(c.rng.normal(size=(c.rows, 512))).cuda().bfloat16()
    out, lse = torch.full((c.rows, 512), 7.5, device="cuda", dtype=torch.bfloat16), torch.full((c.rows, 8), 7.5, device="cuda")
    ws = torch.empty(cache.attention_workspace(s, c.rows, 8), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.attention(s, q, out, ws, lse=lse, status=status)
    torch.cuda.synchronize()
    assert int(status) == uad.UAD_KV_BAD_SEQ and bool((out[77] == 7.5).all()) and bool((lse[77] == 7.5).all())
    keep = [i for i in range(140) if i != 77]
    c.table, c.lens, c.n, c.start = c.table[keep], [lens[i] for i in keep], 139, np.arange(140)
    check_attention(c, q[keep], out[keep], lse[keep])


@pytest.mark.parametrize("heads", [(8, 1, 64), (24, 24, 64), (8, 4, 128), (8, 8, 256)], ids=lambda h: "x".join(map(str, h)))
def test_many_sequences(heads):
    """Enough short sequences that warps have heads of their own, and enough that one CTA has a sequence."""
    c = Case8(heads, 16, [1 + 7 * i % 90 for i in range(150)], [1] * 150, seed=6)
    q, out, lse, status = run_attention(c, max_len=90)
    assert status == 0
    check_attention(c, q, out, lse)


def test_attention_leaves_out_bad_pages():
    c = Case8((4, 2, 64), 16, [70, 40], [2, 1], seed=12)
    mask = torch.ones((2, c.width * 16), dtype=torch.uint8, device="cuda")
    good = c.table.copy()
    c.table[0, 1], c.table[1, 0] = -7, c.pages
    q, out, lse, status = run_attention(c)
    assert status == uad.UAD_KV_BAD_PAGE
    c.table = good
    mask[0, 16:32] = 0
    mask[1, :16] = 0
    check_attention(c, q, out, lse, mask=mask)


@pytest.mark.parametrize("layout", ["apart", "joint"])
def test_offsets_past_32_bits(layout):
    """The same tokens in the first pages of a small pool and the last ones of pools of more than 2^32 bytes: the same bits."""
    c = Case8((8, 1, 256), 64, [200, 65, 333], [5, 1, 70], 32, seed=21)
    cache = c.on_gpu()
    n = 300000   # pages of 16 KiB
    if layout == "apart":
        k, v = (torch.empty((n, 64, 1, 256), dtype=torch.uint8, device="cuda").view(CODES) for _ in range(2))
    else:
        both = torch.empty((n, 2, 64, 1, 256), dtype=torch.uint8, device="cuda").view(CODES)
        k, v = both[:, 0], both[:, 1]
    ks, vs = (torch.empty((n, 2, 1), device="cuda") for _ in range(2))
    shift = n - c.pages
    for far, near in ((k, cache.k), (v, cache.v)):
        far[shift:].view(torch.uint8).copy_(near.view(torch.uint8))
    ks[shift:], vs[shift:] = cache.k_scale, cache.v_scale
    big = uad.PagedCache(k, v, ks, vs, block=32)
    small, seqs = c.sequences(), c.dev
    table = torch.where(seqs[0] >= 0, seqs[0] + shift, seqs[0])
    large = uad.Sequences(table, seqs[1], seqs[2], max_new=70)
    x = torch.randn(c.rows, 10 * 256, device="cuda")
    got = []
    for kv, s in ((cache, small), (big, large)):
        q = torch.zeros(c.rows, 2048, device="cuda", dtype=torch.bfloat16)
        out = torch.zeros_like(q)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kv.append(s, x[:, 2048:2304], x[:, 2304:], q=x[:, :2048], q_out=q, rope=uad.rope(10000.0, 256), status=status)
        ws = torch.empty(kv.attention_workspace(s, c.rows, 8), dtype=torch.uint8, device="cuda")
        kv.attention(s, q, out, ws, status=status)
        torch.cuda.synchronize()
        assert int(status) == 0
        got.append((out, kv.k.view(torch.uint8)[-c.pages:].clone(), kv.v.view(torch.uint8)[-c.pages:].clone(), kv.k_scale[-c.pages:].clone(), kv.v_scale[-c.pages:].clone()))
    assert torch.equal(got[0][0], got[1][0])
    for a, b in zip(got[0][1:], got[1][1:]):
        assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b)


def test_the_same_every_time():
    c = Case8((8, 1, 256), 16, [4000, 17, 900], [3, 1, 2], seed=12)
    s, cache = c.sequences(), c.on_gpu()
    q = torch.randn(c.rows, 2048, device="cuda").bfloat16()
    ws = torch.empty(cache.attention_workspace(s, c.rows, 8), dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(4):
        out = torch.empty_like(q)
        cache.attention(s, q, out, ws)
        outs.append(out)
    torch.cuda.synchronize()
    used = int(c.start[-1])
    assert all(torch.equal(outs[0][:used], o[:used]) for o in outs[1:])
