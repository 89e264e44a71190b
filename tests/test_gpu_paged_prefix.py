"""The paged cache's operators and the 4-bit projection as a vision-language model beside the expert uses them: a small decoder
whose every operator is checked against its 64-bit reference on what the GPU gave it, prompts in pieces and then token by token
from a CUDA graph, and the expert's prefix bound from the pages.

Tolerances: each operator's own, as derived beside its own tests. The whole decoder against a 64-bit one without roundings: a
row meets five roundings to bf16 a layer (projection input, query, key, value, attention output), each of at most 2^-8 of
its size; scores stay below 1/2 in size here, so a rounding of the query or key moves a probability by less than it moves a
value, and nothing between the roundings amplifies more than twice: 2 * 5 * layers * 2^-8 of what the layers add.
"""
import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged
from test_gpu_linear_w4 import check, reference
from test_gpu_paged import HALF
from uad_inputs import ARCHS, group_budgets, make_noise, make_weights

pytestmark = pytest.mark.gpu
TIMEOUT = 120_000_000
THETA = 10000.0


def pools(a, n_pages, page, dtype, layout):
    if layout == "joint":
        pool = torch.full((a.n_layers, n_pages, 2, page, a.n_kv_heads, a.head_dim), float("nan"), device="cuda", dtype=dtype).transpose(1, 2)
    elif layout == "phsd":
        pool = torch.full((a.n_layers, 2, n_pages, a.n_kv_heads, page, a.head_dim), float("nan"), device="cuda", dtype=dtype).transpose(3, 4)
    else:
        pool = torch.full((a.n_layers, 2, n_pages, page, a.n_kv_heads, a.head_dim), float("nan"), device="cuda", dtype=dtype)
    return [uad.PagedCache(p[0], p[1]) for p in pool]


def chunk(ex, a, seed=3):
    bud = group_budgets(a.chunk_len, [(0, 3, 2), (4, a.chunk_len - 1, 4)])
    ex.denoise(make_noise(a, seed=seed), bud[None])
    r = ex.finish(timeout_us=TIMEOUT)
    return r["final"].copy(), r["ghost"].copy()


def same(a, got, want):
    """The same bits; but the bf16 expert with adaptive norms adds up partial sums in the order in which they are ready, so that two
    runs of one prefix differ too: there, the tolerance of a chunk."""
    if a.kind == "adarms" and a.dtype == "bf16":
        return all(np.abs(x - y).max() <= 2e-2 * np.abs(y).max() for x, y in zip(got, want))
    return all(np.array_equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("name", ["tiny", "tiny_f32_rope", "pi0_small", "concat_small"])
@pytest.mark.parametrize("dtype,layout,page", [(torch.float32, "pshd", 16), (torch.bfloat16, "phsd", 5), (torch.bfloat16, "joint", 64), (torch.float32, "joint", 1),
                                               (torch.bfloat16, "pshd", 1000)])
def test_prefix_from_pages(name, dtype, layout, page):
    """The bits of the same prefix given as a contiguous buffer; the table on the host or the GPU, longer than the prefix."""
    a = ARCHS[name]
    used = (a.prefix_len + page - 1) // page
    caches = pools(a, used + 6, page, dtype, layout)
    g = torch.Generator().manual_seed(page)
    table = torch.randperm(used + 6, generator=g)[:used + 2].to(torch.int32)
    kv = torch.randn((2, a.n_layers, a.prefix_len, a.n_kv_heads, a.head_dim), generator=g).to(dtype).cuda()
    at = torch.arange(a.prefix_len)
    pg, sl = table[at // page].long().cuda(), (at % page).cuda()
    for l, c in enumerate(caches):
        c.k[pg, sl], c.v[pg, sl] = kv[0, l], kv[1, l]
    ex = uad.Expert(a, make_weights(a, seed=4), max_batch=2)
    try:
        other = torch.randn(kv.shape[1:], generator=g).cuda()
        code = "f32" if dtype == torch.float32 else "bf16"
        ex.set_prefix(0, kv[0].contiguous(), kv[1].contiguous(), dtype=code)
        want = chunk(ex, a)
        for t in (table, table.cuda(), table.numpy(), table.tolist(), table[:used]):
            ex.set_prefix(0, other, other)
            ex.set_prefix_paged(0, caches, t)
            got = chunk(ex, a)
            assert same(a, got, want)
    finally:
        ex.close()


def test_prefix_from_pages_refusals():
    a = ARCHS["pi0_small"]
    caches = pools(a, 20, 16, torch.bfloat16, "pshd")
    for c in caches:
        c.k.zero_()
        c.v.fill_(0.5)
    table = list(range(13))
    ex = uad.Expert(a, make_weights(a, seed=4), max_batch=1)
    dit = uad.Expert(ARCHS["dit_small"], make_weights(ARCHS["dit_small"], seed=4), max_batch=1)
    wrong_head = [uad.PagedCache(c.k[..., :64], c.v[..., :64]) for c in caches]
    f32 = [caches[0], uad.PagedCache(caches[1].k.float(), caches[1].v.float())]
    fewer = [caches[0], uad.PagedCache(caches[1].k[:10], caches[1].v[:10])]
    longer = [caches[0], uad.PagedCache(caches[1].k.reshape(10, 32, 1, 128), caches[1].v.reshape(10, 32, 1, 128))]
    try:
        ex.set_prefix_paged(0, caches, table)
        want = chunk(ex, a)
        for robot, cs, t in ((1, caches, table), (-1, caches, table), (0, caches[:1], table), (0, [], table), (0, caches * 2, table), (0, wrong_head, table),
                             (0, f32, table), (0, fewer, table), (0, longer, table), (0, caches, table[:12]), (0, caches, []),
                             (0, caches, table[:12] + [20]), (0, caches, [-1] + table[1:])):
            with pytest.raises(uad.UADError) as e:
                ex.set_prefix_paged(robot, cs, t)
            assert e.value.args and "set_prefix_paged" in str(e.value)
        with pytest.raises(ValueError, match="one sequence"):
            ex.set_prefix_paged(0, caches, np.zeros((1, 13), np.int32))
        with pytest.raises(ValueError, match="int32"):
            ex.set_prefix_paged(0, caches, np.zeros(13, np.int64))
        with pytest.raises(uad.UADError, match="DiT"):
            dit.set_prefix_paged(0, caches, table)
        got = chunk(ex, a)   # a refused call leaves the prefix as it was
        assert same(a, got, want)
        bud = group_budgets(a.chunk_len, [(0, 3, 2), (4, a.chunk_len - 1, 4)])
        ex.denoise(make_noise(a, seed=3), bud[None])
        with pytest.raises(uad.UADError, match="in flight"):
            ex.set_prefix_paged(0, caches, table)
        got = ex.finish(timeout_us=TIMEOUT)
        assert same(a, (got["final"], got["ghost"]), want)
    finally:
        ex.close()
        dit.close()


class Decoder:
    """Layers of projection, append, attention and projection with a residual; 4-bit weights."""

    def __init__(self, a, lens, room, seed):
        rng = np.random.default_rng(seed)
        self.a, self.page, self.n = a, 12, len(lens)
        self.hq, self.hkv, self.dh, self.width = a.n_heads, a.n_kv_heads, a.head_dim, a.width
        self.weights = []
        for _ in range(a.n_layers):
            pair = []
            for k, n in ((self.width, (self.hq + 2 * self.hkv) * self.dh), (self.hq * self.dh, self.width)):
                q, s, z = uad.quantize_w4((rng.normal(size=(k, n)) * k ** -0.5 * (0.5 if n != self.width else 1)).astype(np.float32), 64)
                pair.append((torch.from_numpy(q).cuda(), torch.from_numpy(s.view(np.int16)).cuda().view(torch.bfloat16), torch.from_numpy(z).cuda()))
            self.weights.append(pair)
        self.wide = (max(lens) + room + self.page - 1) // self.page
        self.caches = pools(a, self.n * self.wide + 3, self.page, torch.bfloat16, "phsd")
        self.table = torch.from_numpy(rng.permutation(self.n * self.wide + 3)[:self.n * self.wide].astype(np.int32).reshape(self.n, self.wide)).cuda()
        self.rope = uad.rope(THETA, self.dh)

    def buffers(self, rows, seqs):
        f = lambda n, t: torch.full((rows, n), 7.5, device="cuda", dtype=t)
        ws = torch.empty(max(1, max(c.attention_workspace(seqs, rows, self.hq) for c in self.caches)), dtype=torch.uint8, device="cuda")
        per = [dict(x=f(self.width, torch.bfloat16), qkv=f((self.hq + 2 * self.hkv) * self.dh, torch.float32), q=f(self.hq * self.dh, torch.bfloat16),
                    o=f(self.hq * self.dh, torch.bfloat16), y=f(self.width, torch.float32)) for _ in self.caches]
        return dict(h=f(self.width, torch.float32), ws=ws, per=per)

    def step(self, b, seqs, status, stream=None):
        """h -> h + layers, in place; everything in between stays in the buffers."""
        d, kv = self.hq * self.dh, self.hkv * self.dh
        for (wi, wo), c, p in zip(self.weights, self.caches, b["per"]):
            p["x"].copy_(b["h"])
            uad.linear_w4(p["x"], wi[0], wi[1], p["qkv"], zero=wi[2], stream=stream)
            c.append(seqs, p["qkv"][:, d:d + kv], p["qkv"][:, d + kv:], q=p["qkv"][:, :d], q_out=p["q"], rope=self.rope, status=status, stream=stream)
            c.attention(seqs, p["q"], p["o"], b["ws"], status=status, stream=stream)
            uad.linear_w4(p["o"], wo[0], wo[1], p["y"], zero=wo[2], stream=stream)
            b["h"].add_(p["y"])

    def held(self, l, b, n):
        at = torch.arange(n, device="cuda")
        pg, sl = self.table[b][at // self.page].long(), at % self.page
        return [x[pg, sl].double().cpu().numpy() for x in (self.caches[l].k, self.caches[l].v)]

    def verify(self, bufs, lens, start):
        d, kv, group = self.hq * self.dh, self.hkv * self.dh, self.hq // self.hkv
        scale = self.dh ** -0.5
        for l, ((wi, wo), p) in enumerate(zip(self.weights, bufs["per"])):
            for x, w, y in ((p["x"], wi, p["qkv"]), (p["o"], wo, p["y"])):
                want, size = reference(x, *w, None)
                check(y, want, size, x.shape[1], 64, None)
            qkv, q, o = (p[n].double().cpu().numpy() for n in ("qkv", "q", "o"))
            for b in range(self.n):
                keys, values = self.held(l, b, lens[b])
                for t in range(int(start[b]), int(start[b + 1])):
                    pos = lens[b] - (int(start[b + 1]) - t)
                    for got, raw in ((q[t].reshape(self.hq, self.dh), qkv[t, :d]), (keys[pos], qkv[t, d:d + kv])):
                        raw = raw.reshape(-1, self.dh)
                        want = paged.rotate(raw, pos, THETA, self.dh)
                        half = np.abs(raw[:, :self.dh // 2]) + np.abs(raw[:, self.dh // 2:])
                        slack = np.concatenate([half, half], axis=1) * 2.0 ** -22
                        assert np.all(np.abs(got - want) <= slack + HALF[torch.bfloat16] * (np.abs(want) + slack))
                    v = qkv[t, d + kv:].reshape(self.hkv, self.dh)
                    assert np.all(np.abs(values[pos] - v) <= HALF[torch.bfloat16] * np.abs(v))
                    seen = np.arange(lens[b]) <= pos
                    for g in range(self.hkv):
                        qg = q[t].reshape(self.hkv, group, self.dh)[g]
                        want, _ = paged.attend(qg, keys[:, g], values[:, g], seen, scale)
                        size, _ = paged.attend(qg, keys[:, g], np.abs(values[:, g]), seen, scale)
                        off = self.dh * 2.0 ** -23 * scale * (np.abs(qg) @ np.abs(keys[:pos + 1, g]).T).max(axis=1, keepdims=True)
                        rel = 2 * off + 2.0 ** -19 + 2.0 ** -16 + (pos + 3) * 2.0 ** -23
                        got = o[t].reshape(self.hkv, group, self.dh)[g]
                        assert np.all(np.abs(got - want) <= rel * size + HALF[torch.bfloat16] * (np.abs(want) + rel * size) + 1e-30)

    def exact(self, hs):
        """The decoder in 64 bits over a sequence's embeddings, without roundings."""
        h = hs.astype(np.float64)
        for wi, wo in self.weights:
            w = [paged.dequantize(x[0].cpu().numpy(), x[1].float().cpu().numpy(), x[2].cpu().numpy()) for x in (wi, wo)]
            q, k, v = np.split(h @ w[0].T, [self.hq * self.dh, (self.hq + self.hkv) * self.dh], axis=1)
            q, k, v = (x.reshape(len(h), -1, self.dh) for x in (q, k, v))
            for x in (q, k):
                for pos in range(len(h)):
                    x[pos] = paged.rotate(x[pos], pos, THETA, self.dh)
            o = np.zeros((len(h), self.hq, self.dh))
            for pos in range(len(h)):
                for i in range(self.hq):
                    g = i // (self.hq // self.hkv)
                    o[pos, i] = paged.attend(q[pos, i:i + 1], k[:, g], v[:, g], np.arange(len(h)) <= pos, self.dh ** -0.5)[0][0]
            h = h + o.reshape(len(h), -1) @ w[1].T
        return h


@pytest.mark.parametrize("name", ["pi0_small", "concat_small"])
def test_a_decoder_beside_the_expert(name):
    a = ARCHS[name]
    decode, P = 6, a.prefix_len
    lens = [P - 4, 1, 61, P]                        # the first grows past the prefix while it answers
    dec = Decoder(a, lens, decode, seed=5)
    rng = np.random.default_rng(6)
    emb = [rng.normal(size=(n + decode, a.width)).astype(np.float32) for n in lens]
    outs = [[] for _ in lens]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    done = [0] * len(lens)
    # prompts, in calls of up to 64 rows of any of the sequences, three rows of nobody behind them
    while done != lens:
        new, left = [0] * len(lens), 58
        for b in range(len(lens)):
            new[b] = min(lens[b] - done[b], 23 if b == 0 else left, left)
            left -= new[b]
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        done = [x + y for x, y in zip(done, new)]
        seqs = uad.Sequences(dec.table, torch.tensor(done, dtype=torch.int32, device="cuda"), torch.from_numpy(start).cuda(), max_new=max(new), max_len=max(done))
        rows = int(start[-1]) + 3
        bufs = dec.buffers(rows, seqs)
        for p in bufs["per"]:   # rows of nobody are not written by the append and the attention: what the projection then reads
            p["o"].zero_()
        bufs["h"].zero_()
        for b in range(len(lens)):
            bufs["h"][start[b]:start[b + 1]] = torch.from_numpy(emb[b][done[b] - new[b]:done[b]]).cuda()
        dec.step(bufs, seqs, status)
        torch.cuda.synchronize()
        dec.verify(bufs, done, start)
        assert bool((bufs["per"][0]["q"][-3:] == 7.5).all())
        for b in range(len(lens)):
            outs[b] += list(bufs["h"][start[b]:start[b + 1]].cpu().numpy())
    # token by token: one graph, whose lengths and inputs change in place
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    seqs = uad.Sequences(dec.table, length, max_len=max(lens) + decode)
    bufs = dec.buffers(len(lens), seqs)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        length.add_(1)
        dec.step(bufs, seqs, status, stream)
    for i in range(decode):
        bufs["h"].copy_(torch.from_numpy(np.stack([e[n + i] for e, n in zip(emb, lens)])).cuda())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        now = [n + i + 1 for n in lens]
        dec.verify(bufs, now, np.arange(len(lens) + 1))
        for b in range(len(lens)):
            outs[b].append(bufs["h"][b].cpu().numpy())
    assert int(status) == 0
    for b in (0, 2):
        want = dec.exact(emb[b])
        added = np.linalg.norm(want - emb[b], axis=1)
        assert np.all(np.linalg.norm(np.stack(outs[b]) - want, axis=1) <= 2 * 5 * a.n_layers * 2.0 ** -8 * added.max())
    # the expert reads what the decoder has written
    ex = uad.Expert(a, make_weights(a, seed=8), max_batch=1)
    try:
        for b in (0, 3):
            ks, vs = zip(*(dec.held(l, b, P) for l in range(a.n_layers)))
            ex.set_prefix(0, *(torch.from_numpy(np.stack(x)).to(torch.bfloat16) for x in (ks, vs)), dtype="bf16")
            want = chunk(ex, a)
            ex.set_prefix_paged(0, dec.caches, dec.table[b])
            got = chunk(ex, a)
            assert same(a, got, want) and np.isfinite(got[0]).all()
    finally:
        ex.close()
