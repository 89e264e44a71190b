"""The operators of the 8-bit cache as a program uses them together: a small decoder whose prompts and tokens go through the pages'
bookkeeping, the 4-bit projection, the append and the attention, eagerly and from a graph that is replayed with other lengths; drafts that
are taken back; windows with sinks; the expert's prefix from 8-bit pages; streams.

Tolerances are each operator's own, as derived beside its own tests (test_gpu_linear_w4, test_gpu_cache8), each checked on what
the GPU gave it.
"""
import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged, paged8
from test_gpu_cache8 import CODES, Case8, check_attention, half_step
from test_gpu_linear_w4 import check, reference
from test_gpu_paged_prefix import chunk, same
from uad_inputs import ARCHS, make_weights

pytestmark = pytest.mark.gpu
THETA = 10000.0


class Held:
    """What Case8's attention check asks of a batch, taken from the GPU's pools."""

    def __init__(self, heads, page, block, cache, table, lens, start):
        self.hq, self.hkv, self.dh = heads
        self.page, self.block, self.n = page, block, len(lens)
        self.lens, self.start = [int(x) for x in lens], np.asarray(start)
        self.table = table
        self.codes = [x.contiguous().view(torch.uint8).cpu().numpy() for x in (cache.k, cache.v)]
        self.scales = [x.cpu().numpy() for x in (cache.k_scale, cache.v_scale)]

    held = Case8.held


def empty_cache(n_pages, page, heads, block):
    _, hkv, dh = heads
    k, v = (torch.full((n_pages, page, hkv, dh), 0x7f, dtype=torch.uint8, device="cuda").view(CODES) for _ in range(2))
    scales = [torch.full((n_pages, -(-page // block), hkv), float("nan"), device="cuda") for _ in range(2)]
    return uad.PagedCache(k, v, *scales, block=block)


@pytest.mark.parametrize("heads,page,block,window,sinks", [((8, 1, 128), 16, 16, 0, 0), ((8, 2, 64), 12, 16, 40, 4), ((4, 1, 256), 64, 32, 0, 0)], ids=str)
def test_prompts_then_tokens_from_a_graph(heads, page, block, window, sinks):
    """Prompts of four sequences in two calls, then a captured step (lengths + 1, pages, projection, append, attention) replayed, then a draft
    that is taken back and another one: the cache holds what the last accepted tokens were."""
    hq, hkv, dh = heads
    n, width, layers, model = 4, 24, 2, 256
    rng = np.random.default_rng(dh)
    cols = (hq + 2 * hkv) * dh
    w = [uad.quantize_w4((rng.normal(size=(model, cols)) * 0.05).astype(np.float32), 64) for _ in range(layers)]
    q4 = [[torch.from_numpy(w[l][0]).cuda(), torch.from_numpy(w[l][1].view(np.int16)).cuda().view(torch.bfloat16), torch.from_numpy(w[l][2]).cuda()] for l in range(layers)]
    n_pages = 70
    caches = [empty_cache(n_pages, page, heads, block) for _ in range(layers)]
    pool = uad.PagePool(torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda(),
                        torch.tensor([0, n_pages], dtype=torch.int32, device="cuda"), page)
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    lens, want = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    rope = uad.rope(THETA, dh)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    st = torch.cuda.Stream()

    class Step:
        def __init__(self, rows, max_new):
            self.rows = rows
            self.start = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
            self.slot = torch.zeros(rows, dtype=torch.int64, device="cuda")
            self.x = torch.zeros(rows, model, device="cuda", dtype=torch.bfloat16)
            self.qkv = [torch.zeros(rows, cols, device="cuda") for _ in range(layers)]
            self.q = [torch.zeros(rows, hq * dh, device="cuda", dtype=torch.bfloat16) for _ in range(layers)]
            self.out = [torch.zeros(rows, hq * dh, device="cuda", dtype=torch.bfloat16) for _ in range(layers)]
            self.lse = [torch.zeros(rows, hq, device="cuda") for _ in range(layers)]
            self.seqs = uad.Sequences(table, lens, self.start, max_len=200, max_new=max_new)
            self.ws = torch.empty(max(c.attention_workspace(self.seqs, rows, hq) for c in caches), dtype=torch.uint8, device="cuda")

        def run(self, stream):
            pool.resize(table, lens, want, self.start, slot=self.slot, status=status, stream=stream)
            for l, c in enumerate(caches):
                for i in range(0, self.rows, uad.UAD_W4_MAX_ROWS):
                    uad.linear_w4(self.x[i:i + uad.UAD_W4_MAX_ROWS], *q4[l][:2], self.qkv[l][i:i + uad.UAD_W4_MAX_ROWS], zero=q4[l][2], stream=stream)
                q, k, v = self.qkv[l].split([hq * dh, hkv * dh, hkv * dh], dim=1)
                c.append(self.seqs, k, v, q=q, q_out=self.q[l], rope=rope, status=status, stream=stream)
                c.attention(self.seqs, self.q[l], self.out[l], self.ws, window=window, sinks=sinks, lse=self.lse[l], status=status, stream=stream)

        def check(self, before):
            """Against the oracles, from the pools as they were before (a list of codes and scales a layer)."""
            torch.cuda.synchronize()
            assert int(status) == 0
            start, tab, ln = self.start.cpu().numpy(), table.cpu().numpy(), lens.cpu().numpy()
            used = int(start[-1])
            where = paged.rows_of(ln, start)
            assert self.slot.tolist() == [int(tab[b, p // page]) * page + p % page for b, p in where] + [-1] * (self.rows - used)
            for l, c in enumerate(caches):
                check(self.qkv[l][:used], *reference(self.x[:used], *q4[l], None), model, 64, None)
                kv = self.qkv[l][:used].double().cpu().numpy()[:, hq * dh:].reshape(used, 2, hkv, dh)
                now = Held(heads, page, block, c, tab, ln, start)
                for which in range(2):
                    want_codes, want_scales = before[l][0][which].copy(), before[l][1][which].astype(np.float64)
                    exact, s = paged8.append(want_codes, want_scales, tab, ln, start, page, block, kv[:, which], None if which else THETA, dh)
                    assert np.array_equal(now.scales[which].astype(np.float64), want_scales, equal_nan=True)
                    fresh = np.zeros(want_codes.shape[:2], bool)
                    for t, (b, p) in enumerate(where):
                        pg, sl = tab[b, p // page], p % page
                        fresh[pg, sl] = True
                        got = paged8.VALUES[now.codes[which][pg, sl]] * s[t][:, None]
                        off = 0 if which else 2 * np.abs(kv[t, which]).max() * 2.0 ** -22
                        assert np.all(np.abs(got - exact[t]) <= half_step(np.abs(exact[t]) + off, s[t][:, None]) + off)
                    assert np.array_equal(now.codes[which][~fresh], want_codes[~fresh])
                check_attention(now, self.q[l], self.out[l], self.lse[l], True, window, sinks)

    def pools():
        torch.cuda.synchronize()
        return [([x.contiguous().view(torch.uint8).cpu().numpy() for x in (c.k, c.v)], [x.cpu().numpy() for x in (c.k_scale, c.v_scale)]) for c in caches]

    def put(step, lengths):
        want.copy_(torch.tensor(lengths, dtype=torch.int32))
        step.x.copy_(torch.from_numpy(rng.normal(size=tuple(step.x.shape))))
        return pools()

    prompt, one = Step(130, 100), Step(n + 2, 5)
    for lengths in ([30, 5, 0, 77], [55, 5, 90, 80]):   # in two calls, the second joins blocks
        before = put(prompt, lengths)
        prompt.run(st)
        prompt.check(before)
    put(one, lens.tolist())
    one.run(st)   # nothing new: loads what a capture must not
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        one.run(st)
    now = lens.tolist()
    for turn in range(5):
        now = [x + (1 if turn != 2 or b % 2 else 0) for b, x in enumerate(now)]
        before = put(one, now)
        graph.replay()
        one.check(before)
    draft = Step(20, 6)
    for lengths in ([x + 5 for x in now], [x + 1 for x in now], [x + 3 for x in now]):   # a draft, four fifths of it taken back, another one
        before = put(draft, lengths)
        draft.run(st)
        draft.check(before)
    want.zero_()   # the episodes' ends: every page is free again
    torch.cuda.synchronize()
    pool.resize(table, lens, want, one.start, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and pool.state.tolist()[1] == n_pages and sorted(pool.ring.tolist()) == list(range(n_pages))


def test_calls_on_two_streams_at_once():
    """Two caches, two streams, workspaces of their own: the same bits as one after the other."""
    cases = [Case8((8, 1, 128), 16, [900, 40, 333], [2, 1, 3], seed=s) for s in (1, 2)]
    caches, seqs = [c.on_gpu() for c in cases], [c.sequences() for c in cases]
    q = [torch.randn(c.rows, 1024, device="cuda").bfloat16() for c in cases]
    rows = [torch.randn(c.rows, 256, device="cuda") for c in cases]
    ws = [torch.empty(k.attention_workspace(s, c.rows, 8), dtype=torch.uint8, device="cuda") for c, k, s in zip(cases, caches, seqs)]
    streams = [torch.cuda.Stream() for _ in cases]

    def run(at_once):
        outs = [torch.zeros_like(x) for x in q]
        torch.cuda.synchronize()
        for _ in range(5):
            for i, st in enumerate(streams):
                caches[i].append(seqs[i], rows[i][:, :128], rows[i][:, 128:], stream=st)
                caches[i].attention(seqs[i], q[i], outs[i], ws[i], stream=st)
                if not at_once:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return outs

    a, b = run(False), run(True)
    used = int(cases[0].start[-1])
    assert all(torch.equal(x[:used], y[:used]) for x, y in zip(a, b))


@pytest.mark.parametrize("name", ["tiny", "tiny_f32_rope", "pi0_small", "concat_small"])
@pytest.mark.parametrize("page,block", [(16, 16), (5, 32), (100, 64)])
def test_prefix_from_8_bit_pages(name, page, block):
    """The bits of the same values given as a contiguous fp32 buffer."""
    a = ARCHS[name]
    c = [Case8((a.n_kv_heads, a.n_kv_heads, a.head_dim), page, [a.prefix_len], [1], block, ("pshd", "phsd", "joint")[page % 3], seed=l) for l in range(a.n_layers)]
    for x in c[1:]:   # one table for all layers
        for which in range(2):
            fresh = np.full_like(x.codes[which], 0x7f)
            scales = np.full_like(x.scales[which], np.nan)
            fresh[c[0].table[0]], scales[c[0].table[0]] = x.codes[which][x.table[0]], x.scales[which][x.table[0]]
            x.codes[which], x.scales[which] = fresh, scales
        x.table = c[0].table
    caches = [x.on_gpu() for x in c]
    kv = [torch.from_numpy(np.stack([x.held(0, which) for x in c]).astype(np.float32)).cuda() for which in range(2)]
    ex = uad.Expert(a, make_weights(a, seed=4), max_batch=2)
    try:
        ex.set_prefix(0, *kv)
        want = chunk(ex, a)
        ex.set_prefix(0, kv[1], kv[0])
        ex.set_prefix_paged(0, caches, c[0].table[0].tolist())
        assert same(a, chunk(ex, a), want)
        mixed = [caches[0], uad.PagedCache(*(torch.zeros(c[0].pages, page, a.n_kv_heads, a.head_dim, device="cuda") for _ in range(2)))]
        with pytest.raises(ValueError, match="8-bit"):
            ex.set_prefix_paged(0, mixed, c[0].table[0].tolist())
        with pytest.raises(uad.UADError):
            ex.set_prefix_paged(0, caches, [-1] + c[0].table[0].tolist()[1:])
        with pytest.raises(uad.UADError):
            ex.set_prefix_paged(0, caches[:1] if a.n_layers > 1 else caches * 2, c[0].table[0].tolist())
        assert same(a, chunk(ex, a), want)   # a refused call leaves the prefix as it was
    finally:
        ex.close()
