"""The pages' bookkeeping where tables have places without a page: episodes seen through a window, whose hidden pages the program has given back itself
(-1), entries that are no pages, rings that hold some."""
import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged8
from test_gpu_resize import Pool, run

pytestmark = pytest.mark.gpu


def check_ring(p, want, rows, got):
    """As test_gpu_resize.check, but of the ring what it holds: no matter what lies at its free places."""
    ring, state, table, lens, start, made, found = paged8.resize(p.ring, p.state, p.table, p.lens, want, p.page, rows)
    assert tuple(got["state"]) == state
    at = (state[0] + np.arange(state[1])) % p.n
    assert np.array_equal(got["ring"][at], ring[at])
    assert np.array_equal(got["table"], table) and np.array_equal(got["lens"], lens) and np.array_equal(got["start"], start)
    for name, i in (("slot", 0), ("seq", 1), ("pos", 2)):
        assert np.array_equal(got[name], [m[i] for m in made] + [-1] * (rows - len(made))), name
    names = {"no room": uad.UAD_KV_NO_ROOM, "bad sequence": uad.UAD_KV_BAD_SEQ, "bad page": uad.UAD_KV_BAD_PAGE, "bad pool": uad.UAD_KV_BAD_POOL}
    assert got["status"] == sum(names[f] for f in found)


def hide(p, share, rng, sinks=1, near=2, what=(-1,)):
    """Pages between the first and the last ones of a share of the sequences go back to the ring, by the program itself."""
    first, count = (int(x) for x in p.state)
    for b in range(len(p.lens)):
        held = -(-int(p.lens[b]) // p.page)
        if rng.random() >= share:
            continue
        for i in range(sinks, held - near):
            p.ring[(first + count) % p.n] = p.table[b, i]
            p.table[b, i] = rng.choice(what)
            count += 1
    p.state[1] = count


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows", [40, 9000])
@pytest.mark.parametrize("seqs,at,page", [(1, 900, 16), (6, 300, 5), (64, 2000, 16), (300, 90, 1), (2048, 40, 4), (2049, 60, 4), (4500, 60, 4)])
def test_ends_of_windowed_episodes(seqs, at, page, rows, in_place):
    """Some end, some are cut back into what the window has left or hidden, some grow; one block and several, chunks with and without holes."""
    rng = np.random.default_rng(seqs + rows)
    lens = rng.integers(at // 2, at + 1, seqs)
    p = Pool(lens.tolist(), -(-(at + 9) // page), page, 50, first=20, seed=seqs)
    hide(p, 0.6, rng)
    kind = rng.integers(0, 4, seqs)
    if seqs == 1:
        kind[0] = 0
    want = np.choose(kind, [np.zeros(seqs, np.int64), lens // 2, np.maximum(lens - page, 0), lens + rng.integers(0, 9, seqs)])
    check_ring(p, want, rows, run(p, want, rows, in_place))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows", [10, 9000])
def test_more_places_without_a_page_than_the_ring_has(rows, in_place):
    """A long episode behind a window: a table of 5000 pages of which 40 are there, and a pool of 60."""
    rng = np.random.default_rng(3)
    p = Pool([16 * 40, 33], 5000, 16, 17, first=55, seed=3)
    held = p.table[0, :40].copy()
    p.table[0, :5000] = -1
    at = np.sort(rng.choice(5000, 40, replace=False))
    p.table[0, at] = held
    p.lens[0] = 80000
    check_ring(p, [0, 0], rows, run(p, [0, 0], rows, in_place))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows,seqs", [(10, 40), (9000, 40), (10, 2500)])
def test_entries_that_are_no_pages_are_told_and_left_out(rows, seqs, in_place):
    rng = np.random.default_rng(rows + seqs)
    lens = rng.integers(20, 60, seqs)
    p = Pool(lens.tolist(), 16, 4, 9, seed=4)
    hide(p, 0.3, rng, what=(-1, -7, p.n, 2 ** 31 - 1, -2 ** 31))
    want = np.where(rng.random(seqs) < 0.7, 0, lens)
    got = run(p, want, rows, in_place)
    assert got["status"] & uad.UAD_KV_BAD_PAGE
    check_ring(p, want, rows, got)


def test_more_pages_than_places_beside_places_without_a_page():
    """A ring whose count says more than there are: what does not fit is dropped, places without a page do not count for it."""
    for rows in (10, 9000):
        p = Pool([40, 40, 40], 5, 8, 3, seed=5)
        p.table[1, 1:4] = -1
        p.state[1] = p.n - 8
        got = run(p, [0, 0, 0], rows)
        assert got["status"] == uad.UAD_KV_BAD_POOL
        check_ring(p, [0, 0, 0], rows, got)


@pytest.mark.parametrize("rows", [40, 9000])
def test_a_ring_that_holds_no_pages_is_told(rows):
    """What is taken from it is written into the table as it is, and told, with slot maps and without."""
    for maps in ((True, True, True), (False, False, False)):
        p = Pool([5, 0], 4, 8, 6, seed=6)
        p.ring[1], p.ring[2] = -1, p.n
        got = run(p, [8, 30], rows, maps=maps, n_rows=rows)
        assert got["status"] == uad.UAD_KV_BAD_PAGE and got["table"][1].tolist() == p.ring[:4].tolist()


def test_a_windowed_episode_from_its_begin_to_its_end():
    """Tokens appended and seen through a window with sinks; the program gives the hidden pages back; the episode ends; another one takes the pages and
    its tokens arrive in them."""
    heads, page, window, sinks = (4, 1, 64), 16, 40, 4
    hq, hkv, dh = heads
    n_pages, width = 12, 40
    k, v = (torch.zeros(n_pages, page, hkv, dh, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.ones(n_pages, 1, hkv, device="cuda") for _ in range(2))
    cache = uad.PagedCache(k, v, ks, vs)
    whole = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ring, state = torch.arange(n_pages, dtype=torch.int32, device="cuda"), whole(0, n_pages)
    pool = uad.PagePool(ring, state, page)
    table = torch.full((2, width), -1, dtype=torch.int32, device="cuda")
    lens, start, status = whole(0, 0), whole(0, 0, 0), whole(0)
    seqs = uad.Sequences(table, lens, start, max_len=width * page, max_new=30)

    def step(*want):
        before = int(lens.sum())
        pool.resize(table, lens, whole(*want), start, status=status)
        rows = max(1, int(lens.sum()) - before)
        x = torch.randn(rows, 6 * dh, device="cuda")
        q, out = torch.zeros(rows, hq * dh, device="cuda", dtype=torch.bfloat16), torch.zeros(rows, hq * dh, device="cuda", dtype=torch.bfloat16)
        cache.append(seqs, x[:, 4 * dh:5 * dh], x[:, 5 * dh:], q=x[:, :4 * dh], q_out=q, status=status)
        ws = torch.empty(cache.attention_workspace(seqs, rows, hq, window, sinks), dtype=torch.uint8, device="cuda")
        cache.attention(seqs, q, out, ws, window=window, sinks=sinks, status=status)
        torch.cuda.synchronize()
        assert int(status) == 0 and bool(out.isfinite().all()) and bool((out != 0).any())

    for end in range(25, 500, 25):   # 500 tokens of 32 pages: the pool has 12
        step(end, 0)
        hidden = (end - window) // page
        t, s = table[0].tolist(), state.tolist()
        for i in range(1, hidden):
            if t[i] >= 0:
                ring[(s[0] + s[1]) % n_pages] = t[i]
                s[1] += 1
                table[0, i] = -1
        state.copy_(whole(*s))
    pool.resize(table, lens, whole(0, 0), start, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and state.tolist()[1] == n_pages and sorted(ring.tolist()) == list(range(n_pages))
    step(0, 30)
    held = table[1].tolist()
    assert len(set(held[:2])) == 2 and min(held[:2]) >= 0


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows", [40, 9000])
def test_a_captured_call_meets_other_tables(rows, in_place):
    """One graph, replayed over tables with and without places that hold no page, and over a ring that they do not fit."""
    rng = np.random.default_rng(rows)
    seqs, width, page, n = 300, 20, 4, 6000
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    whole = lambda *s: torch.full(s, -9, dtype=torch.int32, device="cuda")  # noqa: E731
    ring, state, table, lens, want, start, status = whole(n), whole(2), whole(seqs, width), whole(seqs), whole(seqs), whole(seqs + 1), whole(1)
    slot, seq, pos = torch.zeros(rows, dtype=torch.int64, device="cuda"), whole(rows), whole(rows)
    out, state_out = (lens, state) if in_place else (whole(seqs), whole(2))
    pool, st = uad.PagePool(ring, state, page), torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        pool.resize(table, lens, want, start, length_out=None if in_place else out, state_out=None if in_place else state_out, slot=slot, row_seq=seq,
                    row_pos=pos, status=status, stream=st)
    for turn in range(6):
        now = rng.integers(20, 60, seqs)
        p = Pool(now.tolist(), width, page, 0, seed=turn)
        spare = n - p.n
        p.ring = np.concatenate([np.arange(p.n, n), np.full(p.n, -1)]).astype(np.int32)
        p.n, p.state = n, np.array([0, spare], np.int32)
        if turn % 2:
            hide(p, 0.5, rng)
        if turn == 4:
            p.state[1] = n - 500   # more than there are: not everything finds a place
        shall = np.where(rng.random(seqs) < 0.5, 0, now + rng.integers(0, 9, seqs))
        for t, x in ((ring, p.ring), (state, p.state), (table, p.table), (lens, p.lens), (want, shall.astype(np.int32)), (status, np.zeros(1, np.int32))):
            t.copy_(up(x))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check_ring(p, shall, rows, dict(ring=ring.cpu().numpy(), state=state_out.cpu().numpy(), table=table.cpu().numpy(), lens=out.cpu().numpy(), start=start.cpu().numpy(),
                                        slot=slot.cpu().numpy(), seq=seq.cpu().numpy(), pos=pos.cpu().numpy(), status=int(status)))
