"""The pages' bookkeeping on the GPU against lists (whole numbers, compared exactly)."""
import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged8

pytestmark = pytest.mark.gpu


class Pool:
    """Sequences that hold pages, and a ring with the others from `first` on."""

    def __init__(self, lens, width, page, spare, first=0, seed=0):
        rng = np.random.default_rng(seed)
        self.page, self.lens = page, np.array(lens, np.int32)
        held = [(n + page - 1) // page for n in lens]
        self.n = sum(held) + spare
        ids = rng.permutation(self.n).astype(np.int32)
        self.table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for b, h in enumerate(held):
            self.table[b, :h] = ids[at:at + h]
            at += h
        self.ring = np.full(self.n, -1, np.int32)
        self.ring[(first + np.arange(spare)) % self.n] = ids[at:]
        self.state = np.array([first, spare], np.int32)


def run(p, want, rows, in_place=False, maps=(True, True, True), n_rows=None, stream=None):
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    n = len(p.lens)
    ring, state, table, lens = up(p.ring), up(p.state), up(p.table), up(p.lens)
    want_t = up(np.array(want, np.int32))
    start = torch.full((n + 1,), -9, dtype=torch.int32, device="cuda")
    out = None if in_place else torch.full((n,), -9, dtype=torch.int32, device="cuda")
    state_out = None if in_place else torch.full((2,), -9, dtype=torch.int32, device="cuda")
    m = [torch.full((rows,), -9, dtype=t, device="cuda") if on else None for t, on in zip((torch.int64, torch.int32, torch.int32), maps)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    uad.PagePool(ring, state, p.page).resize(table, lens, want_t, start, length_out=out, state_out=state_out, slot=m[0], row_seq=m[1],
                                             row_pos=m[2], rows=n_rows, status=status, stream=stream)
    torch.cuda.synchronize()
    if not in_place:
        assert np.array_equal(lens.cpu().numpy(), p.lens) and np.array_equal(state.cpu().numpy(), p.state)
    down = lambda x: None if x is None else x.cpu().numpy()  # noqa: E731
    return dict(ring=down(ring), state=down(state if in_place else state_out), table=down(table), lens=down(lens if in_place else out),
                start=down(start), slot=down(m[0]), seq=down(m[1]), pos=down(m[2]), status=int(status))


def check(p, want, rows, got, limit=None):
    ring, state, table, lens, start, made, found = paged8.resize(p.ring, p.state, p.table, p.lens, want, p.page, rows if limit is None else limit)
    assert np.array_equal(got["table"], table)
    assert np.array_equal(got["ring"], ring)
    assert tuple(got["state"]) == state
    assert np.array_equal(got["lens"], lens)
    assert np.array_equal(got["start"], start)
    for name, i in (("slot", 0), ("seq", 1), ("pos", 2)):
        if got[name] is not None:
            assert np.array_equal(got[name], [m[i] for m in made] + [-1] * (rows - len(made))), name
    bits = (uad.UAD_KV_NO_ROOM if "no room" in found else 0) | (uad.UAD_KV_BAD_SEQ if "bad sequence" in found else 0)
    assert got["status"] == bits


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seqs,new,at,page", [(1, 1, 0, 16), (1, 5000, 3, 16), (64, 5, 1129, 16), (33, 40, 90, 1), (200, 100, 50, 100), (2047, 3, 9, 5),
                                              (2048, 2, 40, 16), (2049, 9, 40, 12), (5000, 60, 60, 16), (7, 3, 0, 65536)])
def test_growth_and_return(seqs, new, at, page, in_place):
    """One and many sequences, on the borders of the chunks that the kernel takes them in; some give pages back, some stay."""
    rng = np.random.default_rng(seqs)
    lens = rng.integers(0, at + 1, seqs)
    step = rng.integers(0, new + 1, seqs)
    want = np.where(rng.random(seqs) < 0.3, np.maximum(lens - step, 0), lens + step)
    width = (at + new + page - 1) // page
    spare = int(((want + page - 1) // page).sum()) + 3
    p = Pool(lens.tolist(), width, page, spare, first=spare // 2, seed=seqs)
    rows = int(np.maximum(want - lens, 0).sum()) + 5
    check(p, want, rows, run(p, want, rows, in_place))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("spare,rows", [(0, 10000), (1, 10000), (40, 10000), (10000, 0), (10000, 1), (10000, 300), (60, 400)])
def test_sequences_that_find_no_room(spare, rows, in_place):
    """Pages and rows that run out before, between and behind the sequences; those that need none are served all the same."""
    rng = np.random.default_rng(spare + rows)
    lens = rng.integers(0, 60, 90)
    want = lens + rng.integers(-20, 30, 90)
    want = np.maximum(want, 0)
    p = Pool(lens.tolist(), 8, 12, spare, first=min(3, spare), seed=1)
    check(p, want, rows, run(p, want, rows, in_place))


def test_the_ring_wraps_around():
    for first in range(0, 30, 7):
        p = Pool([10, 0, 33, 5], 10, 4, 12, first=0, seed=first)
        p.ring = np.roll(p.ring, first % p.n)
        p.state = np.array([first % p.n, 12], np.int32)
        check(p, [2, 20, 0, 25], 60, run(p, [2, 20, 0, 25], 60))


def test_an_empty_batch_and_an_empty_ring():
    p = Pool([], 4, 16, 5)
    p.table = np.zeros((0, 4), np.int32)
    check(p, [], 7, run(p, [], 7))
    p = Pool([16, 3], 1, 16, 0)
    check(p, [16, 16], 20, run(p, [16, 16], 20))


@pytest.mark.parametrize("maps", [(False, False, False), (True, False, False), (False, True, True)])
def test_maps_that_are_not_wanted(maps):
    """Without maps rows have no limit but the one that is asked for."""
    p = Pool([5, 0, 90], 20, 8, 40, seed=2)
    want = [9, 30, 150]
    check(p, want, 120, run(p, want, 120, maps=maps))
    if not any(maps):
        check(p, want, 0, run(p, want, 0, maps=maps, n_rows=50), limit=50)


def test_sequences_out_of_range_stay_as_they_are():
    p = Pool([5, 6, 7, 8, 9], 2, 8, 9, seed=3)
    p.lens[1], p.lens[3] = -1, 17
    check(p, [9, 9, 17, 10, 10], 30, run(p, [9, 9, 17, 10, 10], 30))
    p.lens[1], p.lens[3] = 2 ** 31 - 1, -2 ** 31
    want = [-3, 2 ** 31 - 1, 7, -2 ** 31, 16]
    check(p, want, 30, run(p, want, 30))


def test_a_pool_out_of_range_is_left_alone():
    for state in ([-1, 3], [4, 9], [20, 3], [0, -2], [0, 21]):
        p = Pool([5, 20, 3], 6, 8, 14, seed=4)
        p.state = np.array(state, np.int32)
        sound = 0 <= state[0] < p.n and 0 <= state[1] <= p.n
        got = run(p, [6, 8, 30], 60)
        if sound:
            assert got["status"] & uad.UAD_KV_BAD_POOL == 0
            continue
        assert got["status"] & uad.UAD_KV_BAD_POOL
        assert np.array_equal(got["ring"], p.ring) and np.array_equal(got["table"], p.table) and got["state"].tolist() == state
        assert got["lens"].tolist() == [6, 8, 3]   # what needs no page is served; pages given back are dropped
    # more pages given back than the ring has places
    p = Pool([40, 40], 5, 8, 3, seed=5)
    p.state[1] = p.n - 2
    got = run(p, [0, 0], 1)
    assert got["status"] == uad.UAD_KV_BAD_POOL and got["state"].tolist() == [0, p.n]


def test_wide_tables_and_views():
    """Rows of the table apart from each other; more pages than 2^16 in one sequence."""
    p = Pool([100000, 3], 100000, 2, 60000, seed=6)
    want = [160001, 0]
    check(p, want, 60010, run(p, want, 60010))
    whole = torch.full((2, 12), -1, dtype=torch.int32, device="cuda")
    ring, state = torch.arange(9, dtype=torch.int32, device="cuda"), torch.tensor([0, 9], dtype=torch.int32, device="cuda")
    lens, want, start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 0], [5, 9], [0, 0, 0]))
    uad.PagePool(ring, state, 4).resize(whole[:, 2:6], lens, want, start)
    assert whole.tolist() == [[-1, -1, 0, 1] + [-1] * 8, [-1, -1, 2, 3, 4] + [-1] * 7] and state.tolist() == [5, 4] and lens.tolist() == [5, 9]


def test_the_most_sequences():
    p = Pool([3] * 65535, 2, 4, 70000, seed=7)
    want = np.full(65535, 4)
    want[::2] = 5
    want[7] = 0
    rows = int(np.maximum(want - 3, 0).sum())
    check(p, want, rows, run(p, want, rows, True))


def test_a_captured_loop_of_steps():
    """resize in place in a graph: every replay gives each sequence one more token; in the end some find no page and one is at its table's end."""
    p = Pool([14, 0, 31, 7], 6, 8, 6, seed=8)
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    ring, state, table, lens = up(p.ring), up(p.state), up(p.table), up(p.lens)
    want, start = torch.zeros_like(lens), torch.zeros(5, dtype=torch.int32, device="cuda")
    slot, status = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    pool = uad.PagePool(ring, state, 8)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        torch.add(lens, 1, out=want)
        pool.resize(table, lens, want, start, slot=slot, status=status, stream=st)
    bits = 0
    for _ in range(30):
        made = paged8.resize(p.ring, p.state, p.table, p.lens, p.lens + 1, 8, 4)
        p.ring, p.state, p.table, p.lens = made[0], made[1], made[2], made[3]
        bits |= uad.UAD_KV_NO_ROOM if "no room" in made[6] else 0
        bits |= uad.UAD_KV_BAD_SEQ if "bad sequence" in made[6] else 0
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(table.cpu().numpy(), p.table) and np.array_equal(lens.cpu().numpy(), p.lens) and state.tolist() == list(p.state)
        assert start.tolist() == made[4] and slot.tolist() == [m[0] for m in made[5]] + [-1] * (4 - len(made[5]))
    assert int(status) == bits == uad.UAD_KV_NO_ROOM | uad.UAD_KV_BAD_SEQ


def test_the_binding_refuses_tensors_that_do_not_fit():
    ring, state = torch.arange(9, dtype=torch.int32, device="cuda"), torch.tensor([0, 9], dtype=torch.int32, device="cuda")
    pool = uad.PagePool(ring, state, 4)
    fine = dict(table=torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), length=torch.zeros(2, dtype=torch.int32, device="cuda"),
                want=torch.ones(2, dtype=torch.int32, device="cuda"), start=torch.zeros(3, dtype=torch.int32, device="cuda"))
    slot = torch.zeros(4, dtype=torch.int64, device="cuda")
    for kw in (dict(table=fine["table"].long()), dict(table=fine["table"][:1]), dict(table=fine["table"].t()), dict(length=fine["length"].cpu()),
               dict(want=fine["want"][:1]), dict(start=fine["start"][:2]), dict(want=torch.ones(4, dtype=torch.int32, device="cuda")[::2]),
               dict(length_out=fine["start"]), dict(state_out=fine["start"]), dict(slot=slot.int()), dict(slot=slot, row_seq=fine["start"]),
               dict(slot=slot, rows=5), dict(slot=slot, row_pos=slot), dict(status=fine["want"]), dict(status=slot[:1])):
        with pytest.raises(ValueError):
            pool.resize(**(fine | kw))
    with pytest.raises(uad.UADError):
        pool.resize(**(fine | dict(table=torch.zeros((2, 0), dtype=torch.int32, device="cuda"))))
    torch.cuda.synchronize()
    assert state.tolist() == [0, 9] and fine["length"].tolist() == [0, 0]
    with pytest.raises(uad.UADError):
        uad.PagePool(ring, state, 0).resize(**fine)


@pytest.mark.parametrize("behind", [1, 2, 3])
def test_a_map_as_long_as_31_bits_hold_ends_where_it_ends(behind):
    """2^31 - behind rows end inside four of a store, whose end is past 31 bits."""
    rows = 2 ** 31 - behind
    buf = torch.full((2 ** 31 + 64,), 7, dtype=torch.int32, device="cuda")
    whole = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, start, status = whole(2), whole(-9, -9), whole(0)
    uad.PagePool(torch.arange(4, dtype=torch.int32, device="cuda"), whole(0, 4), 16).resize(
        whole(3, 2).view(1, 2), lens, whole(7), start, row_pos=buf[:rows], status=status)
    torch.cuda.synchronize()
    assert lens.tolist() == [7] and start.tolist() == [0, 5] and int(status) == 0
    assert buf[:8].tolist() == [2, 3, 4, 5, 6, -1, -1, -1]
    assert buf[rows - 64:rows].tolist() == [-1] * 64
    assert buf[rows:].tolist() == [7] * (2 ** 31 + 64 - rows)


def test_arrays_off_their_elements_are_refused():
    buf = {n: torch.zeros(64, dtype=torch.int64, device="cuda") for n in ("ring", "state", "state_out", "table", "len", "want", "len_out", "start", "slot",
                                                                          "row_seq", "row_pos", "status")}
    at = {n: t.data_ptr() for n, t in buf.items()}

    def call(x):
        return uad.uad_kv_resize(uad.uad_page_pool(ring=x["ring"], state=x["state"], state_out=x["state_out"], n_pages=4, page_size=16),
                                 uad.uad_kv_wanted(**{n: x[n] for n in ("table", "len", "want", "len_out", "start", "slot", "row_seq", "row_pos")}, table_stride=4,
                                                   n_seqs=1, table_width=4, n_rows=4), x["status"], None)

    for n in at:
        assert call(at | {n: at[n] + (4 if n == "slot" else 2)}) == uad.UAD_EINVAL, n
    assert call(at) == uad.UAD_OK
    torch.cuda.synchronize()
    assert buf["start"].view(torch.int32)[:2].tolist() == [0, 0] and int(buf["status"][0]) == 0
