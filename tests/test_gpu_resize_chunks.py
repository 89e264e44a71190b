"""The pages' bookkeeping over several chunks of sequences of which pages or rows run out, and over tables of so many tokens that sums need 64 bits."""
import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged8
from test_gpu_resize import Pool, check, run
from test_gpu_resize_windows import check_ring, hide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("what", ["pages", "rows", "both"])
@pytest.mark.parametrize("end", [0.0, 0.2, 0.55, 0.98])
@pytest.mark.parametrize("seqs,new", [(2049, 2), (4096, 9), (6000, 1), (6000, 9)])
def test_refusals_in_every_chunk(seqs, new, end, what, in_place):
    """Pages, rows or both run out in the first, a middle and the last chunk; behind that, those that need none of them are served."""
    rng = np.random.default_rng(seqs + new)
    page = 4
    lens = rng.integers(0, 30, seqs)
    want = np.where(rng.random(seqs) < 0.3, np.maximum(lens - rng.integers(0, 9, seqs), 0), lens + rng.integers(0, new + 1, seqs))
    at = int(end * seqs)
    pages = int(np.maximum(-(-want // page) - -(-lens // page), 0)[:at].sum())
    add = np.maximum(want - lens, 0)
    spare = pages if what != "rows" else 3 * seqs
    rows = int(add[:at].sum()) + 1 if what != "pages" else int(add.sum()) + 5
    p = Pool(lens.tolist(), -(-int(max(lens.max(), want.max())) // page), page, spare, first=spare // 3, seed=seqs)
    got = run(p, want, rows, in_place)
    assert got["status"] == uad.UAD_KV_NO_ROOM
    check(p, want, rows, got)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page,width,seqs,rows", [(65536, 17, 7, 3000), (4096, 300, 40, 9000), (16, 70000, 3, 5000), (1, 1 << 20, 2, 900), (65536, 17, 2500, 9000)])
def test_tables_of_a_million_tokens(page, width, seqs, rows, in_place):
    """Sums in 64 bits: growth from short and long, return, refusal, places without a page."""
    rng = np.random.default_rng(width)
    long = rng.random(seqs) < 0.5
    lens = np.where(long, page * width - rng.integers(0, 600, seqs), rng.integers(0, 50, seqs))
    if seqs > 100:
        lens = np.where(rng.random(seqs) < 0.02, lens, rng.integers(0, 50, seqs))
    kind = rng.integers(0, 4, seqs)
    want = np.choose(kind, [np.zeros(seqs, np.int64), np.maximum(lens - 2 * page, 0), lens, np.minimum(lens + rng.integers(0, 1000, seqs), page * width)])
    for spare in (0, 4000):
        p = Pool(lens.tolist(), width, page, spare, first=spare // 2, seed=seqs)
        check(p, want, rows, run(p, want, rows, in_place))
        if width < 1 << 20:
            hide(p, 0.4, rng)
            check_ring(p, want, rows, run(p, want, rows, in_place))


def served(p, want, limit):
    """paged8.resize without a list of the rows: (table, lens, start, taken, refused)."""
    count, n = int(p.state[1]), len(want)
    table, lens, start, taken, pages, rows, no = p.table.copy(), p.lens.astype(np.int64), np.zeros(n + 1, np.int64), 0, 0, 0, 0
    for b in range(n):
        held, needed, add = -(-int(lens[b]) // p.page), -(-int(want[b]) // p.page), int(want[b]) - int(lens[b])
        start[b + 1] = start[b]
        pages, rows = pages + needed - held, rows + add
        if (needed > held and pages > count) or rows > limit:
            no += 1
            continue
        table[b, held:needed] = p.ring[(int(p.state[0]) + taken + np.arange(needed - held)) % p.n]
        taken += needed - held
        lens[b] = want[b]
        start[b + 1] += add
    return table, lens, start, taken, no


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("share", [1.0, 0.3])
def test_more_rows_than_31_bits_hold_are_asked_for(share, in_place):
    """Sequences that ask for two million tokens each, 5 10^9 in all: as many as 31 bits hold get them, or as many as there are pages."""
    page, width, seqs = 65536, 40, 2300
    rng = np.random.default_rng(5)
    lens, want = rng.integers(0, 3, seqs), rng.integers(1 << 21, page * width, seqs)
    p = Pool(lens.tolist(), width, page, int(share * 32 * 1000) + 40, first=11, seed=1)
    got = run(p, want, 0, in_place, maps=(False, False, False))
    table, out, start, taken, no = served(p, want, 2 ** 31 - 1)
    assert no > 0 and got["status"] == uad.UAD_KV_NO_ROOM and int(start[-1]) > (2 ** 30 if share == 1 else 2 ** 28)
    assert np.array_equal(got["table"], table) and np.array_equal(got["lens"], out) and np.array_equal(got["start"], start)
    assert got["state"].tolist() == [(11 + taken) % p.n, int(p.state[1]) - taken]
