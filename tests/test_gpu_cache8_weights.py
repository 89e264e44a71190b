"""Weights of the 8-bit attention where values' scales lie far apart: what a row does not see, or gives no weight, does not cost it precision.

Tolerances. Scores, probabilities and sums as in test_gpu_cache8: rel = 2 (2 d + 2^-20 + n 2^-23) of sum p |v|, bf16's half step of the output. Weights p sv
are f16, 2^10 to 2^15 where the largest of the row so far is: off by 2^-11 relative, and by 2^-24 where they are not normal numbers, which is 2^-34 of
that largest one for each code. p below 2^-126 counts as nothing.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged, paged8
from test_gpu_cache8 import HALF, Case8, run_attention

pytestmark = pytest.mark.gpu
ONE_F16 = 2.0 ** -11


def check_near(c, q, out, lse, causal=True, window=0, sinks=0, scale=None, weights=ONE_F16):
    """The largest error, in tolerances."""
    scale = 1 / math.sqrt(c.dh) if scale is None else scale
    qn, on, ln = q.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    group, worst = c.hq // c.hkv, 0.0
    for t, (b, pos) in enumerate(paged.rows_of(c.lens, c.start)):
        j = np.arange(c.lens[b])
        seen = j <= pos if causal else np.ones(c.lens[b], bool)
        if window:
            seen &= (j > pos - window) | (j < sinks)
        n = int(seen.sum())
        pg, sl = c.table[b, j // c.page], j % c.page
        scales = c.scales[1].astype(np.float32).astype(np.float64)[pg, sl // c.block][seen]
        k, codes = c.held(b, 0)[seen], paged8.VALUES[c.codes[1][pg, sl]][seen]
        for h in range(c.hkv):
            rows = qn[t].reshape(c.hq, c.dh)[h * group:(h + 1) * group]
            got, gl = on[t].reshape(c.hq, c.dh)[h * group:(h + 1) * group], ln[t, h * group:(h + 1) * group]
            z = scale * rows @ k[:, h].T
            top = z.max(axis=1, keepdims=True)
            p = np.exp(z - top)
            wl = (top + np.log(p.sum(axis=1, keepdims=True)))[:, 0]
            p /= p.sum(axis=1, keepdims=True)
            w = p * scales[:, h]
            want, size = w @ codes[:, h], w @ np.abs(codes[:, h])
            d = (c.dh * 2.0 ** -23 + 2.0 ** -22) * abs(scale) * (np.abs(rows) @ np.abs(k[:, h]).T).max(axis=1, keepdims=True)
            rel = 2 * (2 * d + 2.0 ** -20 + n * 2.0 ** -23) + weights
            tol = rel * size + HALF * np.abs(want) + 2.0 ** -34 * w.max(axis=1, keepdims=True) * np.abs(codes[:, h]).sum(axis=0)
            tol += 2.0 ** -125 * (scales[:, h, None] * np.abs(codes[:, h])).sum(axis=0)
            worst = max(worst, float((np.abs(got - want) / tol).max()))
            assert worst <= 1, (t, b, h, worst)
            assert np.all(np.abs(gl - wl) <= d[:, 0] + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -22 * np.abs(wl)), (t, h)
    return worst


HEADS = [(8, 1, 256), (2, 1, 256), (4, 2, 128), (16, 1, 128), (40, 2, 128), (8, 8, 64), (16, 4, 64), (24, 1, 64)]


@pytest.mark.parametrize("power", [34, 40, 100])
@pytest.mark.parametrize("page", [5, 16])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_scales_of_later_tokens_do_not_reach_earlier_rows(heads, page, power):
    """Drafts whose later tokens lie in a block of far larger values: the same slice of keys, hidden from the earlier rows."""
    c = Case8(heads, page, [20, 36, 710], [9, 7, 12], 16, seed=power)
    for b, first in ((0, 16 if page == 16 else 15), (1, 32 if page == 16 else 35), (2, 704 if page == 16 else 700)):   # from this token on
        for pos in range(first, c.lens[b]):
            pg, _, sub = c.token(b, pos)
            c.scales[1][pg, sub] = 2.0 ** power * 1.25
    q, out, lse, status = run_attention(c)
    assert status == 0
    check_near(c, q, out, lse)


@pytest.mark.parametrize("power", [34, 100])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_scales_before_the_window_do_not_reach_later_rows(heads, power):
    """The first rows' windows hold a token of far larger values that the later rows' do not."""
    c = Case8(heads, 1, [50, 400], [6, 8], 16, seed=power + 1)
    window = 20
    for b in range(2):
        at = c.lens[b] - c.new[b] - window + 2   # rows 0 and 1 see it
        c.scales[1][c.table[b, at]] = 2.0 ** power
    for sinks in (0, 3):
        q, out, lse, status = run_attention(c, True, window, sinks)
        assert status == 0
        check_near(c, q, out, lse, True, window, sinks)


@pytest.mark.parametrize("power", [34, 40, 80])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_scales_of_tokens_without_weight_cost_nothing(heads, power):
    """A token of weight e^-64 with far larger values, first, last and between: with 2^80 it is what the output is made of."""
    c = Case8(heads, 1, [1, 40, 40, 40, 300, 300, 300], [1] * 7, 16, seed=power + 2)
    for b, at in ((1, 0), (2, 39), (3, 17), (4, 0), (5, 299), (6, 130)):
        pg = c.table[b, at]
        c.scales[1][pg] = 2.0 ** power
        c.codes[0][pg], c.scales[0][pg] = paged8.encode(np.float64(-8.0)), 8.0 / c.dh
    q = torch.ones((c.rows, c.hq * c.dh), device="cuda", dtype=torch.bfloat16)
    for b in range(1, 7):   # all other keys: zeros, so that their scores are 0
        for i in range(c.lens[b]):
            if c.codes[0][c.table[b, i]].flat[0] != int(paged8.encode(np.float64(-8.0))):
                c.codes[0][c.table[b, i]] = 0
    q, out, lse, status = run_attention(c, q=q, scale=1.0)
    assert status == 0
    check_near(c, q, out, lse, scale=1.0)


@pytest.mark.parametrize("heads,new", [((8, 1, 256), 5), ((8, 2, 64), 3), ((32, 8, 128), 1)], ids=str)
def test_scales_far_apart_in_keys_that_are_shared_evenly(heads, new):
    """Parts of sequences whose largest values differ by 2^60, joined through the workspace."""
    c = Case8(heads, 16, [1500, 40, 257, 2900], [new, 1, new, new], seed=new, width=60000)
    for b in range(4):
        for i in range(-(-c.lens[b] // 16)):
            c.scales[1][c.table[b, i]] = 2.0 ** c.rng.integers(-30, 31, c.hkv)
    q, out, lse, status = run_attention(c, max_len=900000)
    assert status == 0
    check_near(c, q, out, lse)


def test_scales_far_apart_where_warps_have_heads_of_their_own():
    c = Case8((24, 24, 64), 5, [1 + 7 * i % 90 for i in range(60)], [1] * 60, seed=6)
    c.scales[1] *= 2.0 ** c.rng.integers(-30, 31, c.scales[1].shape)
    q, out, lse, status = run_attention(c, max_len=90)
    assert status == 0
    check_near(c, q, out, lse)


@pytest.mark.parametrize("value", [math.nan, math.inf, 0.0])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_scales_that_a_row_does_not_see_may_hold_anything(heads, value):
    """The bits of the earlier rows, whatever the scales of a later token's block are."""
    outs = []
    for x in (1.0, value):
        c = Case8(heads, 5, [20, 710], [9, 12], 16, seed=15)
        for b, pos in ((0, 15), (1, 700)):
            for which in range(2):
                c.scales[which][c.token(b, pos)[0]] = x
        q, out, lse, status = run_attention(c)
        assert status == 0
        outs.append((out, lse))
    rows = [0, 1, 2, 3, 9, 10]   # positions 11 to 14, 698 and 699
    assert torch.equal(outs[0][0][rows], outs[1][0][rows]) and torch.equal(outs[0][1][rows], outs[1][1][rows])


TWO_F16 = 2.0 ** -20


def test_weights_have_more_than_one_f16():
    """Two tokens of nearly opposite contributions: what is left of them is 2^-9 and less of each, which one f16 a weight misses by up to an eighth."""
    n = 300
    c = Case8((1, 1, 64), 1, [2] * n, [1] * n, 16, seed=13)
    x = paged8.encode((c.rng.normal(size=(n, 64)) * 100).clip(-448, 448))
    q = torch.zeros((c.rows, 64), device="cuda", dtype=torch.bfloat16)
    q[:, 0] = 1.0
    for b in range(n):
        one, two = c.table[b]
        for pg, score in ((one, 0.0), (two, c.rng.uniform(-2, 0))):   # one dim alone: scores whose own error is small
            c.codes[0][pg] = 0
            c.codes[0][pg, 0, 0, 0] = paged8.encode(np.float64(1.0 if score else 0.0))
            c.scales[0][pg] = np.float32(abs(score) or 1.0)
        c.codes[1][one, 0, 0], c.codes[1][two, 0, 0] = x[b], x[b] ^ 0x80
        c.scales[1][one] = np.float32(c.rng.uniform(0.5, 1))
        # the second token's weight e^score: as large as the first one's contribution, but for 2^-9
        c.scales[1][two] = np.float32(c.scales[1][one] * math.exp(-float(c.scales[0][two, 0, 0])) * (1 + 2.0 ** -9))
    q, out, lse, status = run_attention(c, q=q, scale=1.0)
    assert status == 0
    check_near(c, q, out, lse, scale=1.0, weights=TWO_F16)


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_weights_of_drafts_have_more_than_one_f16(heads):
    c = Case8(heads, 16, [33, 300, 9], [5, 3, 9], 16, seed=14)
    c.scales[1] *= 2.0 ** c.rng.integers(-9, 9, c.scales[1].shape)
    for causal in (True, False):
        q, out, lse, status = run_attention(c, causal)
        assert status == 0
        check_near(c, q, out, lse, causal, weights=TWO_F16)
