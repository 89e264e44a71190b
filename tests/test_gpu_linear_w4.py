"""GPU parity of the 4-bit projection against its 64-bit reference.

Tolerance: products of bf16 and whole numbers up to 15 are exact; a group's sum of at most 128 of them is off by an ulp a
step (the tensor cores truncate), 2^-23 of the sum of magnitudes each, as is every group that is added: (group + groups + 2)
2^-23 sum |x w|, and the output's own half step 2^-24. The same is demanded where the zero is subtracted after a group's sum,
although the terms then are |x| (q + zero).
(Every kernel now subtracts the zero before the product.)
"""
import math

import numpy as np
import pytest
import torch

import paper_2609_37772_gb300 as uad
from oracle import paged

pytestmark = pytest.mark.gpu


def operands(M, N, K, group, zero, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scale = (torch.rand((N, K // group), generator=g, device="cuda") * 0.01 - 0.002).bfloat16()
    z = torch.randint(0, 256, (N, K // group), generator=g, device="cuda", dtype=torch.uint8) if zero else None
    x = torch.randn((M, K), generator=g, device="cuda").bfloat16()
    return x, q, scale, z, torch.randn(N, generator=g, device="cuda")


def reference(x, q, scale, z, bias):
    w = paged.dequantize(q.cpu().numpy(), scale.float().cpu().numpy(), None if z is None else z.cpu().numpy())
    xn = x.double().cpu().numpy()
    with np.errstate(all="ignore"):
        return xn @ w.T + (0 if bias is None else bias.double().cpu().numpy()), np.abs(xn) @ np.abs(w).T


def check(out, want, size, K, group, bias):
    tol = (group + K // group + 2) * 2.0 ** -23 * size + 2.0 ** -23 * (np.abs(want) + (0 if bias is None else np.abs(bias.double().cpu().numpy()))) + 1e-30
    err = np.abs(out.double().cpu().numpy() - want)
    assert np.all(err <= tol), float((err / tol).max())


SHAPES = [(1, 1, 32, 32), (1, 16, 64, 64), (1, 17, 128, 128), (1, 2560, 1024, 64), (1, 100, 4096, 128), (2, 33, 96, 32), (3, 1000, 256, 128),
          (5, 2048, 8192, 32), (7, 15, 384, 128), (8, 64, 2048, 64), (9, 640, 160, 32), (16, 129, 512, 64), (17, 77, 704, 64), (24, 4608, 1536, 128),
          (31, 31, 992, 32), (32, 256, 1024, 128), (33, 513, 320, 64), (40, 1409, 4096, 64), (63, 48, 640, 128), (64, 1024, 2048, 32), (64, 7, 12288, 128),
          (16, 40, 36864, 128), (9, 24, 8320, 64), (16, 300, 4224, 32), (4, 16, 16384, 128), (13, 5000, 2304, 64), (1, 9, 2176, 32), (2, 20000, 512, 64)]


@pytest.mark.parametrize("M,N,K,group", SHAPES)
@pytest.mark.parametrize("zero", [False, True])
def test_linear_w4_matches_reference(M, N, K, group, zero):
    x, q, scale, z, bias = operands(M, N, K, group, zero, M + N + K)
    bias = bias if zero else None
    room = torch.full((M + 2, N), 7.5, device="cuda")
    uad.linear_w4(x, q, scale, room[1:M + 1], zero=z, bias=bias)
    torch.cuda.synchronize()
    want, size = reference(x, q, scale, z, bias)
    check(room[1:M + 1], want, size, K, group, bias)
    assert bool((room[0] == 7.5).all()) and bool((room[M + 1] == 7.5).all())


@pytest.mark.parametrize("M", [1, 2, 4, 8, 12, 20, 36, 50, 64])
def test_rows_do_not_depend_on_each_other(M):
    """A row's values are its own whatever is beside it: NaN and infinities stay in their rows."""
    x, q, scale, z, bias = operands(M, 96, 512, 64, True, M)
    clean = torch.empty(M, 96, device="cuda")
    uad.linear_w4(x, q, scale, clean, zero=z, bias=bias)
    x2 = x.clone()
    x2[M // 2, 5] = float("nan")
    x2[M - 1, 500] = float("inf")
    out = torch.empty(M, 96, device="cuda")
    uad.linear_w4(x2, q, scale, out, zero=z, bias=bias)
    torch.cuda.synchronize()
    same = [m for m in range(M) if m not in (M // 2, M - 1)]
    assert torch.equal(out[same], clean[same])
    assert bool(torch.isnan(out[M // 2]).all()) and not bool(torch.isfinite(out[M - 1]).any() and M > 1 and M // 2 != M - 1 and
                                                             bool(((out[M - 1] != clean[M - 1]) & torch.isfinite(out[M - 1])).any()))


def test_quantized_weights_give_what_they_stand_for():
    rng = np.random.default_rng(3)
    w = (rng.normal(size=(512, 200)) * 0.02).astype(np.float32)
    x = torch.from_numpy(rng.normal(size=(3, 512)).astype(np.float32)).cuda().bfloat16()
    for symmetric in (False, True):
        q, s, z = uad.quantize_w4(w, 64, symmetric)
        scale = torch.from_numpy(s.view(np.int16)).cuda().view(torch.bfloat16)
        zt = None if z is None else torch.from_numpy(z).cuda()
        out = torch.empty(3, 200, device="cuda")
        uad.linear_w4(x, torch.from_numpy(q).cuda(), scale, out, zero=zt)
        torch.cuda.synchronize()
        want, size = reference(x, torch.from_numpy(q), scale, zt, None)
        check(out, want, size, 512, 64, None)
        full = x.double().cpu().numpy() @ w.astype(np.float64)
        step = float(scale.float().max())
        assert np.abs(want - full).max() <= step * 1.06 * np.abs(x.double().cpu().numpy()).sum(axis=1).max()


def test_linear_w4_is_the_same_every_time_on_streams_and_in_graphs():
    """In stream order with its weights' and inputs' writers; replayed with other inputs; the same bits every time."""
    x, q, scale, z, bias = operands(5, 2048, 4096, 64, True, 1)
    xs = [torch.randn(5, 4096, device="cuda").bfloat16() for _ in range(4)]
    st, out = torch.cuda.Stream(), torch.empty(5, 2048, device="cuda")
    alone = []
    for v in xs:
        o = torch.empty(5, 2048, device="cuda")
        uad.linear_w4(v, q, scale, o, zero=z, bias=bias)
        alone.append(o)
    torch.cuda.synchronize()
    got = []
    with torch.cuda.stream(st):
        for v in xs * 3:
            x.copy_(v)
            uad.linear_w4(x, q, scale, out, zero=z, bias=bias, stream=st)
            got.append(out.clone())
    torch.cuda.synchronize()
    assert all(torch.equal(o, alone[i % 4]) for i, o in enumerate(got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        uad.linear_w4(x, q, scale, out, zero=z, bias=bias, stream=st)
    for i, v in enumerate(xs):
        x.copy_(v)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, alone[i])


@pytest.mark.parametrize("M", [1, 7, 40])
def test_unaligned_outputs_scales_and_biases(M):
    """Outputs, bias, scales and zeros at any element address; nothing around the output is written."""
    N, K = 75, 320
    x, q, scale, z, bias = operands(M, N, K, 64, True, M)
    room = torch.full((M * N + 3,), 7.5, device="cuda")
    s1, z1 = torch.zeros(scale.numel() + 1, device="cuda", dtype=torch.bfloat16), torch.zeros(z.numel() + 1, device="cuda", dtype=torch.uint8)
    s1[1:] = scale.reshape(-1)
    z1[1:] = z.reshape(-1)
    b1 = torch.cat([bias[:1], bias])
    out = room[1:1 + M * N].view(M, N)
    uad.linear_w4(x, q, s1[1:].view(N, -1), out, zero=z1[1:].view(N, -1), bias=b1[1:])
    torch.cuda.synchronize()
    want, size = reference(x, q, scale, z, bias)
    check(out, want, size, K, 64, bias)
    assert float(room[0]) == 7.5 and bool((room[1 + M * N:] == 7.5).all())


# From 33 tokens and 2^24 weights on: one CTA for all of K, clusters of 2 to 8, an end of K and of N inside a tile
LARGE = [(33, 4101, 4128, 32), (40, 24000, 704, 64), (48, 2050, 8320, 128), (64, 24321, 736, 32), (57, 1030, 16448, 64), (64, 131, 130048, 128),
         (49, 9000, 1888, 32), (36, 14337, 1184, 32), (41, 14337, 1216, 64), (64, 6000, 2816, 128), (34, 20000, 896, 128)]


@pytest.mark.parametrize("M,N,K,group", LARGE)
@pytest.mark.parametrize("zero", [False, True])
def test_many_tokens_and_weights_match_reference(M, N, K, group, zero):
    test_linear_w4_matches_reference(M, N, K, group, zero)


@pytest.mark.parametrize("M,group", [(33, 64), (48, 32), (64, 128)])
def test_rows_of_large_calls_do_not_depend_on_each_other(M, group):
    x, q, scale, z, bias = operands(M, 4100, 4224, group, True, M)
    clean, out = torch.empty(M, 4100, device="cuda"), torch.empty(M, 4100, device="cuda")
    uad.linear_w4(x, q, scale, clean, zero=z, bias=bias)
    x2 = x.clone()
    x2[3, 5], x2[M - 1, 4223] = float("nan"), float("inf")
    uad.linear_w4(x2, q, scale, out, zero=z, bias=bias)
    torch.cuda.synchronize()
    same = [m for m in range(M) if m not in (3, M - 1)]
    assert torch.equal(out[same], clean[same])
    assert bool(torch.isnan(out[3]).all())


def test_large_calls_at_the_same_time():
    """Calls of several sizes on three streams, none of which waits for another, and replayed from graphs: the bits of calls that
    were alone."""
    calls = [operands(M, N, K, group, True, M) for M, N, K, group in ((64, 9000, 1888, 32), (40, 2050, 8320, 64), (48, 14337, 1280, 128))]
    streams = [torch.cuda.Stream() for _ in calls]
    outs = [[torch.empty(x.shape[0], q.shape[0], device="cuda") for _ in range(8)] for x, q, *_ in calls]
    alone = []
    for x, q, s, z, b in calls:
        alone.append(torch.empty(x.shape[0], q.shape[0], device="cuda"))
        uad.linear_w4(x, q, s, alone[-1], zero=z, bias=b)
        torch.cuda.synchronize()
    for i in range(8):
        for (x, q, s, z, b), st, o in zip(calls, streams, outs):
            uad.linear_w4(x, q, s, o[i], zero=z, bias=b, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, a) for os, a in zip(outs, alone) for o in os)
    graphs = []
    for (x, q, s, z, b), st, o in zip(calls, streams, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=st):
            for i in range(8):
                uad.linear_w4(x, q, s, o[i].fill_(7.5), zero=z, bias=b, stream=st)
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, a) for os, a in zip(outs, alone) for o in os)


def test_large_calls_among_the_other_projections():
    """Alternating with uad_linear, which also takes tensor memory and may start before the call in front of it has ended: in one
    stream's order, on two streams at once, and in graphs."""
    M, N, K = 48, 6144, 4096
    calls = [operands(M, N, K, 64, True, 11), operands(40, 14337, 2048, 128, True, 12)]
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    lin = []
    for m, n, k in ((637, 1024, 2048), (50, 1024, 4096), (16, 4608, 1536), (3000, 1024, 128)):
        w = torch.randn((k, n), generator=g, device="cuda").mul_(0.02).cpu().numpy()
        lin.append((torch.randn((m, k), generator=g, device="cuda").bfloat16(), torch.from_numpy(uad.tile_weight(w).view(np.int16)).cuda(), m, n, k))

    def chain(stream):
        outs = []
        for i in range(8):
            x, q, s, z, b = calls[i % 2]
            outs.append(torch.empty(x.shape[0], q.shape[0], device="cuda"))
            uad.linear_w4(x, q, s, outs[-1], zero=z, bias=b, stream=stream)
            x, w, m, n, k = lin[i % 4]
            outs.append(torch.empty(m, n, device="cuda"))
            assert uad.uad_linear(x.data_ptr(), w.data_ptr(), None, outs[-1].data_ptr(), m, n, k, stream.cuda_stream) == 0
        return outs

    streams = [torch.cuda.Stream() for _ in range(2)]
    with torch.cuda.stream(streams[0]):
        alone = chain(streams[0])
    torch.cuda.synchronize()
    for i in range(2):
        want, size = reference(*calls[i])
        check(alone[2 * i], want, size, calls[i][0].shape[1], (64, 128)[i], calls[i][4])
    got = []
    for st in streams:
        with torch.cuda.stream(st):
            got += [chain(st), chain(st)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        got.append(chain(streams[0]))
    with torch.cuda.stream(streams[1]):
        got.append(chain(streams[1]))
    with torch.cuda.stream(streams[0]):
        for _ in range(3):
            graph.replay()
    torch.cuda.synchronize()
    for outs in got:
        for i, (o, a) in enumerate(zip(outs, alone)):
            if i % 2:   # uad_linear's own tolerance
                assert float((o - a).abs().max()) <= 1e-5 * float(a.abs().max())
            else:
                assert torch.equal(o, a)


# From one token to 64: rows of 16 that a CTA's warps share or own, a K that a cluster shares, tiles of 32 rows, tcgen05
NEAR_ZERO = [(M, N, K, group) for group in (32, 64, 128) for M, N, K in ((1, 75, 512), (1, 2560, 4096), (2, 300, 16384), (2, 20000, 512), (3, 2100, 2048),
                                                                        (6, 20000, 512), (8, 640, 1024), (20, 333, 2048), (40, 4101, 4224))]


@pytest.mark.parametrize("M,N,K,group", NEAR_ZERO)
@pytest.mark.parametrize("zero", [False, True])
def test_large_tokens_at_the_zero_point_have_no_influence(M, N, K, group, zero):
    """Half of the tokens' values are thousands of times the others (a model's outlier channels), and all their weights the zero
    point: the terms that are left are small, and so is the tolerance, which counts |x w| alone."""
    x, q, scale, z, bias = operands(M, N, K, group, zero, M + N + K + 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(M + K)
    out = torch.empty(M, N, device="cuda")
    big = torch.rand(K, generator=g, device="cuda") < 0.5
    x = torch.where(big, x.float() * 4096 + 2048, x.float()).bfloat16()
    zp = torch.full((N, K // group), 8, device="cuda", dtype=torch.uint8) if z is None else z & 15
    rep = zp.repeat_interleave(group, dim=1)
    w = torch.where(big, rep, torch.stack([q & 15, q >> 4], dim=-1).reshape(N, K))
    q = (w[:, 0::2] | w[:, 1::2] << 4).contiguous()
    uad.linear_w4(x, q, scale, out, zero=z)
    torch.cuda.synchronize()
    want, size = reference(x, q, scale, z, None)
    check(out, want, size, K, group, None)


@pytest.mark.parametrize("M,N,K,group", NEAR_ZERO)
@pytest.mark.parametrize("zero", [False, True])
def test_rows_of_the_zero_point_alone_give_the_bias(M, N, K, group, zero):
    x, q, scale, z, bias = operands(M, N, K, group, zero, M + N + K + 2)
    x = (x.float() + 1).bfloat16()
    zp = torch.full((N, K // group), 8, device="cuda", dtype=torch.uint8) if z is None else z & 15
    rows = (zp | zp << 4).repeat_interleave(group // 2, dim=1)
    q[::3] = rows[::3]
    out = torch.empty(M, N, device="cuda")
    uad.linear_w4(x, q, scale, out, zero=z, bias=bias)
    torch.cuda.synchronize()
    assert torch.equal(out[:, ::3], bias[::3].expand(M, -1))


INFINITE = [(1, 96, 512), (2, 96, 512), (1, 20000, 512), (3, 20000, 512), (2, 300, 16384), (4, 2100, 2048), (12, 96, 512), (20, 333, 2048), (64, 96, 512), (33, 4100, 4224)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", INFINITE)
def test_infinite_tokens_give_infinities_or_nan(M, N, K, group):
    """Every value of a row with an infinity, by itself or beside others, is what the definition has: an infinity of the weight's
    sign, NaN where the weight is 0 or infinities meet. The rows beside it keep their bits."""
    x, q, scale, z, bias = operands(M, N, K, group, True, M + N)
    clean, out = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda")
    uad.linear_w4(x, q, scale, clean, zero=z, bias=bias)
    for row, at in ((M - 1, {K - 12: math.inf}), (0, {5: -math.inf}), (M // 2, {7: math.inf, K - 3: -math.inf, K // 2: math.inf})):
        x2 = x.clone()
        for k, v in at.items():
            x2[row, k] = v
        uad.linear_w4(x2, q, scale, out, zero=z, bias=bias)
        torch.cuda.synchronize()
        w = paged.dequantize(q.cpu().numpy(), scale.float().cpu().numpy(), z.cpu().numpy())
        with np.errstate(invalid="ignore"):
            want = sum(v * w[:, k] for k, v in at.items())
        got = out[row].double().cpu().numpy()
        assert not np.isfinite(got).any() and np.array_equal(got, want, equal_nan=True)
        same = [m for m in range(M) if m != row]
        assert torch.equal(out[same], clean[same])
