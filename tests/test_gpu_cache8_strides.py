"""The 8-bit cache where strides share large powers of two: pages 2^32 bytes apart are pages of their own."""
import pytest
import torch

import paper_2609_37772_gb300 as uad
from test_gpu_cache8 import CODES, Case8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("apart", [1 << 31, 1 << 32])
def test_pages_4_gib_apart(apart):
    """Pages of one token and one head, keys and values in one buffer: the bits of a small pool."""
    c = Case8((4, 1, 64), 1, [2], [1], seed=1, rows_behind=0, spare=0)
    cache = c.on_gpu()
    buf = torch.empty(apart + 128, dtype=torch.uint8, device="cuda")
    k, v = (buf[x:].as_strided((2, 1, 1, 64), (apart, apart, apart, 1)).view(CODES) for x in (0, 64))
    k.view(torch.uint8).copy_(cache.k.view(torch.uint8))
    v.view(torch.uint8).copy_(cache.v.view(torch.uint8))
    far = uad.PagedCache(k, v, cache.k_scale, cache.v_scale)
    s = c.sequences()
    q = torch.randn(1, 256, device="cuda").bfloat16()
    rows = torch.randn(1, 128, device="cuda")
    got = []
    for x in (cache, far):
        out, lse = torch.zeros_like(q), torch.zeros(1, 4, device="cuda")
        x.append(s, rows[:, :64], rows[:, 64:])
        x.attention(s, q, out, lse=lse)
        torch.cuda.synchronize()
        got.append((out, lse, x.k.view(torch.uint8).clone(), x.v.view(torch.uint8).clone()))
    assert all(torch.equal(a, b) for a, b in zip(*got))
