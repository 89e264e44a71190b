"""What is measured of the operators around an expert's prefix: the work that a program has them do that keeps
the vision-language model's keys and values in a paged cache, extends it by a few tokens at a time and binds it
to the action expert.

- ``append``: keys (and queries) of new tokens are rotated by their positions, keys and values written into
  the pages of their sequences (``PagedCache.append``).
- ``attend``: attention of the new tokens of each sequence over its pages (``PagedCache.attention``).
- ``linear4``: the projections of those tokens with 4-bit weights, a scale and a zero point a group
  (``linear_w4``).

Head layouts, widths and prefix lengths are those of the repository's experts (8 query heads over one
key/value head of 256, 4 over 1 of 128, 8 over 2 and 24 over 24 of 64, fp32 with 4 over 2 of 64; widths 1024, 1536
and 2048; prefixes of 816 tokens) and the generic 32 over 8 of 128. Rows, keys, queries and values are N(0, 1),
everything drawn from the seed.
"""
import math

import torch

own = False

HEADS = {   # query heads, key/value heads, head dim, type of the cache
    "8x1x256": (8, 1, 256, "bf16"),
    "4x1x128": (4, 1, 128, "bf16"),
    "8x2x64": (8, 2, 64, "bf16"),
    "24x24x64": (24, 24, 64, "bf16"),
    "32x8x128": (32, 8, 128, "bf16"),
    "4x2x64-f32": (4, 2, 64, "f32"),
    "8x1x256-f32": (8, 1, 256, "f32"),
}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _append(heads, seqs, new, at, page, ragged=False, rows="f32", layout="pshd", rot=None):
    """`seqs` sequences get `new` tokens each (ragged: 1 to `new`) after `at` earlier ones."""
    return dict(op="append", heads=heads, seqs=seqs, new=new, at=at, page=page, ragged=ragged, rows=rows, layout=layout,
                rot=HEADS[heads][2] if rot is None else rot)


def _attend(heads, seqs, keys, new=1, page=16, ragged=False, causal=True, window=0, masked=False, layout="pshd"):
    """`new` tokens of each sequence over its cache of `keys` tokens (ragged: a quarter of that and more), they included."""
    return dict(op="attend", heads=heads, seqs=seqs, keys=keys, new=new, page=page, ragged=ragged, causal=causal,
                window=window, masked=masked, layout=layout)


def _linear4(rows, k, n, group, zero=True, bias=False):
    return dict(op="linear4", rows=rows, k=k, n=n, group=group, zero=zero, bias=bias)


def listed():
    return [
        # one robot's next text token joins its prefix, straight from the projection's fp32 rows: latency alone
        dict(name="append-1", **_append("8x1x256", 1, 1, 816, 16)),
        # 64 robots' whole prefixes (up to 816 tokens) enter the cache: the most that one call moves
        dict(name="append-64x816", **_append("8x1x256", 64, 816, 0, 16, ragged=True)),
        # fp32 cache, drafts of up to 33 tokens far into long episodes, odd pages, half of each head rotated
        dict(name="append-far", **_append("4x2x64-f32", 7, 33, 900001, 12, ragged=True, layout="phsd", rot=32)),
        # the next text token of one robot over its prefix: latency
        dict(name="attend-1", **_attend("8x1x256", 1, 817)),
        # the same for a batch of 64 robots, each with its own length
        dict(name="attend-64", **_attend("8x1x256", 64, 1129, ragged=True)),
        # two long sequences with generic heads: the largest
        dict(name="attend-long", **_attend("32x8x128", 2, 131071, page=64, ragged=True, layout="phsd")),
        # five drafted tokens a sequence, checked at once
        dict(name="attend-draft", **_attend("8x1x256", 6, 8003, new=5, page=32, ragged=True)),
        # an fp32 chunk of 16 action tokens over prefixes of which absent cameras are masked, odd pages
        dict(name="attend-chunk-f32", **_attend("4x2x64-f32", 33, 592, new=16, page=12, ragged=True, causal=False, masked=True)),
        # one token through a qkv projection of the pi0-like expert's sizes: the smallest weight
        dict(name="linear4-1", **_linear4(1, 1024, 2560, 64, zero=False)),
        # one token through a fused gate and up projection: the largest matrix for a single token
        dict(name="linear4-1-wide", **_linear4(1, 2048, 32768, 128)),
        # five drafted tokens through a long-K down projection, small groups
        dict(name="linear4-5-down", **_linear4(5, 8192, 2048, 32, bias=True)),
        # a batch of 40 robots' tokens, odd number of outputs
        dict(name="linear4-40", **_linear4(40, 4096, 14337, 64)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """The same ranges: one to 64 sequences, caches from one key to 131071, pages of 1 to 128 tokens, drafts and chunks
    of up to 16 tokens, whole prompts for the append; projections of 1 to 64 rows over groups of 32, 64 and 128."""
    op = rng.choice(["append", "attend", "attend", "linear4", "linear4"])
    layout = rng.choice(["pshd", "phsd"])
    page = rng.choice([1, 5, 12, 16, 16, 16, 32, 64, 64, 100, 128])
    if op == "append":
        heads = rng.choice(list(HEADS))
        seqs = _log_int(rng, 1, 64)
        hq, hkv, dh, _ = HEADS[heads]
        new = _log_int(rng, 1, max(1, min(816, 120_000_000 // (seqs * (hq + 2 * hkv) * dh))))
        rot = rng.choice([dh, dh, dh // 2])
        rows = "f32" if HEADS[heads][3] == "f32" else rng.choice(["f32", "bf16"])
        return _append(heads, seqs, new, rng.choice([0, _log_int(rng, 1, 1 << 20)]), page, rng.random() < 0.5, rows, layout, rot)
    if op == "attend":
        heads = rng.choice(list(HEADS))
        hq, hkv, dh, kind = HEADS[heads]
        seqs = _log_int(rng, 1, 64)
        per_key = hkv * dh * 2 * (2 if kind == "bf16" else 4)
        new = rng.choice([1, 1, 1, 2, 3, 4, 5, 8, 16])
        keys = max(new, _log_int(rng, 1, min(131071, 700_000_000 // (seqs * per_key * (1 if new == 1 else 4)))))
        if kind == "f32":
            keys = max(new, min(keys, 300_000_000 // (seqs * per_key * new)))
        window = _log_int(rng, 16, 4096) if rng.random() < 0.25 else 0
        return _attend(heads, seqs, keys, new, page, rng.random() < 0.6, rng.random() < 0.8, window, rng.random() < 0.3, layout)
    rows, group = _log_int(rng, 1, 64), rng.choice([32, 64, 128])
    k = group * _log_int(rng, 256 // group, 8192 // group)
    n = _log_int(rng, 7, min(32768, 67_000_000 * 32 // (k * max(rows, 32))))
    return _linear4(rows, k, n, group, rng.random() < 0.7, rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(shape, g, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _spread(g, lo, hi, n):
    """n whole numbers evenly over lo..hi, in an order drawn from the seed."""
    order = torch.randperm(n, generator=g, device="cuda")
    return (hi - order * (hi - lo) // max(1, n - 1)).to(torch.int32)


def _pool(case, pages, g):
    """A layer's keys and values as [pages][page][heads][dim], in the memory order that the case names."""
    _, hkv, dh, kind = HEADS[case["heads"]]
    shape = (2, pages, case["page"], hkv, dh) if case["layout"] == "pshd" else (2, pages, hkv, case["page"], dh)
    both = _randn(shape, g, TYPES[kind])
    if case["layout"] == "phsd":
        both = both.transpose(2, 3)
    return both[0], both[1]


def _sequences(case, g, lens, counts, kept_from):
    """Lengths, first rows and page table; the pages before token `kept_from` have been given back (-1)."""
    page = case["page"]
    start = torch.zeros(case["seqs"] + 1, dtype=torch.int32, device="cuda")
    start[1:] = counts.cumsum(0)
    width = (int(lens.max()) + page - 1) // page
    first = kept_from // page
    used = width - first
    table = torch.full((case["seqs"], width), -1, dtype=torch.int32, device="cuda")
    ids = torch.randperm(case["seqs"] * used + 3, generator=g, device="cuda").to(torch.int32)
    table[:, first:] = ids[: case["seqs"] * used].reshape(case["seqs"], used)
    return dict(table=table, lens=lens, start=start, rows=int(start[-1])), case["seqs"] * used + 3


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "linear4":
        m, k, n, group = case["rows"], case["k"], case["n"], case["group"]
        s = dict(case=case)
        s["w"] = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
        s["scale"] = torch.rand((n, k // group), generator=g, device="cuda").mul_(0.006).add_(0.002).bfloat16()
        s["zero"] = torch.randint(5, 12, (n, k // group), generator=g, device="cuda", dtype=torch.uint8) if case["zero"] else None
        s["bias"] = _randn((n,), g, torch.float32).mul_(0.02) if case["bias"] else None
        s["x"] = _randn((m, k), g, torch.bfloat16)
        s["out"] = torch.empty((m, n), device="cuda")
        return s
    hq, hkv, dh, kind = HEADS[case["heads"]]
    seqs, new = case["seqs"], case["new"]
    one = torch.ones(seqs, dtype=torch.int32, device="cuda")
    if case["op"] == "append":
        counts = _spread(g, 1, new, seqs) if case["ragged"] else one * new
        s, pages = _sequences(case, g, counts + case["at"], counts, case["at"])
        dtype = TYPES[case["rows"]]
        qkv = _randn((s["rows"], (hq + 2 * hkv) * dh), g, dtype)   # a fused projection's rows
        s["q"], s["k"], s["v"] = qkv.split([hq * dh, hkv * dh, hkv * dh], dim=1)
        s["q_out"] = torch.empty((s["rows"], hq * dh), device="cuda", dtype=TYPES[kind])
    else:
        counts = one * new
        lens = _spread(g, max(new, case["keys"] // 4), case["keys"], seqs) if case["ragged"] else one * case["keys"]
        s, pages = _sequences(case, g, lens, counts, 0)
        s["q"] = _randn((s["rows"], hq * dh), g, TYPES[kind])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((s["rows"], hq), device="cuda")
        s["mask"] = None
        if case["masked"]:   # three cameras' worth of keys: each is there or not, text always is
            width = s["table"].shape[1] * case["page"]
            part = torch.arange(width, device="cuda") * 4 // max(1, case["keys"])
            there = torch.rand((seqs, 4), generator=g, device="cuda") < 0.6
            there[:, 3] = True
            s["mask"] = there[:, part.clamp(max=3)].to(torch.uint8).contiguous()
    s["case"] = case
    s["k_pages"], s["v_pages"] = _pool(case, pages, g)
    if own:   # what a program keeps for its cache: descriptors of the tensors, rotation table, workspace
        import paper_2609_37772_gb300 as uad
        s["cache"] = uad.PagedCache(s["k_pages"], s["v_pages"])
        s["seqs"] = uad.Sequences(s["table"], s["lens"], s["start"], max_len=case["keys"] if case["op"] == "attend" else 0, max_new=new)
        if case["op"] == "append":
            s["rope"] = uad.rope(THETA, case["rot"])
        else:
            s["ws"] = torch.empty(s["cache"].attention_workspace(s["seqs"], s["rows"], hq, case["window"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------

THETA = 10000.0


def _rows_of(s):
    """Sequence and position of every row, in 64-bit whole numbers."""
    row = torch.arange(s["rows"], device=s["table"].device)
    seq = torch.searchsorted(s["start"].long(), row, right=True) - 1
    start, lens = s["start"].long(), s["lens"].long()
    return seq, lens[seq] - (start[seq + 1] - row)


def _rotated(x, pos, rot, heads):
    """Rows of `heads` heads rotated at `pos`: pairs (i, i + rot/2) by pos THETA^(-2i/rot), the rest of a head as it is."""
    x = x.reshape(x.shape[0], heads, -1).float()
    inv = THETA ** (-torch.arange(rot // 2, dtype=torch.float64, device=x.device) * 2 / rot)
    ang = pos.double()[:, None] * inv
    c, n = ang.cos().float()[:, None], ang.sin().float()[:, None]
    a, b = x[..., : rot // 2], x[..., rot // 2: rot]
    return torch.cat([a * c - b * n, b * c + a * n, x[..., rot:]], dim=-1)


def _run_append(s):
    case = s["case"]
    hq, hkv, dh, kind = HEADS[case["heads"]]
    if own:
        s["cache"].append(s["seqs"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=s["rope"])
    else:
        seq, pos = _rows_of(s)
        page, slot = s["table"].long()[seq, pos // case["page"]], pos % case["page"]
        s["q_out"].copy_(_rotated(s["q"], pos, case["rot"], hq).reshape(s["q_out"].shape))
        s["k_pages"][page, slot] = _rotated(s["k"], pos, case["rot"], hkv).to(TYPES[kind])
        s["v_pages"][page, slot] = s["v"].reshape(-1, hkv, dh).to(TYPES[kind])
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _run_attend(s):
    case = s["case"]
    hq, hkv, dh, kind = HEADS[case["heads"]]
    if own:
        s["cache"].attention(s["seqs"], s["q"], s["out"], s["ws"], lse=s["lse"], causal=case["causal"], window=case["window"],
                             key_mask=s["mask"])
        return {"out": s["out"], "lse": s["lse"]}
    seqs, new, rep = case["seqs"], case["new"], hq // hkv
    key = torch.arange(s["table"].shape[1] * case["page"], device=s["q"].device)
    page = s["table"].long()[:, key // case["page"]].clamp(min=0)
    k = s["k_pages"][page, key % case["page"]].float().permute(0, 2, 1, 3)   # [seqs][hkv][keys][dh]
    q = s["q"].float().reshape(seqs, new, hkv, rep, dh).permute(0, 2, 1, 3, 4).reshape(seqs, hkv, new * rep, dh)
    score = (q @ k.transpose(-1, -2)).reshape(seqs, hkv, new, rep, -1) * dh ** -0.5
    del k
    pos = s["lens"].long()[:, None] - new + torch.arange(new, device=key.device)   # [seqs][new]
    seen = key[None, None] < s["lens"].long()[:, None, None]
    if case["causal"]:
        seen = seen & (key[None, None] <= pos[..., None])
    if case["window"]:
        seen = seen & (key[None, None] > pos[..., None] - case["window"])
    if s["mask"] is not None:
        seen = seen & (s["mask"] != 0)[:, None]
    seen = seen.expand(seqs, new, key.numel())
    score = score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = p.sum(-1, keepdim=True)
    v = s["v_pages"][page, key % case["page"]].float()
    v = torch.where(seen.any(1)[..., None, None], v, 0.0).permute(0, 2, 1, 3)
    o = (p.reshape(seqs, hkv, new * rep, -1) @ v).reshape(seqs, hkv, new, rep, dh)
    o = torch.where(total > 0, o / total, 0.0)
    s["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(s["out"].shape))
    s["lse"].copy_((top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(s["lse"].shape))
    return {"out": s["out"], "lse": s["lse"]}


def _run_linear4(s):
    case = s["case"]
    if own:
        import paper_2609_37772_gb300 as uad
        uad.linear_w4(s["x"], s["w"], s["scale"], s["out"], zero=s["zero"], bias=s["bias"])
        return s["out"]
    n, groups = s["scale"].shape
    w = torch.stack([s["w"] & 15, s["w"] >> 4], dim=-1).reshape(n, groups, -1).float()
    w = (w - (8.0 if s["zero"] is None else s["zero"].float()[..., None])) * s["scale"].float()[..., None]
    out = s["x"].float() @ w.reshape(n, case["k"]).t()
    s["out"].copy_(out if s["bias"] is None else out + s["bias"])
    return s["out"]


def run(state):
    return {"append": _run_append, "attend": _run_attend, "linear4": _run_linear4}[state["case"]["op"]](state)


# ---- what a pass cannot do without, and its result in 64 bits ---------------------------------------


def work(case):
    if case["op"] == "linear4":
        m, k, n, groups = case["rows"], case["k"], case["n"], case["k"] // case["group"]
        size = n * k / 2 + n * groups * (3 if case["zero"] else 2) + 2 * m * k + 4 * m * n + (4 * n if case["bias"] else 0)
        return {"bytes": float(size), "flops": 2.0 * m * k * n}
    hq, hkv, dh, kind = HEADS[case["heads"]]
    es = 2 if kind == "bf16" else 4
    if case["op"] == "append":
        rows = case["seqs"] * ((case["new"] + 1) / 2 if case["ragged"] else case["new"])
        values = rows * (hq + 2 * hkv) * dh
        return {"bytes": values * ((4 if case["rows"] == "f32" else 2) + es), "flops": 3.0 * rows * (hq + hkv) * case["rot"]}
    # with ragged lengths from a quarter of the longest: five eighths of it on average
    keys = case["keys"] * (0.625 if case["ragged"] else 1.0)
    if case["window"]:
        keys = min(keys, case["window"] + case["new"] - 1)
    share = 0.7 if case["masked"] else 1.0   # masked keys need not be read
    rows = case["seqs"] * case["new"]
    size = case["seqs"] * keys * (2 * hkv * dh * es * share + (1 if case["masked"] else 0) + 4 / case["page"]) + rows * hq * (2 * dh * es + 4)
    return {"bytes": float(size), "flops": 4.0 * rows * hq * dh * keys * share}


def _exact_rotation(x, pos, rot, dh):
    """x [n][heads][dh] in 64 bits: each pair as a complex number times exp(i angle)."""
    x = x.double().clone()
    half = rot // 2
    freq = torch.exp(torch.arange(half, device=x.device, dtype=torch.float64) * (-2.0 * math.log(THETA) / rot))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), pos.double()[:, None, None] * freq)
    z = torch.complex(x[..., :half].contiguous(), x[..., half:rot].contiguous()) * turn
    x[..., :half], x[..., half:rot] = z.real, z.imag
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear4":
        group, out = case["group"], []
        for i in range(0, case["n"], 4096):
            w = s["w"][i:i + 4096].to(torch.int64)
            q = torch.empty((w.shape[0], case["k"]), dtype=torch.float64, device=w.device)
            q[:, 0::2], q[:, 1::2] = (w % 16).double(), (w // 16).double()
            q = q.reshape(w.shape[0], -1, group)
            q = q - (8 if s["zero"] is None else s["zero"][i:i + 4096].double().unsqueeze(-1))
            q = (q * s["scale"][i:i + 4096].double().unsqueeze(-1)).reshape(w.shape[0], -1)
            out.append(torch.einsum("mk,nk->mn", s["x"].double(), q))
        out = torch.cat(out, dim=1)
        return out if s["bias"] is None else out + s["bias"].double()
    hq, hkv, dh, _ = HEADS[case["heads"]]
    start, lens = s["start"].tolist(), s["lens"].tolist()
    if case["op"] == "append":
        q = torch.empty((s["rows"], hq, dh), dtype=torch.float64, device="cuda")
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        for b in range(case["seqs"]):
            lo, hi = start[b], start[b + 1]
            pos = torch.arange(lens[b] - (hi - lo), lens[b], device="cuda")
            page = s["table"][b].long()[torch.div(pos, case["page"], rounding_mode="floor")]
            at = (page, pos.remainder(case["page"]))
            q[lo:hi] = _exact_rotation(s["q"][lo:hi].reshape(-1, hq, dh), pos, case["rot"], dh)
            kp[at] = _exact_rotation(s["k"][lo:hi].reshape(-1, hkv, dh), pos, case["rot"], dh)
            vp[at] = s["v"][lo:hi].reshape(-1, hkv, dh).double()
        return {"q": q.reshape(s["rows"], -1), "k_pages": kp, "v_pages": vp}
    out = torch.zeros((s["rows"], hq, dh), dtype=torch.float64, device="cuda")
    lse = torch.full((s["rows"], hq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        n = lens[b]
        pages = s["table"][b, : (n + case["page"] - 1) // case["page"]].long()
        k = s["k_pages"][pages].reshape(-1, hkv, dh)[:n].double()
        v = s["v_pages"][pages].reshape(-1, hkv, dh)[:n].double()
        at = torch.arange(n, device="cuda")
        here = torch.ones(n, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"][b, :n] != 0
        for r in range(start[b], start[b + 1]):
            pos = n - (start[b + 1] - r)
            see = here.clone()
            if case["causal"]:
                see &= at <= pos
            if case["window"]:
                see &= at > pos - case["window"]
            if not bool(see.any()):
                continue
            ks, vs = k[see], v[see]
            q = s["q"][r].double().reshape(hkv, -1, dh)
            z = torch.einsum("hgd,khd->hgk", q, ks) / math.sqrt(dh)
            lse[r] = torch.logsumexp(z, dim=-1).reshape(-1)
            out[r] = torch.einsum("hgk,khd->hgd", torch.softmax(z, dim=-1), vs).reshape(hq, dh)
    return {"out": out.reshape(s["rows"], -1), "lse": lse}
