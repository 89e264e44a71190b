"""What is measured of the operators that a program needs to keep a vision-language model's keys and values beside an
expert in 8 bits, for long and many episodes: the pages' bookkeeping on the GPU, the append that rounds, and the
attention that reads them, in full or over a window and the first tokens (sinks).

- ``resize``: page tables, lengths, first rows and slot maps for the lengths that sequences shall have, from a ring of
  free pages (``PagePool.resize``).
- ``append``: keys (and queries) of new tokens are rotated by their positions; keys and values are rounded to e4m3 with a
  scale for each block of tokens and head, and written into the pages (``PagedCache.append`` on an 8-bit cache).
- ``attend``: attention of the new tokens of each sequence over such a cache, and attention over a window and the first
  tokens on caches of every type (``PagedCache.attention``).

Head layouts and prefix lengths are those of the repository's experts (8 query heads over one key/value head of 256, 4
over 1 of 128, 8 over 2 and 24 over 24 of 64, fp32 with 4 over 2 of 64; prefixes of 816 tokens) and the generic 32 over 8
of 128. Rows, keys, queries and values are N(0, 1), keys and values of a head times a power of two of its own, everything
drawn from the seed.
"""
import math

import torch

own = False

HEADS = {   # query heads, key/value heads, head dim
    "8x1x256": (8, 1, 256),
    "4x1x128": (4, 1, 128),
    "8x2x64": (8, 2, 64),
    "24x24x64": (24, 24, 64),
    "32x8x128": (32, 8, 128),
    "4x2x64": (4, 2, 64),
}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}   # of queries and outputs; an e4m3 cache has them in bf16
THETA = 10000.0
LEAST_SCALE = -100   # exponent of the least scale of a block


def _resize(seqs, new, at, page, back=0.0, room=1.0):
    """`seqs` sequences of 0 to `at` tokens get 1 to `new` more each; a share `back` of them gives up to `new` back instead.
    room: the free pages, as a share of what could be needed; sequences that find none stay as they are."""
    return dict(op="resize", seqs=seqs, new=new, at=at, page=page, back=back, room=room)


def _append(heads, seqs, new, at, page, block=16, ragged=False, rows="f32", layout="pshd", rot=None):
    """`seqs` sequences get `new` tokens each (ragged: 1 to `new`) after `at` earlier ones."""
    return dict(op="append", heads=heads, seqs=seqs, new=new, at=at, page=page, block=block, ragged=ragged, rows=rows,
                layout=layout, rot=HEADS[heads][2] if rot is None else rot)


def _attend(heads, seqs, keys, new=1, cache="e4m3", page=16, block=16, ragged=False, causal=True, window=0, sinks=0, masked=False,
            layout="pshd"):
    """`new` tokens of each sequence over its cache of `keys` tokens (ragged: a quarter of that and more), they included."""
    return dict(op="attend", heads=heads, seqs=seqs, keys=keys, new=new, cache=cache, page=page, block=block, ragged=ragged,
                causal=causal, window=window, sinks=sinks, masked=masked, layout=layout)


def listed():
    return [
        # the next token of 64 robots, a few of which take back rejected drafts: what every decoding step begins with
        dict(name="resize-64", **_resize(64, 5, 1129, 16, back=0.2)),
        # a fleet's prompts and ends of episodes at once: the most that one call lays out
        dict(name="resize-4000", **_resize(4000, 816, 816, 16, back=0.3)),
        # one robot's next text token joins a block of its prefix, from the projection's fp32 rows: latency alone
        dict(name="append8-1", **_append("8x1x256", 1, 1, 817, 16)),
        # 64 robots' whole prefixes (up to 816 tokens) enter the cache: the most that one call moves
        dict(name="append8-64x816", **_append("8x1x256", 64, 816, 0, 16, ragged=True)),
        # drafts of up to 9 tokens far into long episodes, blocks that end with odd pages, half of each head rotated
        dict(name="append8-drafts", **_append("24x24x64", 33, 9, 900001, 100, block=64, ragged=True, rows="bf16", layout="phsd", rot=32)),
        # the next text token of one robot over its prefix: latency
        dict(name="attend8-1", **_attend("8x1x256", 1, 817)),
        # the same for a batch of 64 robots, each with its own length
        dict(name="attend8-64", **_attend("8x1x256", 64, 1129, ragged=True)),
        # two long sequences with generic heads: the largest
        dict(name="attend8-long", **_attend("32x8x128", 2, 131071, page=64, block=64, ragged=True, layout="phsd")),
        # five drafted tokens a sequence, checked at once, blocks of odd pages, absent cameras masked
        dict(name="attend8-draft", **_attend("8x1x256", 6, 8003, new=5, page=100, block=32, ragged=True, masked=True)),
        # long episodes seen through a window and four sinks, 8 bits
        dict(name="attend8-sinks", **_attend("32x8x128", 33, 30011, page=64, block=32, ragged=True, window=2048, sinks=4)),
        # the same view of a bf16 cache, drafts of three
        dict(name="sinks-bf16", **_attend("24x24x64", 16, 20011, new=3, cache="bf16", page=12, ragged=True, window=1000, sinks=5)),
        # and of an fp32 one: a single robot, where latency counts
        dict(name="sinks-f32", **_attend("4x2x64", 1, 100003, cache="f32", page=16, window=512, sinks=4)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """The same ranges: one to 64 sequences (tables: to 4000), caches from one key to 131071, pages of 1 to 128 tokens,
    blocks of 16, 32 and 64, drafts and chunks of up to 16 tokens, whole prompts for tables and append, windows of 16 to 4096
    with up to 64 sinks."""
    op = rng.choice(["resize", "append", "append", "attend", "attend", "attend"])
    layout = rng.choice(["pshd", "phsd"])
    page = rng.choice([1, 5, 12, 16, 16, 16, 32, 64, 64, 100, 128])
    block = rng.choice([16, 16, 32, 64])
    if op == "resize":
        seqs = _log_int(rng, 1, 4000)
        return _resize(seqs, _log_int(rng, 1, 816), rng.choice([0, _log_int(rng, 1, 816)]), page, rng.choice([0.0, rng.random()]),
                       rng.choice([1.0, 1.0, 0.4]))
    heads = rng.choice(list(HEADS))
    hq, hkv, dh = HEADS[heads]
    seqs = _log_int(rng, 1, 64)
    if op == "append":
        new = _log_int(rng, 1, max(1, min(816, 85_000_000 // (seqs * (hq + 2 * hkv) * dh))))
        return _append(heads, seqs, new, rng.choice([0, _log_int(rng, 1, 1 << 20)]), page, block, rng.random() < 0.5,
                       rng.choice(["f32", "bf16"]), layout, rng.choice([dh, dh, dh // 2]))
    cache = rng.choice(["e4m3", "e4m3", "e4m3", "bf16", "f32"])
    new = rng.choice([1, 1, 1, 2, 3, 4, 5, 8, 16])
    window, sinks = 0, 0
    if cache != "e4m3" or rng.random() < 0.3:
        window, sinks = _log_int(rng, 16, 4096), rng.choice([1, 4, 4, _log_int(rng, 1, 64)])
    keys = max(new, _log_int(rng, 1, min(131071, 500_000_000 // (seqs * hkv * dh * 8 * (1 if new == 1 else 4)))))
    return _attend(heads, seqs, keys, new, cache, page, block, rng.random() < 0.6, rng.random() < 0.8, window, sinks,
                   rng.random() < 0.3, layout)


# ---- inputs -----------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(shape, g, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _randint(lo, hi, shape, g):
    """Whole numbers from lo to hi, hi included."""
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _spread(g, lo, hi, n):
    """n whole numbers evenly over lo..hi, in an order drawn from the seed."""
    order = torch.randperm(n, generator=g, device="cuda")
    return (hi - order * (hi - lo) // max(1, n - 1)).to(torch.int32)


def _scale_of(amax):
    """The least power of two that takes amax to 448 or below, 2^LEAST_SCALE at the least."""
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=LEAST_SCALE)
    return (torch.where(amax > 0, e, LEAST_SCALE).to(torch.int32) + 127 << 23).view(torch.float32)   # its bits: exact


def _laid_out(case, x):
    """Pages given as [pages][slot][head][dim] in the memory order that the case names."""
    return x.contiguous() if case["layout"] == "pshd" else x.transpose(1, 2).contiguous().transpose(1, 2)


def _pool(case, pages, g):
    """A layer's keys and values as [pages][slot][head][dim]; of an 8-bit cache with their scales [pages][block][head]."""
    hq, hkv, dh = HEADS[case["heads"]]
    page, block, kind = case["page"], case["block"], case.get("cache", "e4m3")
    got = []
    for _ in range(2):
        x = _randn((pages, page, hkv, dh), g, torch.float32)
        if kind != "e4m3":
            got += [_laid_out(case, x.to(TYPES[kind])), None]
            continue
        x *= torch.exp2(_randint(-2, 2, (hkv, 1), g).float())
        blocks = (page + block - 1) // block
        amax = torch.nn.functional.pad(x.abs().amax(-1), (0, 0, 0, blocks * block - page)).reshape(pages, blocks, block, hkv).amax(2)
        scale = _scale_of(amax)
        x /= scale.repeat_interleave(block, dim=1)[:, :page, :, None]
        got += [_laid_out(case, x.to(torch.float8_e4m3fn)), scale]
    return got


def _sequences(case, g, lens, counts, kept_from, pages_from):
    """Lengths, first rows and page table; the pages before `pages_from` have been given back (-1)."""
    page = case["page"]
    start = torch.zeros(case["seqs"] + 1, dtype=torch.int32, device="cuda")
    start[1:] = counts.cumsum(0)
    width = (int(lens.max()) + page - 1) // page
    used = width - pages_from
    table = torch.full((case["seqs"], width), -1, dtype=torch.int32, device="cuda")
    ids = torch.randperm(case["seqs"] * used + 3, generator=g, device="cuda").to(torch.int32)
    table[:, pages_from:] = ids[: case["seqs"] * used].reshape(case["seqs"], used)
    return dict(table=table, lens=lens, start=start, rows=int(start[-1])), case["seqs"] * used + 3


def _prepare_resize(case, g):
    seqs, page, new, at = case["seqs"], case["page"], case["new"], case["at"]
    lens = _spread(g, 0, at, seqs)
    step = _spread(g, 1, new, seqs)
    back = torch.randperm(seqs, generator=g, device="cuda") < round(case["back"] * seqs)
    want = torch.where(back, (lens - step).clamp(min=0), lens + step).to(torch.int32)
    width = (at + new + page - 1) // page
    held = (lens + page - 1) // page
    used = int(held.sum())
    spare = int(case["room"] * int(((step + page - 1) // page + 1).sum()))
    n_pages, rows = used + spare, int(step.sum()) + 5   # room of the token tensors: what all steps could need, and a little
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda")[None] < held[:, None]] = ids[:used]
    first = int(_randint(0, n_pages - 1, (1,), g))
    ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    ring[(first + torch.arange(spare, device="cuda")) % n_pages] = ids[used:]
    s = dict(case=case, table=table, lens=lens, want=want, ring=ring, n_pages=n_pages, rows=rows)
    s["state"] = torch.tensor([first, spare], dtype=torch.int32, device="cuda")
    s["state_out"] = torch.empty_like(s["state"])
    s["lens_out"] = torch.empty_like(lens)
    s["start"] = torch.empty(seqs + 1, dtype=torch.int32, device="cuda")
    s["slot"] = torch.empty(rows, dtype=torch.int64, device="cuda")
    s["row_seq"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    s["row_pos"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    if own:
        import paper_2609_37772_gb300 as uad
        s["pool"] = uad.PagePool(ring, s["state"], page)
    return s


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "resize":
        return _prepare_resize(case, g)
    hq, hkv, dh = HEADS[case["heads"]]
    seqs, new, page = case["seqs"], case["new"], case["page"]
    one = torch.ones(seqs, dtype=torch.int32, device="cuda")
    if case["op"] == "append":
        counts = _spread(g, 1, new, seqs) if case["ragged"] else one * new
        s, pages = _sequences(case, g, counts + case["at"], counts, case["at"], case["at"] // page)
        qkv = _randn((s["rows"], (hq + 2 * hkv) * dh), g, TYPES[case["rows"]])   # a fused projection's rows
        s["q"], s["k"], s["v"] = qkv.split([hq * dh, hkv * dh, hkv * dh], dim=1)
        s["q_out"] = torch.empty((s["rows"], hq * dh), device="cuda", dtype=torch.bfloat16)
    else:
        counts = one * new
        lens = _spread(g, max(new, case["keys"] // 4), case["keys"], seqs) if case["ragged"] else one * case["keys"]
        s, pages = _sequences(case, g, lens, counts, 0, 0)
        s["q"] = _randn((s["rows"], hq * dh), g, TYPES.get(case["cache"], torch.bfloat16))
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((s["rows"], hq), device="cuda")
        s["mask"] = None
        if case["masked"]:   # three cameras' worth of keys: each is there or not, text always is
            width = s["table"].shape[1] * page
            part = torch.arange(width, device="cuda") * 4 // max(1, case["keys"])
            there = torch.rand((seqs, 4), generator=g, device="cuda") < 0.6
            there[:, 3] = True
            s["mask"] = there[:, part.clamp(max=3)].to(torch.uint8).contiguous()
    s["case"] = case
    s["k_pages"], s["k_scale"], s["v_pages"], s["v_scale"] = _pool(case, pages, g)
    if own:   # what a program keeps for its cache: descriptors of the tensors, rotation table, workspace
        import paper_2609_37772_gb300 as uad
        s["cache"] = uad.PagedCache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], block=case["block"])
        s["seqs"] = uad.Sequences(s["table"], s["lens"], s["start"], max_len=case["keys"] if case["op"] == "attend" else 0, max_new=new)
        if case["op"] == "append":
            s["rope"] = uad.rope(THETA, case["rot"])
        else:
            need = s["cache"].attention_workspace(s["seqs"], s["rows"], hq, case["window"], sinks=case["sinks"])
            s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------


def _segments(counts, room):
    """Of `room` items in the order of their owners: owner and number within it; owner = len(counts) behind the last."""
    ends = counts.cumsum(0)
    item = torch.arange(room, device=counts.device)
    owner = torch.searchsorted(ends, item, right=True)
    first = torch.cat([ends - counts, ends[-1:]])
    return owner, item - first[owner]


def _run_resize(s):
    case = s["case"]
    if own:
        s["pool"].resize(s["table"], s["lens"], s["want"], s["start"], length_out=s["lens_out"], state_out=s["state_out"],
                         slot=s["slot"], row_seq=s["row_seq"], row_pos=s["row_pos"])
    else:
        page, seqs, n, width = case["page"], case["seqs"], s["n_pages"], s["table"].shape[1]
        lens, want = s["lens"].long(), s["want"].long()
        first, count = s["state"][0].long(), s["state"][1].long()
        held, needed = (lens + page - 1) // page, (want + page - 1) // page
        take, give, add = (needed - held).clamp(min=0), (held - needed).clamp(min=0), (want - lens).clamp(min=0)
        served = (take.cumsum(0) <= count) | (take == 0)
        served &= (add.cumsum(0) <= s["rows"]) | (add == 0)
        take, add = take * served, add * served
        # pages taken into the table, from the ring's front
        b, i = _segments(take, seqs * width)
        ok, b = b < seqs, b.clamp(max=seqs - 1)
        col = (held[b] + i).clamp(max=width - 1)
        item = torch.arange(seqs * width, device=lens.device)
        got = s["ring"][(first + item) % n]
        put = torch.full((seqs * width + 1,), -1, dtype=torch.int32, device=lens.device)
        flat = torch.where(ok, b * width + col, seqs * width)
        is_new = torch.zeros(seqs * width + 1, dtype=torch.bool, device=lens.device)
        put[flat], is_new[flat] = got, ok
        table = torch.where(is_new[:-1].reshape(seqs, width), put[:-1].reshape(seqs, width), s["table"])
        # pages given back, to the ring's end
        b, i = _segments(give, n)
        ok, b = b < seqs, b.clamp(max=seqs - 1)
        back = s["table"][b, (needed[b] + i).clamp(max=width - 1)]
        at = (first + count + torch.arange(n, device=lens.device)) % n
        s["ring"][at] = torch.where(ok, back, s["ring"][at])
        s["table"].copy_(table)
        # rows
        b, i = _segments(add, s["rows"])
        ok, b = b < seqs, b.clamp(max=seqs - 1)
        pos = lens[b] + i
        slot = s["table"][b, (pos // page).clamp(max=width - 1)].long() * page + pos % page
        s["slot"].copy_(torch.where(ok, slot, -1))
        s["row_seq"].copy_(torch.where(ok, b, -1))
        s["row_pos"].copy_(torch.where(ok, pos, -1))
        s["start"][0] = 0
        s["start"][1:] = add.cumsum(0)
        s["lens_out"].copy_(torch.where((want < lens) | (add > 0), want, lens))
        s["state_out"][0] = (first + take.sum()) % n
        s["state_out"][1] = count - take.sum() + give.sum()
    return {k: s[k] for k in ("table", "ring", "lens_out", "start", "state_out", "slot", "row_seq", "row_pos")}


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


def _bytes_of(x):
    return x.view(torch.uint8)


def _rounded_into(s, pages, scales, raw, values, doubled):
    """The new tokens' `values` [rows][heads][dim] into their blocks. A block's scale comes from the largest of its new tokens'
    raw values (doubled where they are rotated) and is never below that of its earlier tokens, which are rounded again where it grew."""
    case, block, page = s["case"], s["case"]["block"], s["case"]["page"]
    blocks, hkv = scales.shape[1], scales.shape[2]
    seq, pos = _rows_of(s)
    lens, counts = s["lens"].long(), (s["start"][1:] - s["start"][:-1]).long()
    at_page, slot = s["table"].long()[seq, pos // page], pos % page
    where = at_page * blocks + slot // block
    amax = torch.zeros((scales.shape[0] * blocks, hkv), device=raw.device)
    amax.scatter_reduce_(0, where[:, None].expand(-1, hkv), raw.float().abs().amax(-1), "amax")
    need = _scale_of(amax * 2 if doubled else amax)
    # the earlier tokens of each sequence's first block
    p0 = lens - counts
    in_page = p0 % page
    sub = in_page // block
    lo = sub * block                                    # the block's first slot
    first_page = s["table"].long()[torch.arange(case["seqs"], device=raw.device), (p0 // page).clamp(max=s["table"].shape[1] - 1)]
    earlier = (in_page > lo) & (counts > 0)
    old = scales.reshape(-1, hkv)
    floor = torch.zeros_like(old)
    fb = first_page * blocks + sub
    floor[fb[earlier]] = old[fb[earlier]]
    touched = torch.zeros(old.shape[0], dtype=torch.bool, device=raw.device)
    touched[where] = True
    fresh = torch.where(touched[:, None], torch.maximum(need, floor), old)
    slots = lo[:, None] + torch.arange(block, device=raw.device)
    kept = (slots < in_page[:, None]) & earlier[:, None]
    b = torch.arange(case["seqs"], device=raw.device)[:, None].expand(-1, block)[kept]
    pg, sl = first_page[b], slots[kept]
    x = _bytes_of(pages)[pg, sl].view(torch.float8_e4m3fn).float() * old[fb[b]][..., None] / fresh[fb[b]][..., None]
    _bytes_of(pages)[pg, sl] = _bytes_of(x.to(torch.float8_e4m3fn))
    _bytes_of(pages)[at_page, slot] = _bytes_of((values / fresh[where][..., None]).to(torch.float8_e4m3fn))
    scales.copy_(fresh.reshape(scales.shape))


def _run_append(s):
    case = s["case"]
    hq, hkv, dh = HEADS[case["heads"]]
    if own:
        s["cache"].append(s["seqs"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=s["rope"])
    else:
        seq, pos = _rows_of(s)
        s["q_out"].copy_(_rotated(s["q"], pos, case["rot"], hq).reshape(s["q_out"].shape))
        k, v = s["k"].reshape(-1, hkv, dh), s["v"].reshape(-1, hkv, dh)
        _rounded_into(s, s["k_pages"], s["k_scale"], k, _rotated(s["k"], pos, case["rot"], hkv), True)
        _rounded_into(s, s["v_pages"], s["v_scale"], v, v.float(), False)
    return {k: s[k] for k in ("q_out", "k_pages", "v_pages", "k_scale", "v_scale")}


def _read(s, pages, scales, page, slot):
    """Tokens [seqs][keys] of the cache in fp32, [seqs][heads][keys][dim]."""
    if scales is None:
        return pages[page, slot].float().permute(0, 2, 1, 3)
    x = _bytes_of(pages)[page, slot].view(torch.float8_e4m3fn).float()
    x *= scales[page, slot // s["case"]["block"]][..., None]
    return x.permute(0, 2, 1, 3)


def _run_attend(s):
    case = s["case"]
    hq, hkv, dh = HEADS[case["heads"]]
    if own:
        s["cache"].attention(s["seqs"], s["q"], s["out"], s["ws"], lse=s["lse"], causal=case["causal"], window=case["window"],
                             sinks=case["sinks"], key_mask=s["mask"])
        return {"out": s["out"], "lse": s["lse"]}
    seqs, new, rep, window, sinks = case["seqs"], case["new"], hq // hkv, case["window"], case["sinks"]
    lens = s["lens"].long()
    key = torch.arange(s["table"].shape[1] * case["page"], device=lens.device)[None]   # [1 or seqs][keys]
    seen = key < lens[:, None]
    if window and window + new - 1 + sinks < key.shape[1]:   # no more than the sinks and what the first token's window sees
        i = torch.arange(window + new - 1 + sinks, device=lens.device)[None]
        key = torch.where(i < sinks, i, lens[:, None] - (window + new - 1) + i - sinks)
        seen = (key < lens[:, None]) & ((i < sinks) | (key >= sinks))
        key = key.clamp(min=0)
    key = key.expand(seqs, -1)
    page = s["table"].long().gather(1, (key // case["page"]).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)
    slot = key % case["page"]
    k = _read(s, s["k_pages"], s["k_scale"], page, slot)
    q = s["q"].float().reshape(seqs, new, hkv, rep, dh).permute(0, 2, 1, 3, 4).reshape(seqs, hkv, new * rep, dh)
    score = (q @ k.transpose(-1, -2)).reshape(seqs, hkv, new, rep, -1) * dh ** -0.5
    del k
    pos = lens[:, None] - new + torch.arange(new, device=lens.device)   # [seqs][new]
    seen = seen[:, None]
    if case["causal"]:
        seen = seen & (key[:, None] <= pos[..., None])
    if window:
        seen = seen & ((key[:, None] > pos[..., None] - window) | (key[:, None] < sinks))
    if s["mask"] is not None:
        seen = seen & (s["mask"].gather(1, key.clamp(max=s["mask"].shape[1] - 1)) != 0)[:, None]
    seen = seen.expand(seqs, new, key.shape[1])
    score = score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = p.sum(-1, keepdim=True)
    v = _read(s, s["v_pages"], s["v_scale"], page, slot)
    v = torch.where(seen.any(1)[:, None, :, None], v, 0.0)
    o = (p.reshape(seqs, hkv, new * rep, -1) @ v).reshape(seqs, hkv, new, rep, dh)
    o = torch.where(total > 0, o / total, 0.0)
    s["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(s["out"].shape))
    s["lse"].copy_((top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(s["lse"].shape))
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    return {"resize": _run_resize, "append": _run_append, "attend": _run_attend}[state["case"]["op"]](state)


# ---- what a pass cannot do without, and its result in 64 bits ---------------------------------------


def work(case):
    seqs, new, page = case["seqs"], case["new"], case["page"]
    if case["op"] == "resize":
        rows = seqs * (1 - case["back"]) * (new + 1) / 2 * case["room"]
        pages = seqs * (new + 1) / 2 / page * case["room"]
        return {"bytes": seqs * 16 + rows * 16 + pages * 8 + 16.0, "flops": 0.0}
    hq, hkv, dh = HEADS[case["heads"]]
    if case["op"] == "append":
        rows = seqs * ((new + 1) / 2 if case["ragged"] else new)
        es = 4 if case["rows"] == "f32" else 2
        size = rows * ((hq + 2 * hkv) * dh * es + hq * dh * 2 + 2 * hkv * dh + 8 * hkv / min(page, case["block"]))
        return {"bytes": float(size), "flops": 3.0 * rows * (hq + hkv) * case["rot"] + 2.0 * rows * 2 * hkv * dh}
    # with ragged lengths from a quarter of the longest: five eighths of it on average
    keys = case["keys"] * (0.625 if case["ragged"] else 1.0)
    if case["window"]:
        keys = min(keys, case["window"] + new - 1 + case["sinks"])
    share = 0.7 if case["masked"] else 1.0   # masked keys need not be read
    kind = case["cache"]
    per_key = 2 * hkv * (dh + 4 / min(page, case["block"]) if kind == "e4m3" else dh * (2 if kind == "bf16" else 4))
    rows, es = seqs * new, 4 if kind == "f32" else 2
    size = seqs * keys * (per_key * share + (1 if case["masked"] else 0) + 4 / page) + rows * hq * (2 * dh * es + 4)
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


def _exact_resize(s):
    """By lists, sequence after sequence."""
    case, page, n, room = s["case"], s["case"]["page"], s["n_pages"], s["rows"]
    table, ring, lens, want = s["table"].tolist(), s["ring"].tolist(), s["lens"].tolist(), s["want"].tolist()
    first, count = s["state"].tolist()
    free = [ring[(first + i) % n] for i in range(count)]
    back, taken, out, start, rows = [], 0, [], [0], []
    asked_pages = asked_rows = 0
    for b in range(case["seqs"]):
        held, needed = -(-lens[b] // page), -(-want[b] // page)
        end = want[b]
        if want[b] >= lens[b]:
            asked_pages += needed - held
            asked_rows += want[b] - lens[b]
            if (needed > held and asked_pages > count) or asked_rows > room:
                end = lens[b]
            else:
                for i in range(held, needed):
                    table[b][i] = free[taken]
                    taken += 1
                rows += [(table[b][p // page] * page + p % page, b, p) for p in range(lens[b], want[b])]
        else:
            back += table[b][needed:held]
        out.append(end)
        start.append(len(rows))
    for i, p in enumerate(back):
        ring[(first + count + i) % n] = p
    rows += [(-1, -1, -1)] * (room - len(rows))
    whole = lambda v, t: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    slot, seq, pos = (list(x) for x in zip(*rows))
    return {"table": whole(table, torch.int32), "ring": whole(ring, torch.int32), "lens_out": whole(out, torch.int32),
            "start": whole(start, torch.int32), "state_out": whole([(first + taken) % n, count - taken + len(back)], torch.int32),
            "slot": whole(slot, torch.int64), "row_seq": whole(seq, torch.int32), "row_pos": whole(pos, torch.int32)}


def _exact_blocks(s, pages, scales, rows, turned, doubled):
    """Pages (before their rounding) and scales after the append, block after block."""
    case, page, block = s["case"], s["case"]["page"], s["case"]["block"]
    start, lens, table = s["start"].tolist(), s["lens"].tolist(), s["table"].tolist()
    pages, scales = pages.double(), scales.double().clone()
    for b in range(case["seqs"]):
        n = start[b + 1] - start[b]
        p = lens[b] - n
        while p < lens[b]:
            at, sub = table[b][p // page], p % page // block
            lo = p // page * page + sub * block
            hi = min(lo + block, p // page * page + page, lens[b])
            r = slice(start[b] + p - (lens[b] - n), start[b] + hi - (lens[b] - n))
            top = rows[r].double().abs().amax(-1).amax(0) * (2.0 if doubled else 1.0)
            e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / 448.0))
            e = torch.where(448.0 * torch.exp2(e - 1) >= top, e - 1, e)   # a logarithm that was rounded up
            fresh = torch.exp2(e.clamp(min=float(LEAST_SCALE)))
            if p > lo:
                fresh = torch.maximum(fresh, scales[at, sub])
                pages[at, sub * block: p % page] *= (scales[at, sub] / fresh)[:, None]
            scales[at, sub] = fresh
            pages[at, p % page: p % page + hi - p] = turned[r] / fresh[:, None]
            p = hi
    return pages, scales


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "resize":
        return _exact_resize(s)
    hq, hkv, dh = HEADS[case["heads"]]
    start, lens = s["start"].tolist(), s["lens"].tolist()
    if case["op"] == "append":
        pos = torch.cat([torch.arange(lens[b] - (start[b + 1] - start[b]), lens[b], device="cuda") for b in range(case["seqs"])])
        k, v = s["k"].reshape(-1, hkv, dh), s["v"].reshape(-1, hkv, dh)
        kp, ks = _exact_blocks(s, s["k_pages"], s["k_scale"], k, _exact_rotation(k, pos, case["rot"], dh), True)
        vp, vs = _exact_blocks(s, s["v_pages"], s["v_scale"], v, v.double(), False)
        q = _exact_rotation(s["q"].reshape(-1, hq, dh), pos, case["rot"], dh).reshape(s["rows"], -1)
        return {"q_out": q, "k_pages": kp, "v_pages": vp, "k_scale": ks, "v_scale": vs}
    out = torch.zeros((s["rows"], hq, dh), dtype=torch.float64, device="cuda")
    lse = torch.full((s["rows"], hq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        n = lens[b]
        at = torch.arange(n, device="cuda")
        if case["window"]:
            at = at[(at < case["sinks"]) | (at > n - case["new"] - case["window"])]
        page, slot = s["table"][b].long()[torch.div(at, case["page"], rounding_mode="floor")], at.remainder(case["page"])
        k, v = [x.view(torch.uint8)[page, slot].view(x.dtype).double() if sc is not None else x[page, slot].double()
                for x, sc in ((s["k_pages"], s["k_scale"]), (s["v_pages"], s["v_scale"]))]
        if s["k_scale"] is not None:
            sub = torch.div(slot, case["block"], rounding_mode="floor")
            k, v = k * s["k_scale"][page, sub].double()[..., None], v * s["v_scale"][page, sub].double()[..., None]
        here = torch.ones(at.numel(), dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"][b, at] != 0
        for r in range(start[b], start[b + 1]):
            pos = n - (start[b + 1] - r)
            see = here.clone()
            if case["causal"]:
                see &= at <= pos
            if case["window"]:
                see &= (at > pos - case["window"]) | (at < case["sinks"])
            if not bool(see.any()):
                continue
            ks, vs = k[see], v[see]
            q = s["q"][r].double().reshape(hkv, -1, dh)
            z = torch.einsum("hgd,khd->hgk", q, ks) / math.sqrt(dh)
            lse[r] = torch.logsumexp(z, dim=-1).reshape(-1)
            out[r] = torch.einsum("hgk,khd->hgd", torch.softmax(z, dim=-1), vs).reshape(hq, dh)
    return {"out": out.reshape(s["rows"], -1), "lse": lse}
