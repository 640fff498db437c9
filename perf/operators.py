"""Cases of the paged 8-bit cache: attention over it, the write that fills it, and the moves of its pages.

The cache keeps keys and values in 8 bits (int8 or e4m3) in pages of `page` tokens; every block of 16 tokens
of a (layer, page, head) has one magnitude for its keys and one for its values:

    value = code * amax / 127   (int8)        value = code * amax / 448   (e4m3)

Buffers, all on the device:
    codes  uint8  [layers, pages, heads, 2 (K, V), page * D]   16-token tiles of 16 * D bytes, see `unpack`
    amax   fp32   [layers, pages, heads, 2, page / 16]
    table  int32  [seqs, seq_pages]   page of every stretch of `page` tokens of a sequence, -1 = none
    lens   int32  [seqs]              tokens of a sequence
    refs   int32  [pages]             sequences that hold a page; 0 = free

A case's sequence lengths and page numbers follow from the case, what the buffers hold from the seed.
"""
import math
import random

import torch

own = False

BLOCK = 16
TOP = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"fp16": torch.float16, "bf16": torch.bfloat16}


# --------------------------------------------------------------------------- #
# the cases
# --------------------------------------------------------------------------- #
def attention(name, n, lo, hi, heads, group, dim, new_lo=1, new_hi=1, page=64, dtype="bf16", fmt="int8", window=0,
              sinks=0):
    c = {"op": "attention", "n": n, "len_lo": lo, "len_hi": hi, "new_lo": new_lo, "new_hi": new_hi, "layers": 1,
         "heads": heads, "group": group, "dim": dim, "page": page, "dtype": dtype, "fmt": fmt, "window": window,
         "sinks": sinks}
    return dict(c, name=name) if name else c


def write(name, n, lo, hi, new_lo, new_hi, layers, heads, dim, page=64, dtype="bf16", fmt="int8"):
    c = {"op": "write", "n": n, "len_lo": lo, "len_hi": hi, "new_lo": new_lo, "new_hi": new_hi, "layers": layers,
         "heads": heads, "group": 1, "dim": dim, "page": page, "dtype": dtype, "fmt": fmt}
    return dict(c, name=name) if name else c


def beam(name, n, children, lo, hi, layers, heads, dim, page=64, fmt="int8"):
    c = {"op": "beam", "n": n, "children": children, "len_lo": lo, "len_hi": hi, "layers": layers, "heads": heads,
         "group": 1, "dim": dim, "page": page, "dtype": "fp16", "fmt": fmt}
    return dict(c, name=name) if name else c


def compact(name, n, lo, hi, done, layers, heads, dim, window, sinks, page=64, fmt="int8"):
    c = {"op": "compact", "n": n, "done": done, "len_lo": lo, "len_hi": hi, "layers": layers, "heads": heads,
         "group": 1, "dim": dim, "page": page, "dtype": "fp16", "fmt": fmt, "window": window, "sinks": sinks}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one short conversation, eight heads: what counts is latency
        attention("step_small", 1, 250, 250, 8, 1, 128, dtype="fp16"),
        # a serving batch between its shortest and its longest conversation, four query heads per KV head
        attention("step_ragged", 64, 1, 4000, 8, 4, 128),
        # two long documents, eight query heads per KV head: few rows, a long axis
        attention("step_long", 2, 100003, 131072, 8, 8, 128, fmt="e4m3"),
        # first tokens and a sliding window over long conversations, a query head per KV head
        attention("step_window", 16, 4000, 8192, 40, 1, 128, dtype="fp16", window=1024, sinks=4),
        # the multi-query model: 71 query heads over one KV head of dimension 64
        attention("step_multiquery", 64, 200, 2048, 1, 71, 64, dtype="fp16"),
        # prompts that go in by pieces beside sequences that generate: 1 to 2048 new tokens each
        attention("chunk_ragged", 5, 700, 8000, 8, 4, 128, 1, 2048),
        # a whole prompt under first tokens and window
        attention("chunk_window", 1, 8192, 8192, 32, 1, 128, 8192, 8192, dtype="fp16", window=1024, sinks=4),
        # every sequence of a batch grows by one token in four layers
        write("write_step", 64, 2, 500, 1, 1, 4, 8, 128),
        # the prompts of a batch, four layers
        write("write_prompt", 8, 517, 4096, 517, 4096, 4, 8, 128, dtype="fp16", fmt="e4m3"),
        # four continuations of one conversation, one layer: what counts is latency
        beam("beam_small", 1, 4, 250, 250, 1, 8, 128),
        # beam search: the children of 32 beams let go of their pages and fork again, eight layers
        beam("beam_large", 32, 3, 100, 1000, 8, 8, 128),
        # a quarter of the sequences has ended, the others keep first tokens and window: the pool closes up
        compact("compact_window", 64, 500, 4000, 16, 4, 4, 128, 512, 4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["step", "step", "chunk", "write", "beam", "compact"])
    dim = rng.choice([128, 128, 64])
    page = rng.choice([16, 32, 64, 128])
    dtype, fmt = rng.choice(["fp16", "bf16"]), rng.choice(["int8", "e4m3"])
    heads = rng.choice([1, 2, 3, 8, 8, 32, 40])
    if op in ("step", "chunk"):
        group = rng.choice([1, 2, 4, 5, 8]) if heads > 1 else rng.choice([1, 8, 16, 71])
        window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 100, 4000), rng.choice([0, 4, 17]))])
    if op == "step":
        n = _log(rng, 1, 128)
        hi = _log(rng, 16, min(120000, 400_000_000 // (n * heads * dim)))
        return attention("", n, rng.randint(1, hi), hi, heads, group, dim, page=page, dtype=dtype, fmt=fmt,
                         window=window, sinks=sinks)
    if op == "chunk":
        n = rng.randint(1, 6)
        rows = 65536 // (heads * group)
        new = _log(rng, 2, max(8, min(2048, rows)))
        hi = new + _log(rng, 16, min(8000, max(64, 200_000_000 // (n * heads * group * new))))
        return attention("", n, max(new, rng.randint(1, hi)), hi, heads, group, dim, rng.randint(1, new), new, page,
                         dtype, fmt, window, sinks)
    layers = rng.choice([1, 2, 4])
    heads = min(heads, 8)
    if op == "write":
        n = _log(rng, 1, 64)
        hi = _log(rng, 2, 90_000 // n)
        new = rng.choice([1, hi, rng.randint(1, hi)])
        return write("", n, max(new, rng.randint(1, hi)), hi, rng.randint(1, new), new, layers, heads, dim, page,
                     dtype, fmt)
    if op == "beam":
        n = _log(rng, 1, 32)
        hi = _log(rng, 20, 1000)
        return beam("", n, rng.randint(1, 4), rng.randint(1, hi), hi, layers, heads, dim, page, fmt)
    n = rng.randint(2, 64)
    hi = _log(rng, 300, 4000)
    return compact("", n, rng.randint(1, hi), hi, rng.randint(1, n - 1), min(layers, 2), min(heads, 4), dim,
                   rng.randint(64, 700), rng.choice([0, 4]), page, fmt)


def _spread(lo, hi, n):
    """n whole numbers over [lo, hi], hi first, lo last."""
    v = [lo + int((hi - lo + 1) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]
    v[-1] = lo
    v[0] = hi
    return v


def _shape(case):
    """Lengths and page table of a case: what a scheduler has in hand."""
    pt, n = case["page"], case["n"]
    rnd = random.Random(7)
    new = _spread(case.get("new_lo", 0), case.get("new_hi", 0), n)
    lens = [max(a, b) for a, b in zip(_spread(case["len_lo"], case["len_hi"], n), new)]
    kids = case.get("children", 0)
    total = n * (1 + kids)
    seqs = total + 2                                    # two sequences of the table are not in use
    rows = list(range(seqs))
    rnd.shuffle(rows)
    old = [a - b if case["op"] == "write" else a for a, b in zip(lens, new)]
    used = [-(-a // pt) for a in old]
    room = max(-(-a // pt) for a in lens)
    spare = sum(-(-a // pt) for a in lens) - sum(used) + 3
    ids = list(range(sum(used) + n * kids + spare))
    rnd.shuffle(ids)
    take = iter(ids)
    table = [[-1] * room for _ in range(seqs)]
    length = [0] * seqs
    refs = [0] * len(ids)
    for i in range(n):
        r = rows[i]
        for p in range(used[i]):
            table[r][p] = next(take)
        length[r] = old[i]
    for i in range(n):                                  # the children of the beam step before
        for c in range(kids):
            r = rows[n + i * kids + c]
            table[r] = list(table[rows[i]])
            if old[i] % pt:
                table[r][old[i] // pt] = next(take)
            length[r] = old[i]
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] += 1
    return {"table": table, "lens": length, "refs": refs, "rows": rows[:n], "kids": rows[n:total], "want": lens,
            "new": new, "pages": len(ids), "seqs": seqs, "room": room}


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _fill(case, s, g):
    """Codes of about normal values and their magnitudes; one key block in a hundred is four times as large."""
    pt, D, L, H = case["page"], case["dim"], case["layers"], case["heads"]
    codes = torch.empty((L, s["pages"], H, 2, pt * D), dtype=torch.uint8, device="cuda")
    for layer in range(L):
        x = torch.randn(codes[layer].shape, generator=g, device="cuda", dtype=torch.float32)
        if case["fmt"] == "int8":
            codes[layer] = x.mul_(36.0).round_().clamp_(-127, 127).to(torch.int8).view(torch.uint8)
        else:
            codes[layer] = x.mul_(128.0).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    amax = torch.rand((L, s["pages"], H, 2, pt // BLOCK), generator=g, device="cuda") * 1.5 + 2.5
    big = torch.rand(amax[:, :, :, 0].shape, generator=g, device="cuda") < 0.01
    amax[:, :, :, 0] = torch.where(big, amax[:, :, :, 0] * 4, amax[:, :, :, 0])
    amax = amax.to(DTYPE[case["dtype"]]).float()        # a magnitude is one of the 16-bit inputs'
    return codes, amax


def prepare(case, seed):
    s = _shape(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    L, H, D = case["layers"], case["heads"], case["dim"]
    codes, amax = _fill(case, s, g)
    st = {"case": case, "codes": codes, "amax": amax, "table": ints(s["table"]), "lens": ints(s["lens"]),
          "refs": ints(s["refs"]), "seqs": ints(s["rows"])}
    if case["op"] in ("attention", "write"):
        starts = [0]
        for x in s["new"]:
            starts.append(starts[-1] + x)
        st["starts"] = ints(starts)
        shape = (starts[-1], L, H * case["group"] if case["op"] == "attention" else H, D)
        draw16 = lambda: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        if case["op"] == "attention":
            st["q"] = draw16().to(DTYPE[case["dtype"]])
        else:
            k = draw16()
            heavy = torch.rand(shape[:3] + (1,), generator=g, device="cuda") < 0.01
            st["k"] = torch.where(heavy, k * 4, k).to(DTYPE[case["dtype"]])
            st["v"] = draw16().to(DTYPE[case["dtype"]])
            st["want"] = ints(s["want"])
    elif case["op"] == "beam":
        st["kids"] = ints(s["kids"])
        st["parents"] = st["seqs"].repeat_interleave(case["children"])
        st["zeros"] = torch.zeros_like(st["kids"])
    else:
        st["ended"] = st["seqs"][:case["done"]].clone()
        st["kept"] = st["seqs"][case["done"]:].clone()
        st["zeros"] = torch.zeros_like(st["ended"])
        st["before"] = [st[k].clone() for k in ("table", "lens", "refs")]
    if own:                                             # the handle that a program keeps beside these buffers
        from paper_2402_09398_b200 import binding
        st["cache"] = binding.PagedCache(L, H, D, s["pages"], s["seqs"], s["room"], group=case["group"],
                                         page_tokens=case["page"], fmt=case["fmt"], dtype=DTYPE[case["dtype"]],
                                         buffers={k: st[k] for k in ("codes", "amax", "table", "lens", "refs")})
    return st


# --------------------------------------------------------------------------- #
# one pass
# --------------------------------------------------------------------------- #
def run(state):
    op = state["case"]["op"]
    if op == "attention":
        return (own_attention if own else plain_attention)(state)
    if op == "write":
        (own_write if own else plain_write)(state)
    elif op == "beam":
        (own_beam if own else plain_beam)(state)
    else:
        for k, v in zip(("table", "lens", "refs"), state["before"]):  # the same holes in every pass
            state[k].copy_(v)
        (own_compact if own else plain_compact)(state)
    return {k: state[k] for k in ("table", "lens", "refs", "codes", "amax")}


def own_attention(st):
    c = st["case"]
    if c["new_hi"] == 1:
        return st["cache"].attention(st["q"], st["seqs"], window=c["window"], sinks=c["sinks"])
    return st["cache"].attention(st["q"], st["seqs"], st["starts"], max_new=c["new_hi"], window=c["window"],
                                 sinks=c["sinks"])


def own_write(st):
    c = st["case"]
    st["cache"].resize(st["seqs"], st["want"])
    if c["new_hi"] == 1:
        st["cache"].write(st["k"], st["v"], st["seqs"])
    else:
        st["cache"].write(st["k"], st["v"], st["seqs"], st["starts"])


def own_beam(st):
    st["cache"].resize(st["kids"], st["zeros"])
    st["cache"].fork(st["parents"], st["kids"])


def own_compact(st):
    c = st["case"]
    st["cache"].resize(st["ended"], st["zeros"])
    st["cache"].trim(st["kept"], c["sinks"], c["window"])
    st["cache"].compact()


# --------------------------------------------------------------------------- #
# plain forms
# --------------------------------------------------------------------------- #
def unpack(kv, is_v, D):
    """Tiles of 16 tokens in stored order [..., 16 * D] -> [..., 16, D]."""
    lead = kv.shape[:-1]
    n = len(lead)
    if is_v:    # [D / 32][8 dim groups][4 token groups][4 dims][4 tokens]
        x = kv.reshape(*lead, D // 32, 8, 4, 4, 4).permute(*range(n), n + 2, n + 4, n + 1, n, n + 3)
    else:       # [2 token halves][D / 64][4 token groups][2 tokens][4 dim groups][16 dims]
        x = kv.reshape(*lead, 2, D // 64, 4, 2, 4, 16).permute(*range(n), n + 2, n, n + 3, n + 4, n + 1, n + 5)
    return x.reshape(*lead, BLOCK, D)


def pack(x, is_v):
    lead, D = x.shape[:-2], x.shape[-1]
    n = len(lead)
    if is_v:
        y = x.reshape(*lead, 4, 4, 8, D // 32, 4).permute(*range(n), n + 3, n + 2, n, n + 4, n + 1)
    else:
        y = x.reshape(*lead, 4, 2, 2, 4, D // 64, 16).permute(*range(n), n + 1, n + 4, n, n + 2, n + 3, n + 5)
    return y.reshape(*lead, BLOCK * D)


def decode(codes, fmt):
    return codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()


def encode(x, fmt):
    if fmt == "int8":
        return x.round().to(torch.int8).view(torch.uint8)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def plain_attention(st):
    c = st["case"]
    pt, D, H, G, n = c["page"], c["dim"], c["heads"], c["group"], c["n"]
    q, starts = st["q"], st["starts"].long()
    rows = st["table"][st["seqs"].long()].long()                          # [n, P]
    lens = st["lens"][st["seqs"].long()].long()
    new = starts[1:] - starts[:-1]
    most, P = c["new_hi"], rows.shape[1]
    at = rows.clamp(min=0)
    tiles = st["codes"][:, at].reshape(-1, n, P, H, 2, pt // BLOCK, BLOCK * D)
    scale = st["amax"][:, at] / TOP[c["fmt"]]                             # [L, n, P, H, 2, pt / 16]
    order = lambda x: x.permute(0, 1, 3, 2, 4, 5, 6).reshape(-1, n, H, P * pt, D)  # noqa: E731
    k = order(unpack(decode(tiles[:, :, :, :, 0], c["fmt"]), False, D) * scale[:, :, :, :, 0, :, None, None])
    v = order(unpack(decode(tiles[:, :, :, :, 1], c["fmt"]), True, D) * scale[:, :, :, :, 1, :, None, None])
    i = torch.arange(most, device=q.device)
    here = i < new[:, None]                                               # [n, most]
    src = (starts[:-1, None] + i).clamp(max=max(0, q.shape[0] - 1))
    qp = q[src].float().reshape(n, most, -1, H, G, D).permute(2, 0, 3, 4, 1, 5).reshape(-1, n, H, G * most, D)
    s = torch.matmul(qp, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    pos = (lens - new)[:, None] + i                                       # [n, most]
    j = torch.arange(P * pt, device=q.device)
    seen = (j <= pos[..., None]) & (j < lens[:, None, None]) & (rows >= 0).repeat_interleave(pt, 1)[:, None]
    if c["window"]:
        seen &= (j > pos[..., None] - c["window"]) | (j < c["sinks"])
    s = s.reshape(-1, n, H, G, most, P * pt).masked_fill_(~seen[None, :, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, torch.zeros_like(m)))
    del s
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(-1, n, H, G * most, P * pt), v).reshape(-1, n, H, G, most, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    o = o.permute(1, 4, 0, 2, 3, 5).reshape(n, most, -1, H * G, D)        # [n, most, L, heads, D]
    return o[here].to(q.dtype)


def plain_resize(st, seqs, want):
    """Pages behind the new ends go, then the missing ones come: the lowest free ones, in the order of the list. A
    sequence that grows inside a page that others hold too gets a copy of that page."""
    pt, table, lens, refs = st["case"]["page"], st["table"], st["lens"], st["refs"]
    at = seqs.long()
    rows, old, want = table[at].long(), lens[at].long(), want.long()
    ordinal = torch.arange(table.shape[1], device=table.device)
    need = (want + pt - 1) // pt
    drop = (ordinal >= need[:, None]) & (rows >= 0)
    refs.index_add_(0, rows.clamp(min=0).flatten(), -drop.flatten().int())
    rows = torch.where(drop, -1, rows)
    last = (old // pt).clamp(max=table.shape[1] - 1)
    held = rows.gather(1, last[:, None])[:, 0]
    split = (want > old) & (old % pt > 0) & (held >= 0) & (refs[held.clamp(min=0)] > 1)
    first = torch.where(split, old // pt, (old + pt - 1) // pt)
    grow = (ordinal >= first[:, None]) & (ordinal < need[:, None])
    free = torch.nonzero(refs == 0)[:, 0]
    number = grow.flatten().cumsum(0).reshape(grow.shape) - 1
    rows = torch.where(grow, free[number.clamp(min=0, max=free.shape[0] - 1)], rows)
    refs[rows[grow]] = 1
    refs.index_add_(0, held[split], -torch.ones_like(held[split]).int())
    copies = rows.gather(1, last[:, None])[:, 0]
    st["codes"][:, copies[split]] = st["codes"][:, held[split]]
    st["amax"][:, copies[split]] = st["amax"][:, held[split]]
    table[at] = rows.int()
    lens[at] = want.int()


def plain_write(st):
    """The last new tokens of every sequence, block by block: a block's magnitude is the largest of its values (what
    it held before among them); older codes are rounded again where it has grown."""
    plain_resize(st, st["seqs"], st["want"])
    c = st["case"]
    pt, D, H, fmt, n = c["page"], c["dim"], c["heads"], c["fmt"], c["n"]
    top = TOP[fmt]
    at, starts = st["seqs"].long(), st["starts"].long()
    lens, new = st["lens"][at].long(), starts[1:] - starts[:-1]
    first = (lens - new) // BLOCK
    blocks = (c["new_hi"] + BLOCK - 2) // BLOCK + 1
    b = first[:, None] + torch.arange(blocks, device=at.device)           # [n, blocks]
    i, o = torch.nonzero((b * BLOCK < lens[:, None]) & (new > 0)[:, None], as_tuple=True)
    b = b[i, o]                                                           # the blocks that are written
    page = st["table"][at[i], b * BLOCK // pt].long()
    inner = b % (pt // BLOCK)
    pos = (b * BLOCK)[:, None] + torch.arange(BLOCK, device=at.device)    # [m, 16]
    begin = (lens - new)[i][:, None]
    fresh = ((pos >= begin) & (pos < lens[i][:, None]))[:, None, None, :, None]
    older = (pos < begin)[:, None, None, :, None]
    src = (starts[:-1][i][:, None] + pos - begin).clamp(min=0, max=max(0, st["k"].shape[0] - 1))
    for which, x in ((0, st["k"]), (1, st["v"])):
        tiles = st["codes"].view(c["layers"], -1, H, 2, pt // BLOCK, BLOCK * D)
        was = unpack(decode(tiles[:, page, :, which, inner], fmt), which == 1, D)   # [m, layers, H, 16, D]
        mag = st["amax"][:, page, :, which, inner][..., None, None]
        val = x[src].float().permute(0, 2, 3, 1, 4)                       # [m, layers, H, 16, D]
        val = torch.where(fresh, val, torch.zeros_like(val))
        mag = torch.where(older.any(3, keepdim=True), mag, torch.zeros_like(mag))
        now = torch.maximum(mag, val.abs().amax((-1, -2), keepdim=True))
        some = torch.where(now > 0, now, torch.ones_like(now))
        code = torch.where(older, was * mag / some, val * top / some)
        tiles[:, page, :, which, inner] = pack(encode(code, fmt), which == 1)
        st["amax"][:, page, :, which, inner] = now[..., 0, 0]


def plain_fork(st, src, dst):
    """Whole pages are shared, the page that is still being filled is copied: to the lowest free pages, in order."""
    pt, table, lens, refs = st["case"]["page"], st["table"], st["lens"], st["refs"]
    src, dst = src.long(), dst.long()
    rows, length = table[src].long(), lens[src].long()
    ordinal = torch.arange(table.shape[1], device=table.device)
    last = (length // pt).clamp(max=table.shape[1] - 1)
    held = rows.gather(1, last[:, None])[:, 0]
    part = (length % pt > 0) & (held >= 0)
    free = torch.nonzero(refs == 0)[:, 0]
    number = part.cumsum(0) - 1
    fresh = free[number.clamp(min=0, max=free.shape[0] - 1)]
    shared = (ordinal < (length // pt)[:, None]) & (rows >= 0)
    refs.index_add_(0, rows.clamp(min=0).flatten(), shared.flatten().int())
    refs[fresh[part]] = 1
    rows = torch.where((ordinal == last[:, None]) & part[:, None], fresh[:, None], rows)
    st["codes"][:, fresh[part]] = st["codes"][:, held[part]]
    st["amax"][:, fresh[part]] = st["amax"][:, held[part]]
    table[dst] = rows.int()
    lens[dst] = length.int()


def plain_beam(st):
    plain_resize(st, st["kids"], st["zeros"])
    plain_fork(st, st["parents"], st["kids"])


def plain_trim(st, seqs, sinks, window):
    """Pages that hold neither one of the first `sinks` tokens nor one of the last `window` go."""
    pt, table, refs, at = st["case"]["page"], st["table"], st["refs"], seqs.long()
    rows, lens = table[at].long(), st["lens"][at].long()
    begin = torch.arange(table.shape[1], device=table.device) * pt
    drop = (begin >= sinks) & (begin + pt <= (lens - window)[:, None]) & (rows >= 0)
    refs.index_add_(0, rows.clamp(min=0).flatten(), -drop.flatten().int())
    table[at] = torch.where(drop, -1, rows).int()


def plain_compact(st):
    """The pages in use move down into the free ones, in order, until they are the first ones of the pool."""
    c, table, refs = st["case"], st["table"], st["refs"]
    plain_resize(st, st["ended"], st["zeros"])
    plain_trim(st, st["kept"], c["sinks"], c["window"])
    used = (refs > 0)
    index = torch.arange(refs.shape[0], device=refs.device)
    live = used.sum()
    src, dst = index[used & (index >= live)], index[~used & (index < live)]
    to = index.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    st["codes"][:, dst] = st["codes"][:, src]
    st["amax"][:, dst] = st["amax"][:, src]
    refs[dst] = refs[src]
    refs[src] = 0


# --------------------------------------------------------------------------- #
# the work that a pass cannot do without
# --------------------------------------------------------------------------- #
def _pairs(case, begin, end):
    """Key / query pairs of the queries at positions [begin, end), and the keys that any of them sees."""
    w, s = case["window"], case["sinks"]
    if not w:
        return (begin + 1 + end) * (end - begin) // 2, end
    pairs = sum(min(i + 1, w) + min(s, max(0, i + 1 - w)) for i in range(begin, end))
    low = max(0, begin + 1 - w)
    return pairs, end - low + min(s, low)


def work(case):
    s = _shape(case)
    pt, D, L, H, G = case["page"], case["dim"], case["layers"], case["heads"], case["group"]
    row = 2 * H * D + 2 * H * 4 / BLOCK                 # bytes of a token's keys and values in one layer
    if case["op"] == "attention":
        pairs = keys = 0
        for a, b in zip(s["want"], s["new"]):
            p, k = _pairs(case, a - b, a)
            pairs, keys = pairs + p, keys + k
        return {"bytes": L * (keys * row + 2 * 2 * sum(s["new"]) * H * G * D), "flops": 4.0 * D * pairs * H * G * L}
    if case["op"] == "write":
        n = sum(s["new"])
        return {"bytes": L * n * (2 * 2 * H * D + row), "flops": 4.0 * L * n * 2 * H * D}
    maps = 4.0 * (len(s["refs"]) + sum(len(r) for r in s["table"]))
    if case["op"] == "beam":
        part = sum(case["children"] * (a % pt) for a in s["want"])
        return {"bytes": 2.0 * L * part * row + maps, "flops": 0.0}
    for i, r in enumerate(s["rows"]):
        for p, page in enumerate(s["table"][r]):
            gone = i < case["done"] or (p * pt >= case["sinks"] and (p + 1) * pt <= s["lens"][r] - case["window"])
            if page >= 0 and gone:
                s["refs"][page] -= 1
    live = sum(x > 0 for x in s["refs"])
    return {"bytes": 2.0 * L * sum(x > 0 for x in s["refs"][live:]) * pt * row + maps, "flops": 0.0}


# --------------------------------------------------------------------------- #
# the definitions in 64 bits
# --------------------------------------------------------------------------- #
def _places(D):
    """Byte of (token, dimension) in a tile of 16 tokens: of the keys, and of the values."""
    r, d = torch.meshgrid(torch.arange(BLOCK), torch.arange(D), indexing="ij")
    lane = 2 * (r // 4) + r % 2
    kx = d % (D // 4)
    k = ((((r // 2 % 2) * (D // 64) + kx // 16) * 8 + lane) * 4 + d // (D // 4)) * 16 + kx % 16
    vx = d % (D // 8)
    v = ((vx // 4 * 8 + d // (D // 8)) * 4 + r // 4) * 16 + vx % 4 * 4 + r % 4
    return k.cuda(), v.cuda()


def _values(b, fmt):
    """What the 256 codes stand for, in units of amax / TOP."""
    if fmt == "int8":
        t = [float(x - 256 if x > 127 else x) for x in range(256)]
    else:
        t = []
        for x in range(256):
            e, m = x >> 3 & 15, x & 7
            y = math.nan if x & 127 == 127 else (m / 512.0 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7))
            t.append(-y if x & 128 else y)
    return torch.tensor(t, dtype=torch.float64, device="cuda")[b.long()]


def _codes(x, fmt):
    """The nearest code, ties to even, of a value in units of amax / TOP."""
    if fmt == "int8":
        return torch.remainder(torch.round(x), 256).to(torch.uint8)
    table = _values(torch.arange(127, device="cuda"), fmt)                # ascending
    mag = x.abs()
    up = torch.searchsorted(table, mag.contiguous()).clamp(max=126)
    low = (up - 1).clamp(min=0)
    a, b = mag - table[low], table[up] - mag
    code = torch.where((a < b) | ((a == b) & (low % 2 == 0)), low, up)
    return (code + 128 * torch.signbit(x)).to(torch.uint8)


def _exact_attention(case, st):
    pt, D, H, G, fmt = case["page"], case["dim"], case["heads"], case["group"], case["fmt"]
    places = _places(D)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    starts, lens, seqs = st["starts"].tolist(), st["lens"].tolist(), st["seqs"].tolist()
    for s, seq in enumerate(seqs):
        n, m = lens[seq], starts[s + 1] - starts[s]
        if not n or not m:
            continue
        j = torch.arange(n, device="cuda")
        page = st["table"][seq].long()[j // pt]
        for layer in range(case["layers"]):
            for h in range(H):
                kv = []
                for which in (0, 1):
                    inner = (j % pt // BLOCK)
                    byte = inner[:, None] * BLOCK * D + places[which][j % BLOCK]
                    val = _values(st["codes"][layer, page[:, None], h, which, byte], fmt)
                    kv.append(val * (st["amax"][layer, page, h, which, inner].double() / TOP[fmt])[:, None])
                step = max(1, (1 << 27) // (n * G))
                for a in range(0, m, step):
                    rows = torch.arange(a, min(m, a + step), device="cuda")
                    q = st["q"][starts[s] + rows, layer, h * G:(h + 1) * G].double()          # [r, G, D]
                    z = (q.reshape(-1, D) @ kv[0].T / math.sqrt(D)).reshape(len(rows), G, n)
                    i = (n - m + rows)[:, None, None]
                    hide = (j > i) | ((j <= i - case["window"]) & (j >= case["sinks"]) & (case["window"] > 0))
                    p = torch.softmax(z.masked_fill(hide, -math.inf), -1)
                    out[starts[s] + rows, layer, h * G:(h + 1) * G] = (p.reshape(-1, n) @ kv[1]).reshape(len(rows), G, D)
    return out


def _resize(maps, pt, rows, want):
    table, lens, refs = maps
    for r, w in zip(rows, want):
        for p in range(-(-w // pt), len(table[r])):
            if table[r][p] >= 0:
                refs[table[r][p]] -= 1
                table[r][p] = -1
    free = iter([p for p, x in enumerate(refs) if x == 0])
    for r, w in zip(rows, want):
        for p in range(-(-lens[r] // pt), -(-w // pt)):
            table[r][p] = next(free)
            refs[table[r][p]] = 1
        lens[r] = w


def _exact_write(case, st, maps):
    pt, D, H, fmt = case["page"], case["dim"], case["heads"], case["fmt"]
    places, top = _places(D), TOP[fmt]
    codes, amax = st["codes"].clone(), st["amax"].double()
    starts, seqs, want = st["starts"].tolist(), st["seqs"].tolist(), st["want"].tolist()
    _resize(maps, pt, seqs, want)
    for s, seq in enumerate(seqs):
        m, n = starts[s + 1] - starts[s], want[s]
        if not m:
            continue
        first, last = (n - m) // BLOCK, -(-n // BLOCK)
        block = torch.arange(first, last, device="cuda")
        page = torch.tensor(maps[0][seq], device="cuda")[block * BLOCK // pt]
        inner = block % (pt // BLOCK)
        keep = n - m - first * BLOCK                                       # older tokens of the first block
        for layer in range(case["layers"]):
            for which, x in ((0, st["k"]), (1, st["v"])):
                val = torch.zeros(((last - first) * BLOCK, H, D), dtype=torch.float64, device="cuda")
                val[keep:keep + m] = x[starts[s]:starts[s + 1], layer].double()
                val = val.reshape(-1, BLOCK, H, D).transpose(1, 2)          # [blocks, H, 16, D]
                mag = val.abs().amax((2, 3))
                if keep:
                    mag[0] = torch.maximum(mag[0], amax[layer, page[0], :, which, inner[0]])
                unit = torch.where(mag > 0, mag, 1.0)[:, :, None, None]
                new = _codes(val * top / unit, fmt)
                if keep:
                    byte = inner[0] * BLOCK * D + places[which][:keep]
                    was = _values(codes[layer, page[0], :, which][:, byte], fmt)            # [H, keep, D]
                    old = amax[layer, page[0], :, which, inner[0]][:, None, None]
                    new[0, :, :keep] = _codes(was * old / unit[0], fmt)
                byte = inner[:, None, None] * BLOCK * D + places[which]     # [blocks, 16, D]
                for h in range(H):
                    codes[layer, page[:, None, None], h, which, byte] = new[:, h]
                    amax[layer, page, h, which, inner] = mag[:, h]
    return codes, amax


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, st)
    pt = case["page"]
    maps = [st[k].tolist() for k in ("table", "lens", "refs")]
    table, lens, refs = maps
    codes, amax = st["codes"], st["amax"].double()
    if case["op"] == "write":
        codes, amax = _exact_write(case, st, maps)
    elif case["op"] == "beam":
        kids = st["kids"].tolist()
        _resize(maps, pt, kids, [0] * len(kids))
        free = iter([p for p, x in enumerate(refs) if x == 0])
        for a, b in zip(st["parents"].tolist(), kids):
            lens[b] = lens[a]
            table[b] = list(table[a])
            for p in range(lens[a] // pt):
                refs[table[a][p]] += 1
            if lens[a] % pt:
                p = lens[a] // pt
                table[b][p] = next(free)
                codes[:, table[b][p]] = codes[:, table[a][p]]
                amax[:, table[b][p]] = amax[:, table[a][p]]
        for p in {x for row in table for x in row if x >= 0}:
            refs[p] = sum(row.count(p) for row in table)
    else:
        _resize(maps, pt, st["ended"].tolist(), [0] * case["done"])
        for r in st["kept"].tolist():
            for p, page in enumerate(table[r]):
                if page >= 0 and p * pt >= case["sinks"] and (p + 1) * pt <= lens[r] - case["window"]:
                    refs[page] -= 1
                    table[r][p] = -1
        live = sum(x > 0 for x in refs)
        holes = [p for p in range(live) if refs[p] == 0]
        to = dict(zip([p for p in range(live, len(refs)) if refs[p] > 0], holes))
        for a, b in to.items():
            codes[:, b], amax[:, b] = codes[:, a].clone(), amax[:, a].clone()
            refs[b], refs[a] = refs[a], 0
        maps[0] = [[to.get(p, p) for p in row] for row in table]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"table": ints(maps[0]), "lens": ints(maps[1]), "refs": ints(maps[2]), "codes": codes, "amax": amax}
