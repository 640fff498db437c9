"""Cases of beam search and of many continuations of one text: the selection over beams and vocabulary, the
reordering that it asks of the two caches (LESS's own state, the paged 8-bit cache), and attention over the paged
cache for sequences that share their first pages.

Selection: logits [groups, beams, vocab], running scores fp32 [groups, beams] (-inf = no such beam); a candidate is
    value(beam, token) = score + logit - log sum exp logit         NaN counts as -inf, +inf as the largest finite value
    value(beam, end token) = score, nothing else                   for a beam that has ended
and the `keep` largest finite values of a group, ties to the lowest (beam, token), give its next beams: score, token,
row of the parent in [groups * beams], and whether it has ended.  Where candidates run out: -inf, -1, the row in the
same place, false.

Reordering: row (or sequence) i becomes what row parents[i] was.  In the paged cache whole pages are shared; of the
children of a sequence one takes over the page that is still being filled (the sequence itself if it is its own child,
else the first of the list), the others get copies of its 16-token blocks in use, in the lowest free pages, in order.

Buffers of the paged cache, all on the device (see `unpack` for the order of a tile):
    codes  uint8  [layers, pages, heads, 2 (K, V), page * D]      value = code * amax / 127 (int8) or / 448 (e4m3)
    amax   fp32   [layers, pages, heads, 2, page / 16]
    table  int32  [seqs, seq_pages]   lens   int32  [seqs]   refs   int32  [pages]

Shapes, lengths, page numbers and parents follow from the case, what the buffers hold from the seed.
"""
import math
import random

import torch

own = False

BLOCK = 16
TOP = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


# --------------------------------------------------------------------------- #
# the cases
# --------------------------------------------------------------------------- #
def select(name, groups, beams, vocab, keep=0, dtype="fp16", alive=0, ended=0, pad=0):
    """alive: beams of a group that exist (0 = all); ended: every how manieth beam has ended (0 = none); pad: elements
    between the rows of the logits."""
    c = {"op": "select", "groups": groups, "beams": beams, "vocab": vocab, "keep": keep or beams, "dtype": dtype,
         "alive": alive, "ended": ended, "pad": pad}
    return dict(c, name=name) if name else c


def state(name, groups, beams, layers, heads, slots, rank=8, dim=128):
    c = {"op": "state", "groups": groups, "beams": beams, "layers": layers, "heads": heads, "slots": slots,
         "rank": rank, "dim": dim}
    return dict(c, name=name) if name else c


def reorder(name, groups, beams, lo, hi, layers, heads, dim, page=64, fmt="int8"):
    c = {"op": "reorder", "groups": groups, "beams": beams, "len_lo": lo, "len_hi": hi, "layers": layers,
         "heads": heads, "group": 1, "dim": dim, "page": page, "dtype": "fp16", "fmt": fmt}
    return dict(c, name=name) if name else c


def shared(name, groups, each_lo, each_hi, pre_lo, pre_hi, own_lo, own_hi, heads, group, dim, new=1, page=64,
           dtype="bf16", fmt="int8", window=0, sinks=0):
    """each: sequences of a group; pre: tokens they have in common; own: tokens of their own; new: new ones, 1 to
    `new` per sequence."""
    c = {"op": "shared", "groups": groups, "each_lo": each_lo, "each_hi": each_hi, "pre_lo": pre_lo, "pre_hi": pre_hi,
         "own_lo": own_lo, "own_hi": own_hi, "new": new, "layers": 1, "heads": heads, "group": group, "dim": dim,
         "page": page, "dtype": dtype, "fmt": fmt, "window": window, "sinks": sinks}
    return dict(c, name=name) if name else c


def listed():
    return [
        # four beams of one text: what counts is latency
        select("select_small", 1, 4, 32000),
        # the first step of a batch: of the beams of a text only one exists; an odd vocabulary
        select("select_first", 16, 8, 50257, dtype="fp32", alive=1),
        # a full batch in the midst of its search, candidates for two beams each, some beams have ended
        select("select_large", 64, 8, 128256, keep=16, dtype="bf16", ended=11),
        # LESS's state of four beams, one layer
        state("state_small", 1, 4, 1, 8, 64),
        # of eight texts with eight beams, eight layers of 32 heads
        state("state_large", 8, 8, 8, 32, 204),
        # four beams of one text in the paged cache, one layer
        reorder("reorder_small", 1, 4, 250, 250, 1, 8, 128),
        # 64 texts with eight beams, eight layers
        reorder("reorder_large", 64, 8, 100, 1000, 8, 8, 128),
        # four beams of a short text: what counts is latency
        shared("shared_small", 1, 4, 4, 256, 256, 10, 10, 8, 1, 128, dtype="fp16"),
        # a batch of beam searches over texts between short and long, four query heads per KV head
        shared("shared_beams", 16, 4, 4, 100, 3000, 1, 70, 8, 4, 128),
        # conversations behind one long instruction, a query head per KV head
        shared("shared_prompt", 1, 64, 64, 4096, 4096, 1, 1000, 32, 1, 128, dtype="fp16"),
        # answers to questions about one long document
        shared("shared_long", 1, 16, 16, 100003, 100003, 1, 300, 8, 8, 128, fmt="e4m3"),
        # drafted tokens, first tokens and a window, the multi-query shape
        shared("shared_draft", 6, 1, 8, 200, 4000, 1, 200, 1, 71, 64, new=4, page=32, dtype="fp16", window=1024,
               sinks=4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["select", "select", "state", "reorder", "shared", "shared", "shared"])
    dim = rng.choice([128, 128, 64])
    page = rng.choice([16, 32, 64, 128])
    fmt = rng.choice(["int8", "e4m3"])
    if op == "select":
        groups, beams = _log(rng, 1, 64), rng.choice([1, 2, 3, 4, 5, 8, 16])
        dtype = rng.choice(["fp16", "bf16", "fp32"])
        vocab = _log(rng, 500, min(160000, (32_000_000 if dtype == "fp32" else 64_000_000) // (groups * beams)))
        return select("", groups, beams, vocab, rng.choice([beams, 2 * beams, 2 * beams + 1]), dtype,
                      rng.choice([0, 0, 0, 1]), rng.choice([0, 0, 3, 7]), rng.choice([0, 0, 1, 24]))
    if op == "state":
        groups, beams = _log(rng, 1, 16), rng.choice([2, 3, 4, 5, 8])
        layers, heads = _log(rng, 1, 16), rng.choice([1, 2, 3, 8, 32])
        most = 400_000_000 // (groups * beams * layers * heads * dim)
        return state("", groups, beams, layers, heads, _log(rng, 5, max(8, min(1000, most))), rng.choice([8, 16]), dim)
    if op == "reorder":
        groups, beams = _log(rng, 1, 64), rng.choice([2, 3, 4, 5, 8, 16])
        hi = _log(rng, 20, 1000)
        return reorder("", groups, beams, rng.randint(1, hi), hi, rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 8]),
                       dim, page, fmt)
    dtype = rng.choice(["fp16", "bf16"])
    heads = rng.choice([1, 2, 3, 8, 8, 32])
    group = rng.choice([1, 2, 4, 5, 8]) if heads > 1 else rng.choice([1, 8, 16, 71])
    groups = _log(rng, 1, 16)
    each = _log(rng, 2, 96 // groups)
    new = rng.choice([1, 1, 1, 2, 5])
    most = 600_000_000 // (groups * each * heads * dim)
    tail = max(new, _log(rng, 1, max(2, min(2000, most // 4))))
    pre = _log(rng, 16, max(20, min(120000, most - tail)))
    window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 100, 4000), rng.choice([0, 4, 17]))])
    return shared("", groups, rng.randint(1, each), each, rng.randint(1, pre), pre, rng.randint(1, tail), tail, heads,
                  group, dim, new, page, dtype, fmt, window, sinks)


def _spread(lo, hi, n):
    """n whole numbers over [lo, hi], hi first, lo last."""
    v = [lo + int((hi - lo + 1) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]
    v[-1] = lo
    v[0] = hi
    return v


def _parents(groups, beams):
    """What a step of the search chose: of a group some beams die, some have two or three children."""
    rnd = random.Random(11)
    out = []
    for g in range(groups):
        out += [g * beams + min(rnd.randrange(beams), rnd.randrange(beams)) for _ in range(beams)]
    return out


def _shape(case):
    """Lengths and page table of a case in the paged cache: what a scheduler has in hand."""
    pt, rnd = case["page"], random.Random(7)
    sizes = []                                          # per group: sequences, tokens in common, their own, new ones
    if case["op"] == "reorder":                         # beams part some tokens before the end
        for n in _spread(case["len_lo"], case["len_hi"], case["groups"]):
            pre = max(0, n - 1 - rnd.randrange(3 * pt // 2))
            sizes.append((pre, [n - pre] * case["beams"], [1] * case["beams"]))
        moved = case["groups"] * case["beams"]
    else:
        each = _spread(case["each_lo"], case["each_hi"], case["groups"])
        pres = _spread(case["pre_lo"], case["pre_hi"], case["groups"])
        tails, news = _spread(case["own_lo"], case["own_hi"], sum(each)), _spread(1, case["new"], sum(each))
        at = 0
        for k, pre in zip(each, pres):
            sizes.append((pre, [max(a, b) for a, b in zip(tails[at:at + k], news[at:at + k])], news[at:at + k]))
            at += k
        moved = 0
    total = sum(len(t) for _, t, _ in sizes)
    seqs = total + 2                                    # two sequences of the table are not in use
    rows = list(range(seqs))
    rnd.shuffle(rows)
    room = max(-(-(pre + max(t)) // pt) for pre, t, _ in sizes)
    used = sum(pre // pt + sum(-(-(pre + x) // pt) - pre // pt for x in t) for pre, t, _ in sizes)
    ids = list(range(used + moved + 3))
    rnd.shuffle(ids)
    take = iter(ids)
    table = [[-1] * room for _ in range(seqs)]
    lens, refs, groups, new = [0] * seqs, [0] * len(ids), [0], []
    at = 0
    for pre, tails, news in sizes:
        common = [next(take) for _ in range(pre // pt)]
        for x in tails:
            pages = common + [next(take) for _ in range(-(-(pre + x) // pt) - pre // pt)]
            table[rows[at]][:len(pages)] = pages
            lens[rows[at]] = pre + x
            for p in pages:
                refs[p] += 1
            at += 1
        groups.append(at)
        new += news
    return {"table": table, "lens": lens, "refs": refs, "rows": rows[:total], "groups": groups, "new": new,
            "pages": len(ids), "seqs": seqs, "room": room,
            "most": max(sum(new[a:b]) for a, b in zip(groups, groups[1:])), "pres": [pre // pt * pt for pre, _, _ in sizes]}


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


def _prepare_select(case, g):
    G, B, V = case["groups"], case["beams"], case["vocab"]
    dtype = DTYPE[case["dtype"]]
    rows = torch.empty((G, B, V + case["pad"]), dtype=dtype, device="cuda")
    for i in range(G):                                  # logits of a language model: a broad body, a few that stand out
        x = torch.randn((B, V + case["pad"]), generator=g, device="cuda") * 2.0
        x += 6.0 * torch.rand(x.shape, generator=g, device="cuda").pow_(24)
        x[torch.rand(x.shape, generator=g, device="cuda") < 0.01] = -math.inf          # tokens that are not allowed
        rows[i] = x.to(dtype)
    scores = -60.0 * torch.rand((G, B), generator=g, device="cuda") - 1.0
    scores = scores.sort(-1, descending=True).values * 0.1
    if case["alive"]:
        scores[:, case["alive"]:] = -math.inf
    at = torch.arange(G * B, device="cuda").reshape(G, B)
    ended = at % case["ended"] == case["ended"] - 1 if case["ended"] else None
    st = {"case": case, "logits": rows[:, :, :V], "scores": scores, "ended": ended, "end": V // 3}
    if own:
        from paper_2402_09398_b200 import binding
        st["select"] = binding.BeamSelect(G, B, V, keep=case["keep"], dtype=dtype, end_token=st["end"])
    return st


def _prepare_state(case, g):
    B, L, H, N = case["groups"] * case["beams"], case["layers"], case["heads"], case["slots"]
    R, D = case["rank"], case["dim"]
    st = {"case": case, "parents": torch.tensor(_parents(case["groups"], case["beams"]), dtype=torch.int32,
                                                device="cuda")}
    if own:
        from paper_2402_09398_b200 import binding
        shapes = {"w_phi1": (L, H, D, 64), "w_phi2": (L, H, 64, R), "w_psi1": (L, H, D, 64), "w_psi2": (L, H, 64, R),
                  "w_psi3": (L, H, R, R)}
        weights = {k: torch.randn(s, generator=g, device="cuda").mul_(0.02).half() for k, s in shapes.items()}
        st["context"] = binding.LessContext(B, L, H, D, R, 64, N // 2, N - N // 2, 0, weights)
        st["state"] = st["context"].state_tensors()
        g.manual_seed(g.initial_seed())                 # the state does not depend on the weights
    else:
        f32 = lambda *s: torch.empty(s, dtype=torch.float32, device="cuda")  # noqa: E731
        st["state"] = {"K": f32(B, L, H, N, D).half(), "V": f32(B, L, H, N, D).half(),
                       "pos": f32(B, L, H, N).int(), "acc": f32(B, L, H, N), "psi": f32(B, L, H, N, R),
                       "H": f32(B, L, H, R, D), "z": f32(B, L, H, R), "count": f32(B, L, H).int()}
    for k in ("K", "V", "acc", "psi", "H", "z", "pos", "count"):
        for b in range(B):
            t = st["state"][k][b]
            if k == "pos":
                step = torch.randint(1, 9, t.shape, generator=g, device="cuda", dtype=torch.int32)
                t.copy_(step.cumsum(-1))
            elif k == "count":
                t.fill_(N)
            else:
                x = torch.randn(t.shape, generator=g, device="cuda")
                t.copy_(x if k in "KV" else x.abs())
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] == "select":
        return _prepare_select(case, g)
    if case["op"] == "state":
        return _prepare_state(case, g)
    s = _shape(case)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    L, H, D = case["layers"], case["heads"], case["dim"]
    codes, amax = _fill(case, s, g)
    st = {"case": case, "codes": codes, "amax": amax, "table": ints(s["table"]), "lens": ints(s["lens"]),
          "refs": ints(s["refs"]), "seqs": ints(s["rows"])}
    if case["op"] == "reorder":
        st["parents"] = ints(_parents(case["groups"], case["beams"]))
    else:
        starts = [0]
        for x in s["new"]:
            starts.append(starts[-1] + x)
        st["starts"], st["groups"], st["most"] = ints(starts), ints(s["groups"]), s["most"]
        shape = (starts[-1], L, H * case["group"], D)
        st["q"] = torch.randn(shape, generator=g, device="cuda").to(DTYPE[case["dtype"]])
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
    if op == "select":
        return (own_select if own else plain_select)(state)
    if op == "shared":
        return (own_shared if own else plain_shared)(state)
    if op == "state":
        (own_state if own else plain_state)(state)
        return dict(state["state"])
    (own_reorder if own else plain_reorder)(state)
    return {k: state[k] for k in ("table", "lens", "refs", "codes", "amax")}


def own_select(st):
    c = st["select"].select(st["logits"], st["scores"], st["ended"])
    return {"scores": c.scores, "tokens": c.tokens, "parents": c.parents, "ended": c.ended}


def own_state(st):
    st["context"].reorder(st["parents"], beams=st["case"]["beams"])


def own_reorder(st):
    st["cache"].reorder(st["seqs"], st["parents"])


def own_shared(st):
    c = st["case"]
    return st["cache"].shared_attention(st["q"], st["seqs"], st["groups"], None if c["new"] == 1 else st["starts"],
                                        max_new=c["new"], max_group=st["most"], window=c["window"], sinks=c["sinks"])


# --------------------------------------------------------------------------- #
# plain forms
# --------------------------------------------------------------------------- #
def plain_select(st):
    """In 64 bits: what decides is the order of values that may lie next to one another."""
    c, logits, scores, ended = st["case"], st["logits"], st["scores"], st["ended"]
    G, B, V = logits.shape
    x = logits.double()
    x = torch.where(torch.isnan(x), -math.inf, x).clamp(max=torch.finfo(logits.dtype).max)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    lse = torch.log(torch.exp(x - top).sum(-1, keepdim=True)) + top
    lse = torch.where(lse > -math.inf, lse, 0.0)
    x += scores.double()[..., None] - lse
    if ended is not None:
        x.masked_fill_(ended[..., None], -math.inf)
        x[:, :, st["end"]] = torch.where(ended, scores.double(), x[:, :, st["end"]])
    x = x.reshape(G, B * V)
    index = torch.arange(B * V, device=x.device)
    found = []
    for _ in range(c["keep"]):                          # the largest, at its lowest place, and without it again
        m = x.amax(-1, keepdim=True)
        at = torch.where(x == m, index, B * V).amin(-1, keepdim=True)
        found.append((m, at))
        x.scatter_(1, at, -math.inf)
    value, at = (torch.cat(t, 1) for t in zip(*found))
    beam, some = at // V, value > -math.inf
    row = torch.arange(G, device=x.device)[:, None] * B
    slot = torch.arange(c["keep"], device=x.device).clamp(max=B - 1)
    token = torch.where(some, at % V, -1)
    done = token == st["end"]
    return {"scores": value.float(), "tokens": token.int(), "parents": torch.where(some, row + beam, row + slot).int(),
            "ended": done}


def plain_state(st):
    at = st["parents"].long()
    for t in st["state"].values():
        t.copy_(t[at])


def unpack(kv, is_v, D):
    """Tiles of 16 tokens in stored order [..., 16 * D] -> [..., 16, D]."""
    lead = kv.shape[:-1]
    n = len(lead)
    if is_v:    # [D / 32][8 dim groups][4 token groups][4 dims][4 tokens]
        x = kv.reshape(*lead, D // 32, 8, 4, 4, 4).permute(*range(n), n + 2, n + 4, n + 1, n, n + 3)
    else:       # [2 token halves][D / 64][4 token groups][2 tokens][4 dim groups][16 dims]
        x = kv.reshape(*lead, 2, D // 64, 4, 2, 4, 16).permute(*range(n), n + 2, n, n + 3, n + 4, n + 1, n + 5)
    return x.reshape(*lead, BLOCK, D)


def decode(codes, fmt):
    return codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()


def plain_reorder(st):
    c, pt, table, lens, refs = st["case"], st["case"]["page"], st["table"], st["lens"], st["refs"]
    at, parents = st["seqs"].long(), st["parents"].long()
    n = at.shape[0]
    old = table[at].long()
    rows, length = old[parents], lens[at][parents].long()
    index = torch.arange(n, device=at.device)
    first = torch.full((n,), n, device=at.device).scatter_reduce_(0, parents, index, "amin")
    heir = torch.where(parents == index, index, first)[parents]           # the child that takes over the last page
    last = (length // pt).clamp(max=table.shape[1] - 1)
    held = rows.gather(1, last[:, None])[:, 0]
    copy = (length % pt > 0) & (held >= 0) & (heir != index)
    kept = torch.where(copy[:, None] & (torch.arange(table.shape[1], device=at.device) == last[:, None]), -1, rows)
    refs.index_add_(0, old.clamp(min=0).flatten(), -(old >= 0).flatten().int())
    refs.index_add_(0, kept.clamp(min=0).flatten(), (kept >= 0).flatten().int())
    free = torch.nonzero(refs == 0)[:, 0]
    number = (copy.cumsum(0) - 1).clamp(min=0, max=free.shape[0] - 1)
    rows[index[copy], last[copy]] = free[number[copy]]
    refs[free[number[copy]]] = 1
    tiles = st["codes"].view(c["layers"], -1, c["heads"], 2, pt // BLOCK, BLOCK * c["dim"])
    used = (length % pt + BLOCK - 1) // BLOCK
    which, tile = torch.nonzero(copy[:, None] & (torch.arange(pt // BLOCK, device=at.device) < used[:, None]),
                                as_tuple=True)
    to = rows.gather(1, last[:, None])[:, 0]
    tiles[:, to[which], :, :, tile] = tiles[:, held[which], :, :, tile]
    st["amax"][:, to[which], :, :, tile] = st["amax"][:, held[which], :, :, tile]
    table[at] = rows.int()
    lens[at] = length.int()


def plain_shared(st):
    """Every sequence over all its keys, a KV head at a time."""
    c = st["case"]
    pt, D, H, G, n = c["page"], c["dim"], c["heads"], c["group"], st["seqs"].shape[0]
    q, starts = st["q"], st["starts"].long()
    rows = st["table"][st["seqs"].long()].long()                          # [n, P]
    lens = st["lens"][st["seqs"].long()].long()
    new = starts[1:] - starts[:-1]
    most, P = c["new"], rows.shape[1]
    at = rows.clamp(min=0)
    i = torch.arange(most, device=q.device)
    here = i < new[:, None]                                               # [n, most]
    src = (starts[:-1, None] + i).clamp(max=max(0, q.shape[0] - 1))
    pos = (lens - new)[:, None] + i                                       # [n, most]
    j = torch.arange(P * pt, device=q.device)
    seen = (j <= pos[..., None]) & (j < lens[:, None, None]) & (rows >= 0).repeat_interleave(pt, 1)[:, None]
    if c["window"]:
        seen &= (j > pos[..., None] - c["window"]) | (j < c["sinks"])
    out = torch.empty((n, most, c["layers"], H, G, D), device=q.device)
    for layer in range(c["layers"]):
        for h in range(H):
            kv = []
            for w in (0, 1):
                tiles = decode(st["codes"][layer, at, h, w].reshape(n, P, pt // BLOCK, BLOCK * D), c["fmt"])
                scale = st["amax"][layer, at, h, w] / TOP[c["fmt"]]
                kv.append((unpack(tiles, w == 1, D) * scale[..., None, None]).reshape(n, P * pt, D))
            qh = q[src][:, :, layer, h * G:(h + 1) * G].float().reshape(n, most * G, D)
            s = torch.matmul(qh, kv[0].transpose(-1, -2)) * (1.0 / math.sqrt(D))
            s = s.reshape(n, most, G, P * pt).masked_fill_(~seen[:, :, None], -math.inf)
            m = s.amax(-1, keepdim=True)
            p = torch.exp(s - torch.where(m > -math.inf, m, torch.zeros_like(m)))
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p.reshape(n, most * G, P * pt), kv[1]).reshape(n, most, G, D)
            out[:, :, layer, h] = torch.where(total > 0, o / total, torch.zeros_like(o))
    return out.reshape(n, most, c["layers"], H * G, D)[here].to(q.dtype)


# --------------------------------------------------------------------------- #
# the work that a pass cannot do without
# --------------------------------------------------------------------------- #
def work(case):
    if case["op"] == "select":
        n = case["groups"] * case["beams"]
        rows = n if not case["alive"] else case["groups"] * min(case["alive"], case["beams"])
        if case["ended"]:
            rows -= sum(i % case["ended"] == case["ended"] - 1 and
                        (not case["alive"] or i % case["beams"] < case["alive"]) for i in range(n))
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": float(rows * case["vocab"] * size + 5 * n + 13 * case["groups"] * case["keep"]),
                "flops": 4.0 * rows * case["vocab"]}
    if case["op"] == "state":
        N, R, D = case["slots"], case["rank"], case["dim"]
        row = case["layers"] * case["heads"] * (N * (4 * D + 4 + 4 + 4 * R) + 4 * R * D + 4 * R + 4)
        parents = _parents(case["groups"], case["beams"])
        moved = [(p, i) for i, p in enumerate(parents) if p != i]
        return {"bytes": float(row * (len(moved) + len({p for p, _ in moved})) + 4 * len(parents)), "flops": 0.0}
    s = _shape(case)
    pt, D, L, H, G = case["page"], case["dim"], case["layers"], case["heads"], case["group"]
    row = 2 * H * D + 2 * H * 4 / BLOCK                 # bytes of a token's keys and values in one layer
    lens = [s["lens"][r] for r in s["rows"]]
    if case["op"] == "reorder":
        parents = _parents(case["groups"], case["beams"])
        counts = {}
        for p in parents:
            counts[p] = counts.get(p, 0) + 1
        once = sum(lens[p] % pt for p, k in counts.items() if k > 1)     # a page that is copied is read once
        often = sum((k - 1) * (lens[p] % pt) for p, k in counts.items() if k > 1)
        maps = 4.0 * sum(2 * -(-n // pt) for i, n in enumerate(lens) if parents[i] != i)
        return {"bytes": L * row * (once + often) + maps + 12.0 * len(lens), "flops": 0.0}
    w, first = case["window"], case["sinks"]
    pairs = keys = 0
    for g, (a, b) in enumerate(zip(s["groups"], s["groups"][1:])):
        low, lead = s["pres"][g], 0                      # of the pages in common: tokens from `low` on, first ones
        for i in range(a, b):
            begin, end = lens[i] - s["new"][i], lens[i]
            for t in range(begin, end):
                pairs += t + 1 if not w else min(t + 1, w) + min(first, max(0, t + 1 - w))
            lo = max(0, begin + 1 - w) if w else 0
            lead = max(lead, min(first, lo, s["pres"][g]))
            low = min(low, lo)
            keys += end - max(lo, s["pres"][g]) + max(0, min(first, lo) - s["pres"][g])
        keys += s["pres"][g] - low + min(lead, low)
    return {"bytes": L * (keys * row + 2 * 2 * sum(s["new"]) * H * G * D), "flops": 4.0 * D * pairs * H * G * L}


# --------------------------------------------------------------------------- #
# the definitions in 64 bits
# --------------------------------------------------------------------------- #
def _exact_select(case, st):
    """Group by group, by sorting every candidate."""
    G, B, V, keep = case["groups"], case["beams"], case["vocab"], case["keep"]
    most = torch.finfo(DTYPE[case["dtype"]]).max
    values, tokens, parents = [], [], []
    for i in range(G):
        z = torch.nan_to_num(st["logits"][i].double(), nan=-math.inf, posinf=most, neginf=-math.inf)
        v = st["scores"][i].double()[:, None] + torch.log_softmax(z, -1)
        v = torch.where(torch.isnan(v), -math.inf, v)
        if st["ended"] is not None:
            for b in range(B):
                if st["ended"][i, b]:
                    v[b] = -math.inf
                    v[b, st["end"]] = st["scores"][i, b].double()
        top, at = torch.sort(v.flatten(), descending=True, stable=True)
        top, at = top[:keep].tolist(), at[:keep].tolist()
        top += [-math.inf] * (keep - len(top))
        at += [0] * (keep - len(at))
        values.append(top)
        tokens.append([a % V if x > -math.inf else -1 for x, a in zip(top, at)])
        parents.append([i * B + (a // V if x > -math.inf else min(k, B - 1)) for k, (x, a) in enumerate(zip(top, at))])
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"scores": torch.tensor(values, dtype=torch.float64, device="cuda"), "tokens": ints(tokens),
            "parents": ints(parents), "ended": ints(tokens) == st["end"]}


def _exact_state(case, st):
    out = {}
    for k, t in st["state"].items():
        t = t if t.dtype == torch.int32 else t.double()
        out[k] = torch.stack([t[p] for p in st["parents"].tolist()])
    return out


def _exact_reorder(case, st):
    pt = case["page"]
    table, lens, refs = (st[k].tolist() for k in ("table", "lens", "refs"))
    codes, amax = st["codes"].clone(), st["amax"].double()
    seqs, parents = st["seqs"].tolist(), st["parents"].tolist()
    before, length = [list(table[s]) for s in seqs], [lens[s] for s in seqs]
    for row in before:
        for p in row:
            if p >= 0:
                refs[p] -= 1
    given, waiting = set(), []
    order = sorted(range(len(seqs)), key=lambda i: parents[i] != i)      # those that stay what they are come first
    for i in order:
        a = parents[i]
        row = list(before[a])
        tail = length[a] // pt
        if length[a] % pt and row[tail] >= 0:
            if a in given:
                waiting.append((i, tail, row[tail]))
                row[tail] = -1
            given.add(a)
        for p in row:
            if p >= 0:
                refs[p] += 1
        table[seqs[i]], lens[seqs[i]] = row, length[a]
    free = iter([p for p, x in enumerate(refs) if x == 0])
    for i, tail, page in sorted(waiting):
        to = next(free)
        table[seqs[i]][tail], refs[to] = to, 1
        tiles = -(-(lens[seqs[i]] % pt) // BLOCK)
        codes[:, to, :, :, :tiles * BLOCK * case["dim"]] = st["codes"][:, page, :, :, :tiles * BLOCK * case["dim"]]
        amax[:, to, :, :, :tiles] = st["amax"][:, page, :, :, :tiles].double()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"table": ints(table), "lens": ints(lens), "refs": ints(refs), "codes": codes, "amax": amax}


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


def _exact_shared(case, st):
    """A sequence and a KV head at a time."""
    pt, D, H, G, fmt = case["page"], case["dim"], case["heads"], case["group"], case["fmt"]
    places = _places(D)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    starts, lens, seqs = st["starts"].tolist(), st["lens"].tolist(), st["seqs"].tolist()
    for s, seq in enumerate(seqs):
        n, m = lens[seq], starts[s + 1] - starts[s]
        j = torch.arange(n, device="cuda")
        page, inner = st["table"][seq].long()[j // pt], j % pt // BLOCK
        i = (n - m + torch.arange(m, device="cuda"))[:, None, None]
        hide = (j > i) | ((j <= i - case["window"]) & (j >= case["sinks"]) & (case["window"] > 0))
        for layer in range(case["layers"]):
            for h in range(H):
                kv = []
                for which in (0, 1):
                    byte = inner[:, None] * BLOCK * D + places[which][j % BLOCK]
                    val = _values(st["codes"][layer, page[:, None], h, which, byte], fmt)
                    kv.append(val * (st["amax"][layer, page, h, which, inner].double() / TOP[fmt])[:, None])
                q = st["q"][starts[s]:starts[s + 1], layer, h * G:(h + 1) * G].double()       # [m, G, D]
                z = (q.reshape(-1, D) @ kv[0].T / math.sqrt(D)).reshape(m, G, n)
                p = torch.softmax(z.masked_fill(hide, -math.inf), -1)
                out[starts[s]:starts[s + 1], layer, h * G:(h + 1) * G] = (p.reshape(-1, n) @ kv[1]).reshape(m, G, D)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"select": _exact_select, "state": _exact_state, "reorder": _exact_reorder,
            "shared": _exact_shared}[case["op"]](case, st)
