"""Attention for groups of sequences that share their first pages, against the 64-bit model of pages_ref.py (which knows
nothing of groups) within its bound, and beside ordinary attention."""
import numpy as np
import pytest
import torch

from test_gpu_pages import DEV, HALF_STEP, ints, make
import pages_ref

pytestmark = pytest.mark.gpu


def reach(saved, layers=1, heads=2, dim=128, pt=64, **_):
    """Pages per sequence with which sharing is tried: what `saved` sequences could read less is 16 MB at least."""
    return -(-(16 << 20) // (saved * layers * heads * pt * 2 * dim))


def family(groups, seed=0, spare=2, wide=False, **kw):
    """groups: of each (tokens in common, [tokens of their own ...]).  Sequences in random rows of the table; the pages in
    common are forks'.  wide: tables so long that groups of few rows take tiles of 16.  Returns cache, model, the listed sequences, the group bounds."""
    pt = kw.get("pt", 64)
    rng = np.random.default_rng(seed)
    n = sum(len(t) for _, t in groups)
    room = max(reach(1, **kw) * (12 if wide else 1), max(-(-(pre + max(t)) // pt) for pre, t in groups))
    pages = sum(-(-(pre + x) // pt) for pre, t in groups for x in t) + 3
    c, m = make(pages=pages, seqs=n + spare, seq_pages=room, **kw)
    rows = rng.permutation(n + spare)[:n].tolist()
    bounds, at = [0], 0
    for pre, tails in groups:
        first, others = rows[at], rows[at + 1:at + len(tails)]
        c.resize(ints([first]), ints([pre]))
        assert m.resize([first], [pre])
        if others:
            c.fork(ints([first] * len(others)), ints(others))
            m.fork([first] * len(others), others)
        at += len(tails)
        bounds.append(at)
    lens = [pre + x for pre, tails in groups for x in tails]
    c.resize(ints(rows), ints(lens))
    assert m.resize(rows, lens)
    codes = np.clip(np.rint(rng.normal(size=m.codes.shape) * 36), -127, 127)
    m.codes[:] = codes.astype(np.int64) % 256 if m.fmt == "int8" else pages_ref.encode(codes * 3.0, "e4m3")
    m.amax[:] = np.float32(rng.uniform(2.5, 4.0, m.amax.shape) * np.where(rng.random(m.amax.shape) < 0.02, 4, 1))
    if m.fmt == "e4m3":                                    # what no token owns holds NaN
        own = np.zeros((len(m.refs), pt), bool)
        for s, n_tok in zip(rows, lens):
            for j in range(n_tok):
                own[m.table[s, j // pt], j % pt] = True
        for page, tok in zip(*np.nonzero(~own)):
            for which in (0, 1):
                m.codes[:, page, :, which, tok // 16 * 16 * m.D + m.at[which][tok % 16]] = 0x7f
    c.codes.copy_(torch.from_numpy(m.codes))
    c.amax.copy_(torch.from_numpy(m.amax))
    return c, m, rows, bounds


def attend(c, m, seqs, bounds, new=None, tail=3, seed=1, max_new=None, max_group=None, window=0, sinks=0, layers=None,
           layer_begin=0, q=None, slack=0.0, status=0):
    """One call against the model; `tail` rows behind the last entry stay as they were.  The joining of parts rounds twice
    more: 2^-22 of the largest |v|, which the model's 2^-19 covers."""
    rng = np.random.default_rng(seed)
    new = [1] * len(seqs) if new is None else new
    starts = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
    layers = m.L - layer_begin if layers is None else layers
    shape = (starts[-1] + tail, layers, m.H * m.G, m.D)
    q = torch.from_numpy(rng.normal(size=shape)).to(c.dtype) if q is None else q
    out = torch.full(shape, 7.0, dtype=c.dtype, device=DEV)
    one = all(x == 1 for x in new) and not tail
    c.shared_attention(q.to(DEV), ints(seqs), ints(bounds), None if one else ints(starts), max_new=max_new or max(new),
                       max_group=max_group, layer_begin=layer_begin, window=window, sinks=sinks, out=out)
    got = out.double().cpu().numpy()
    rows = starts[-1]
    assert (got[rows:] == 7.0).all()
    want, bound = m.attention(q[:rows].double().numpy(), seqs, starts, layer_begin, window, sinks)
    if not m.bf16 and (shape[0] if max_group is None else max_group) * m.G > 32:
        # by the caller's hint the groups are the many-token kernel's, which rounds probabilities to fp16 once: as for
        # entries of more than 16 rows in the model, |p' - p| <= 2^-11 p + 2^-25 moves the sum of p' v by at most
        # (2^-11 + n 2^-25) max |v| times the sum of p
        most = np.abs(m.val[np.isfinite(m.val)]).max() * np.nanmax(m.amax) / pages_ref.TOP[m.fmt]
        bound = bound + (2.0 ** -11 + int(m.lens[seqs].max()) * 2.0 ** -25) * most
    tol = HALF_STEP[c.dtype] * np.abs(want) + bound * (1 + slack) + 2.0 ** -24
    err = np.abs(got[:rows] - want)
    assert np.isfinite(got).all()
    worst = np.unravel_index(np.argmax(err - tol), err.shape) if err.size else None
    assert (err <= tol).all(), (worst, got[:rows][worst], want[worst], tol[worst])
    assert c.poll_status() == status
    return got


def near(got, want, m):
    """Two kernels' fp16 results for the same call: each is rounded to half a step, 2^-11 of at most the largest |v|, one's
    probabilities may be rounded to fp16 (2^-11 + n 2^-25 of it, see the model), and both sums in fp32 (2^-19 each)."""
    most = np.abs(m.val[np.isfinite(m.val)]).max() * np.nanmax(m.amax) / pages_ref.TOP[m.fmt]
    tol = most * (3 * 2.0 ** -11 + int(m.lens.max()) * 2.0 ** -25 + 2.0 ** -18)
    return float((got.double() - want.double()).abs().max()) <= tol


KINDS = [("int8", torch.float16), ("e4m3", torch.float16), ("int8", torch.bfloat16), ("e4m3", torch.bfloat16)]


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("dim,pt,heads,group", [(128, 64, 2, 1), (64, 16, 1, 4), (128, 128, 1, 8), (64, 32, 3, 5)])
@pytest.mark.parametrize("hint", [None, 5])
def test_shapes(fmt, dtype, dim, pt, heads, group, hint):
    c, m, seqs, b = family([(300, [1, 5, 40, 130]), (20, [1, 1]), (129, [3]), (10, [20, 30, 9]), (64, [1, 64, 65])],
                           dim=dim, pt=pt, heads=heads, group=group, fmt=fmt, dtype=dtype)
    attend(c, m, seqs, b, max_group=hint)
    attend(c, m, seqs, b, tail=0, max_group=hint)
    attend(c, m, seqs, b, new=[1, 3, 2, 5, 1, 1, 3, 2, 4, 1, 1, 6, 1], max_group=hint)


@pytest.mark.parametrize("fmt,dtype", KINDS)
@pytest.mark.parametrize("dim,pt,heads,group", [(128, 64, 2, 1), (64, 16, 1, 4), (128, 128, 1, 8), (64, 32, 3, 5)])
def test_tiles_of_sixteen_rows(fmt, dtype, dim, pt, heads, group):
    c, m, seqs, b = family([(300, [1, 5, 40, 130]), (20, [1, 1]), (129, [3]), (10, [20, 30, 9]), (64, [1, 64, 65])],
                           dim=dim, pt=pt, heads=heads, group=group, fmt=fmt, dtype=dtype, wide=True)
    for window, sinks in ((0, 0), (100, 20)):
        attend(c, m, seqs, b, window=window, sinks=sinks, max_group=32 // group)
        attend(c, m, seqs, b, window=window, sinks=sinks, tail=0, max_group=32 // group)
        attend(c, m, seqs, b, window=window, sinks=sinks, new=[1, 3, 2, 5, 1, 1, 3, 2, 0, 1, 1, 6, 1], max_group=32 // group)
    attend(c, m, seqs, [0, 13], max_group=32 // group)     # one group of strangers


@pytest.mark.parametrize("each", [2, 17, 70])
def test_tiles_of_sixteen_rows_of_long_groups(each):
    tails = [1 + 7 * i % 60 for i in range(each)]
    c, m, seqs, b = family([(900, tails), (1100, tails[:each // 2 + 1])], heads=2, group=4, pt=32, wide=True)
    attend(c, m, seqs, b, max_group=8)
    attend(c, m, seqs, b, new=[1 + i % 5 for i in range(len(seqs))], max_group=8)


@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("each", [2, 9, 33, 70, 150])
def test_rows_of_a_group(each, group):
    """From a few rows to several tiles of the many-token kernel, with and without its keys split."""
    tails = [1 + 7 * i % 60 for i in range(each)]
    c, m, seqs, b = family([(500, tails), (1100, tails[:each // 2 + 1])], dim=64, pt=32, heads=2, group=group)
    attend(c, m, seqs, b)
    attend(c, m, seqs, b, max_group=1)                     # tiles of eight rows, however many there are
    c, m, seqs, b = family([(1500, tails)], heads=1, group=group, dtype=torch.bfloat16, fmt="e4m3")
    attend(c, m, seqs, b, max_group=each)


@pytest.mark.parametrize("each", [9, 40, 150])
def test_more_rows_than_the_hint(each):
    """Two chains of key tiles for 128 rows each, however many there are."""
    tails = [1 + 7 * i % 60 for i in range(each)]
    c, m, seqs, b = family([(1500, tails), (10, [1, 2]), (700, tails[:each // 2 + 1])], dim=64, pt=32, heads=2, group=4)
    for hint in (9, 20, 32):
        attend(c, m, seqs, b, max_group=hint)
    attend(c, m, seqs, b, new=[1 + i % 4 for i in range(len(seqs))], max_group=20)


def test_hints_that_are_wrong():
    c, m, seqs, b = family([(400, [5, 9, 30, 70]), (90, [6, 6])], heads=2, group=4)
    new = [3, 5, 1, 4, 6, 2]
    for max_new, max_group in ((1, 1), (1, 1000), (6, 1), (200, 5), (32, 40)):
        attend(c, m, seqs, b, new=new, max_new=max_new, max_group=max_group)


@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 0), (100, 4), (37, 33), (64, 16), (1000, 20), (5000, 0), (300, 200)])
@pytest.mark.parametrize("group", [2, 8])
@pytest.mark.parametrize("hint", [1, 1000])
def test_windows(window, sinks, group, hint):
    c, m, seqs, b = family([(700, [1, 50, 90, 200]), (40, [1, 30]), (333, [20] * 5), (64, [600, 5])], heads=1, group=group,
                           dim=64, pt=32)
    attend(c, m, seqs, b, window=window, sinks=sinks, max_group=hint)
    attend(c, m, seqs, b, new=[1, 4, 2, 1, 1, 3, 1, 2, 3, 4, 5, 7, 1], window=window, sinks=sinks, max_group=hint)


def test_tokens_that_are_themselves_in_shared_pages():
    """Forks that have not parted: the new tokens' own keys lie in pages in common, or right at their end."""
    for pre in (16, 63, 64, 65, 127, 128, 129, 192):
        c, m = make(heads=2, pages=30, seqs=5, seq_pages=reach(1), pt=64)
        c.resize(ints([1]), ints([pre]))
        m.resize([1], [pre])
        rng = np.random.default_rng(pre)
        m.codes[:] = rng.integers(0, 255, m.codes.shape)
        m.amax[:] = np.float32(rng.uniform(1, 2, m.amax.shape))
        c.codes.copy_(torch.from_numpy(m.codes))
        c.amax.copy_(torch.from_numpy(m.amax))
        c.fork(ints([1, 1]), ints([3, 0]))
        m.fork([1, 1], [3, 0])
        for hint in (1, 1000):
            for new in ([1, 1, 1], [2, 1, 5], [16, 16, 16]):
                attend(c, m, [3, 1, 0], [0, 3], new=new, max_group=hint)
            attend(c, m, [3, 3, 1, 1], [0, 2, 4], max_group=hint)    # a sequence listed twice shares all with itself
            attend(c, m, [0, 1], [0, 1, 2], max_group=hint)


def test_groups_that_share_nothing():
    c, m, seqs, b = family([(5, [9, 60]), (80, [4]), (0, [30, 31, 0]), (33, [1, 1])], heads=2, pt=64)
    for hint in (1, 1000):
        attend(c, m, seqs, [0, len(seqs)], new=[1, 2, 1, 4, 1, 0, 1, 1], max_group=hint)    # one group of strangers
        attend(c, m, seqs, b, new=[0, 2, 1, 0, 0, 0, 1, 0], max_group=hint)
        attend(c, m, seqs, [0, 0, 2, 2, 3, 8], new=[1, 2, 1, 4, 1, 0, 1, 1], max_group=hint)   # groups without entries


def test_small_caches_share_nothing():
    """Where sequences cannot be long enough for sharing to pay, it is ordinary attention, bit for bit."""
    c, m = make(heads=2, pages=30, seqs=5, seq_pages=5, pt=64)
    c.resize(ints([1]), ints([200]))
    c.fork(ints([1, 1]), ints([3, 0]))
    c.codes.random_(0, 120), c.amax.uniform_(1, 2)
    q = torch.randn(3, 1, 2, 128, dtype=torch.float16, device=DEV)
    s = ints([3, 0, 1])
    assert torch.equal(c.shared_attention(q, s, ints([0, 3])), c.attention(q, s)) and c.poll_status() == 0


def test_more_new_tokens_than_a_sequence_has():
    c, m, seqs, b = family([(3, [2, 4]), (100, [5, 6])], heads=1, pt=16, dim=64)
    starts = [0, 9, 10, 11, 12]
    q = torch.randn(12, 1, 1, 64).half()
    want = c.attention(q.to(DEV), ints(seqs), ints(starts))
    for hint in (9, 1000):
        got = c.shared_attention(q.to(DEV), ints(seqs), ints(b), ints(starts), max_group=hint)
        assert near(got, want, m) and (got[:4] == 0).all() and c.poll_status() == 0


def test_trimmed_and_reordered_beams():
    c, m, seqs, b = family([(700, [3, 40, 41]), (300, [7, 9])], heads=2, pt=32)
    c.trim(ints(seqs), 32, 150)
    m.trim(seqs, 32, 150)
    for hint in (3, 1000):
        attend(c, m, seqs, b, window=150, sinks=20, max_group=hint)
        attend(c, m, seqs, b, max_group=hint)              # what is not there any more is not seen


def test_many_layers_pass_in_turns():
    """More rows than there is room for the parts of: layers in several turns, and a layer that does not fit."""
    c, m, seqs, b = family([(40, [1] * 60), (30, [2] * 60)], heads=16, group=1, dim=128, pt=16, layers=40)
    q = torch.randn(120, 40, 16, 128, dtype=torch.float16, device=DEV)
    got = c.shared_attention(q, ints(seqs), ints(b))
    want = c.attention(q, ints(seqs))
    assert near(got, want, m) and c.poll_status() == 0
    assert torch.equal(c.shared_attention(q[:, 3:7].contiguous(), ints(seqs), ints(b), layer_begin=3),
                       c.shared_attention(q[:, 3:7], ints(seqs), ints(b), layer_begin=3))
    c, m, seqs, b = family([(40, [30] * 60)], heads=32, group=4, dim=64, pt=16)
    new = [20] * 60
    q = torch.randn(1200, 1, 128, 64, dtype=torch.float16, device=DEV)
    starts = ints(np.arange(61) * 20)
    got = c.shared_attention(q, ints(seqs), ints(b), starts, max_new=20)
    assert near(got, c.attention(q, ints(seqs), starts, max_new=20), m) and c.poll_status() == 0


def test_lists_that_are_wrong():
    c, m, seqs, b = family([(200, [3, 4, 5]), (90, [2, 2])], heads=2, group=2)
    for hint in (3, 1000):
        for bounds in ([0, 3, 4], [1, 3, 5], [0, 4, 3, 5], [0, -1, 5], [0, 6, 5], [0, 3, 1 << 30]):
            attend(c, m, seqs, bounds, status=-8, max_group=hint)      # nothing is shared, the result is right
        bad = list(seqs)
        bad[1] = 99
        q = torch.randn(5, 1, 4, 128, dtype=torch.float16, device=DEV)
        out = torch.full_like(q, 7.0)
        c.shared_attention(q, ints(bad), ints(b), out=out, max_group=hint)
        assert c.poll_status() == -8 and (out[1] == 7).all()
        want = c.attention(q, ints(seqs))
        keep = [0, 2, 3, 4]
        assert near(out[keep], want[keep], m)
        for starts in ([0, 2, 1, 3, 4, 5], [0, 1, 2, 3, 4, 9], [5, 0, 5, 0, 5, 0], [-1, 1, 2, 3, 4, 5]):
            c.shared_attention(q, ints(seqs), ints(b), ints(starts), out=out, max_group=hint)
            assert c.poll_status() == -8, starts


@pytest.mark.parametrize("many", [False, True])
def test_values_and_scores_far_apart(many):
    """A first token that holds nearly all probability in the shared half, or in the rest; magnitudes 2^60 apart."""
    each = 40 if many else 3
    for where in ("shared", "rest", "zero"):
        c, m, seqs, b = family([(256, [20] * each)], heads=1, group=1, dim=64, pt=64, seed=4, dtype=torch.bfloat16)
        q = torch.randn(each, 1, 1, 64)
        if where == "zero":
            m.amax[:, m.table[seqs[0], 0]] = 0.0
        else:
            page = m.table[seqs[0], 0 if where == "shared" else 4]
            m.amax[:, page, :, 1] *= 2.0 ** 60
            m.amax[:, page, :, 0] *= 3.0
        c.amax.copy_(torch.from_numpy(m.amax))
        attend(c, m, seqs, b, tail=0, q=q.to(torch.bfloat16), max_group=each)


def test_captured_beside_other_calls_and_on_a_stream():
    c, m, seqs, b = family([(300, [4, 40, 80]), (65, [9, 2])], heads=2, group=2, pt=32)
    q = torch.randn(5, 1, 4, 128, dtype=torch.float16, device=DEV)
    s, g = ints(seqs), ints(b)
    want = c.shared_attention(q, s, g, max_group=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [c.shared_attention(q, s, g, max_group=3, stream=side) for _ in range(20)]
    side.synchronize()
    assert all(torch.equal(x, want) for x in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one = c.shared_attention(q, s, g, max_group=3)
        two = c.attention(q, s)
        three = c.shared_attention(q, s, g, max_group=1000)
        four = c.shared_attention(q, s, g, max_group=3)
    for _ in range(3):
        one.zero_(), four.zero_()
        graph.replay()
        assert torch.equal(one, want) and torch.equal(four, want)
        assert near(two, want, m) and near(three, want, m)
    assert c.poll_status() == 0


@pytest.mark.parametrize("groups,heads", [([(3000, [4, 40, 80] * 4)], 2), ([(300, [30, 60] * 3)] * 40, 4)])
def test_calls_right_behind_one_another(groups, heads):
    """Writes and attention without a pause give what they give with one after each: in parts that are joined by a kernel of
    their own (one long text), and in one or two (many groups)."""
    c, m, seqs, b = family(groups, heads=heads, group=4, pt=32)
    s, g = ints(seqs), ints(b)
    gen = torch.Generator(device=DEV).manual_seed(3)
    qs = [torch.randn(len(seqs), 1, heads * 4, 128, dtype=torch.float16, device=DEV, generator=gen) for _ in range(6)]
    kv = [torch.randn(len(seqs), 1, heads, 128, dtype=torch.float16, device=DEV, generator=gen) for _ in range(6)]
    codes, amax = c.codes.clone(), c.amax.clone()

    def run(pause):
        c.codes.copy_(codes), c.amax.copy_(amax)
        out = []
        for i in range(6):
            c.write(kv[i], kv[-1 - i], s)
            pause()
            out.append(c.shared_attention(qs[i], s, g, max_group=100))
            pause()
            out.append(c.shared_attention(qs[-1 - i], s, g, max_group=100))
            pause()
        torch.cuda.synchronize()
        return torch.stack(out)

    want = run(torch.cuda.synchronize)
    assert not torch.equal(want[0], want[2])
    for _ in range(5):
        assert torch.equal(run(lambda: None), want)
    assert c.poll_status() == 0
