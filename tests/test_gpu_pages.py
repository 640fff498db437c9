"""The paged 8-bit cache on the GPU against the 64-bit model of pages_ref.py: maps and codes exactly, attention within
the model's bound plus half a rounding step of the output type (fp16 2^-11, bf16 2^-8 of the value)."""
import numpy as np
import pytest
import torch

import pages_ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def ints(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device=DEV)


def make(layers=1, heads=2, dim=128, pages=40, seqs=6, seq_pages=12, group=1, pt=64, fmt="int8", dtype=torch.float16):
    from paper_2402_09398_b200 import binding as B
    cache = B.PagedCache(layers, heads, dim, pages, seqs, seq_pages, group=group, page_tokens=pt, fmt=fmt, dtype=dtype)
    cache.codes.zero_()                                    # layers that a test never writes compare equal
    cache.amax.zero_()
    model = pages_ref.Model(layers, heads, dim, pages, seqs, seq_pages, group, pt, fmt, dtype == torch.bfloat16)
    return cache, model


def same_maps(cache, model):
    assert np.array_equal(cache.table.cpu().numpy(), model.table)
    assert np.array_equal(cache.lens.cpu().numpy(), model.lens)
    assert np.array_equal(cache.refs.cpu().numpy(), model.refs)


def same_contents(cache, model):
    """Codes and magnitudes of every block that holds a token (of the last one, the tokens behind the end too)."""
    same_maps(cache, model)
    codes, amax = cache.codes.cpu().numpy(), cache.amax.double().cpu().numpy()
    for s in range(len(model.lens)):
        for b in range(-(-int(model.lens[s]) // 16)):
            page, inner = model.table[s, b * 16 // model.pt], b % (model.pt // 16)
            if page < 0:
                continue
            tile = slice(inner * 16 * model.D, (inner + 1) * 16 * model.D)
            assert np.array_equal(amax[:, page, :, :, inner], model.amax[:, page, :, :, inner]), (s, b)
            assert np.array_equal(codes[:, page, :, :, tile], model.codes[:, page, :, :, tile]), (s, b)


def fill(cache, model, lens, seed=0, amp=1.0):
    """Sequences 0, 1, ... get these lengths and random codes; what no token owns holds NaN."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    cache.resize(ints(range(n)), ints(lens))
    assert model.resize(list(range(n)), list(lens))
    same_maps(cache, model)
    codes = np.clip(np.rint(rng.normal(size=model.codes.shape) * 36), -127, 127)
    if model.fmt == "int8":
        model.codes[:] = codes.astype(np.int64) % 256
    else:
        model.codes[:] = pages_ref.encode(codes * 3.0, "e4m3")
    model.amax[:] = np.float32(rng.uniform(2.5, 4.0, model.amax.shape) * amp)
    own = np.zeros((len(model.refs), model.pt), bool)
    for s in range(n):
        for j in range(lens[s]):
            own[model.table[s, j // model.pt], j % model.pt] = True
    if model.fmt == "e4m3":
        for page, tok in zip(*np.nonzero(~own)):
            for which in (0, 1):
                byte = tok // 16 * 16 * model.D + model.at[which][tok % 16]
                model.codes[:, page, :, which, byte] = 0x7f
    dead = ~own.reshape(len(model.refs), -1, 16).any(2)
    model.amax[:, dead.nonzero()[0], :, :, dead.nonzero()[1]] = np.nan
    cache.codes.copy_(torch.from_numpy(model.codes))
    cache.amax.copy_(torch.from_numpy(model.amax))


def attend(cache, model, seqs, starts, max_new=None, layers=None, layer_begin=0, window=0, sinks=0, scale=None, seed=1,
           slack=0.0, tail=3):
    """One call against the model; `tail` rows behind the last entry stay as they were."""
    rng = np.random.default_rng(seed)
    layers = model.L - layer_begin if layers is None else layers
    rows = starts[-1]
    shape = (rows + tail, layers, model.H * model.G, model.D)
    q = torch.from_numpy(rng.normal(size=shape)).to(cache.dtype)
    out = torch.full(shape, 7.0, dtype=cache.dtype, device=DEV)
    one = all(b - a == 1 for a, b in zip(starts, starts[1:])) and not tail
    cache.attention(q.to(DEV), ints(seqs), None if one else ints(starts), max_new=max_new, layer_begin=layer_begin,
                    window=window, sinks=sinks, scale=scale, out=out)
    got = out.double().cpu().numpy()
    assert (got[rows:] == 7.0).all()
    want, bound = model.attention(q[:rows].double().numpy(), seqs, starts, layer_begin, window, sinks, scale)
    tol = HALF_STEP[cache.dtype] * np.abs(want) + bound * (1 + slack) + 2.0 ** -24
    err = np.abs(got[:rows] - want)
    assert np.isfinite(got).all()
    worst = np.unravel_index(np.argmax(err - tol), err.shape) if err.size else None
    assert (err <= tol).all(), (worst, got[:rows][worst], want[worst], tol[worst])
    assert cache.poll_status() == 0
    return got


# --------------------------------------------------------------------------- #
# maps
# --------------------------------------------------------------------------- #
def test_resize_grows_shrinks_and_refuses():
    c, m = make(pages=10, seqs=5, seq_pages=8, pt=16)
    for seqs, lens in (([0, 1, 2], [1, 33, 0]), ([2, 0], [16, 17]), ([1, 3], [16, 40]), ([0, 1, 2, 3], [0, 0, 16, 7]),
                       ([4, 4, 0], [20, 99, 5]), ([1], [0]), ([1], [128 - 80])):
        c.resize(ints(seqs), ints(lens))
        assert m.resize(seqs, lens)
        same_maps(c, m)
    assert c.poll_status() == 0
    from paper_2402_09398_b200 import binding as B
    # 1 + 3 + 1 + 1 + 2 pages are in use: with 2 free ones the growth is refused, the shrinking is done
    c.resize(ints([2, 1, 4]), ints([0, 128, 128]))
    assert not m.resize([2, 1, 4], [0, 128, 128])
    same_maps(c, m)
    c.resize(ints([2]), ints([16]))                       # until the status is read, nothing changes
    same_maps(c, m)
    assert c.poll_status() == B.LESS_ERR_PAGES_EXHAUSTED and c.poll_status() == 0
    for seqs, lens in (([5], [1]), ([-1], [1]), ([0], [-1]), ([0], [129])):
        c.resize(ints(seqs), ints(lens))
        assert c.poll_status() == -8
        same_maps(c, m)
    c.resize(ints([2]), ints([16]))
    assert m.resize([2], [16]) and c.poll_status() == 0
    same_maps(c, m)


@pytest.mark.parametrize("seed", range(6))
def test_a_life_of_the_maps(seed):
    """Random operations; every sequence's contents follow it through forks, copies and compaction."""
    rng = np.random.default_rng(seed)
    pt = [16, 32, 64][seed % 3]
    c, m = make(layers=2, heads=1, dim=64, pages=60, seqs=12, seq_pages=9, pt=pt, fmt=["int8", "e4m3"][seed % 2])
    for step in range(40):
        op = rng.integers(0, 6)
        if op <= 2:
            seqs = rng.permutation(12)[:rng.integers(1, 8)].tolist()
            lens = [0 if rng.random() < 0.3 else int(rng.integers(0, 9 * pt + 1)) for _ in seqs]
            if op == 2:                                    # cut back a little: growth inside shared pages follows
                lens = [max(0, int(m.lens[s]) - int(rng.integers(0, 2 * pt))) for s in seqs]
            ok = m.resize(seqs, lens)
            c.resize(ints(seqs), ints(lens))
            assert (c.poll_status() == 0) == ok
            if ok and op < 2:                              # new tokens for those that have any
                new = [int(min(m.lens[s], rng.integers(0, 20))) for s in seqs]
                new = [k if all(m.refs[m.table[s, o]] == 1 for o in range((int(m.lens[s]) - k) // pt, -(-int(m.lens[s]) // pt)))
                       else 0 for k, s in zip(new, seqs)]
                starts = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
                k, v = (torch.from_numpy(rng.normal(size=(starts[-1], 2, 1, 64))).half() for _ in range(2))
                c.write(k.to(DEV), v.to(DEV), ints(seqs), ints(starts))
                m.write(seqs, starts, k.double().numpy(), v.double().numpy())
                assert c.poll_status() == 0
        elif op == 3:
            empty = [s for s in range(12) if m.lens[s] == 0]
            full = [s for s in range(12) if m.lens[s] > 0]
            if empty and full:
                dst = empty[:3]
                src = [full[rng.integers(0, len(full))] for _ in dst]
                if (m.refs == 0).sum() >= 3:
                    m.fork(src, dst)
                    c.fork(ints(src), ints(dst))
                    assert c.poll_status() == 0
        else:
            m.compact()
            c.compact()
        same_maps(c, m)


def test_forked_pages_are_copied_before_they_change():
    c, m = make(layers=2, heads=3, dim=64, pages=30, seqs=6, seq_pages=6, pt=32)
    rng = np.random.default_rng(3)

    def grow(seqs, lens):
        old = [int(m.lens[s]) for s in seqs]
        assert m.resize(seqs, lens)
        c.resize(ints(seqs), ints(lens))
        new = [b - a for a, b in zip(old, lens)]
        starts = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
        k, v = (torch.from_numpy(rng.normal(size=(starts[-1], 2, 3, 64)) * 2.0 ** rng.integers(-2, 3)).half()
                for _ in range(2))
        c.write(k.to(DEV), v.to(DEV), ints(seqs), ints(starts))
        m.write(seqs, starts, k.double().numpy(), v.double().numpy())
        assert c.poll_status() == 0
        same_contents(c, m)

    grow([0, 1], [75, 64])
    m.fork([0, 0, 1], [2, 3, 4])
    c.fork(ints([0, 0, 1]), ints([2, 3, 4]))
    same_contents(c, m)
    grow([0, 2, 3, 4], [80, 76, 110, 65])
    # back behind the fork, into a page that three sequences hold: all of them get copies as they grow
    for s in (0, 2, 3):
        assert m.resize([s], [40 + s])
    c.resize(ints([0, 2, 3]), ints([40, 42, 43]))
    same_maps(c, m)
    grow([3, 0, 2], [50, 70, 43])
    m.compact()
    c.compact()
    same_contents(c, m)
    assert c.poll_status() == 0


def test_fork_refusals():
    from paper_2402_09398_b200 import binding as B
    c, m = make(pages=6, seqs=5, seq_pages=4, pt=16)
    c.resize(ints([0, 1]), ints([40, 10]))
    m.resize([0, 1], [40, 10])
    for src, dst, code in (([0], [1], -10), ([0, 1], [2, 2], -10), ([0], [0], -10), ([0, 2], [2, 3], -10),
                           ([0, 0, 0], [2, 3, 4], B.LESS_ERR_PAGES_EXHAUSTED), ([5], [2], -8), ([0], [-1], -8)):
        c.fork(ints(src), ints(dst))
        assert c.poll_status() == code, (src, dst)
        same_maps(c, m)
    c.fork(ints([0, 0]), ints([2, 3]))
    m.fork([0, 0], [2, 3])
    assert c.poll_status() == 0
    same_maps(c, m)


def test_trim_and_what_follows():
    from paper_2402_09398_b200 import binding as B
    c, m = make(pages=40, seqs=4, seq_pages=12, pt=16)
    c.resize(ints([0, 1, 2]), ints([190, 64, 5]))
    m.resize([0, 1, 2], [190, 64, 5])
    for sinks, window in ((4, 50), (0, 33), (0x7fffffff, 1), (17, 16), (0, 0x7fffffff)):
        c.trim(ints([0, 1, 2, 0]), sinks, window)
        m.trim([0, 1, 2], sinks, window)
        same_maps(c, m)
    c.compact()
    m.compact()
    same_maps(c, m)
    assert c.poll_status() == 0
    c.resize(ints([0]), ints([100]))                       # into what was trimmed: cut, but not grown again
    m.resize([0], [100])
    c.resize(ints([0]), ints([120]))
    assert not m.resize([0], [120])
    assert c.poll_status() == -10
    same_maps(c, m)
    c.trim(ints([9]), 0, 5)
    assert c.poll_status() == -8
    assert B.LESS_PAGE_BLOCK == 16


@pytest.mark.parametrize("pages", [1, 3, 1023, 1025, 70001])
def test_large_and_odd_pools(pages):
    c, m = make(heads=1, dim=64, pages=pages, seqs=40, seq_pages=max(2, min(4000, pages)), pt=16)
    rng = np.random.default_rng(pages)
    lens = [int(x) for x in rng.integers(0, max(2, pages * 16 // 45), 40)]
    ok = m.resize(list(range(40)), lens)
    c.resize(ints(range(40)), ints(lens))
    assert (c.poll_status() == 0) == ok
    gone = list(range(0, 40, 3))
    m.resize(gone, [0] * len(gone))
    c.resize(ints(gone), ints([0] * len(gone)))
    same_maps(c, m)
    m.compact()
    c.compact()
    same_maps(c, m)


# --------------------------------------------------------------------------- #
# the write
# --------------------------------------------------------------------------- #
@pytest.mark.parametrize("dim,heads,pt,fmt,dtype", [(128, 3, 64, "int8", torch.float16), (64, 1, 16, "e4m3", torch.bfloat16),
                                                    (64, 5, 32, "int8", torch.bfloat16), (128, 2, 256, "e4m3", torch.float16)])
def test_write_codes_exactly(dim, heads, pt, fmt, dtype):
    c, m = make(layers=3, heads=heads, dim=dim, pages=60, seqs=7, seq_pages=8, pt=pt, fmt=fmt, dtype=dtype)
    rng = np.random.default_rng(dim + pt)
    order = [4, 0, 6, 2, 5]
    lens = np.zeros(7, int)
    for round_, new in enumerate(([1, 0, 15, 16, 40], [1, 1, 1, 1, 1], [3, 33, 0, 1, 17], [1, 1, 1, 1, 1])):
        lens[order] += new
        assert m.resize(order, lens[order].tolist())
        c.resize(ints(order), ints(lens[order]))
        starts = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
        amp = 2.0 ** rng.integers(-3, 4)
        shape = (starts[-1] + 2, 2, heads, dim)
        k, v = (torch.from_numpy(rng.normal(size=shape) * amp).to(dtype) for _ in range(2))
        k[::3] *= 4
        if round_ == 2:
            v[:, :, 0] = 0                                  # a head whose values are all zero
            k[0, 0, 0, 3], k[1, 0, 0, 5] = float("inf"), float("nan")
            v[2, 1, heads - 1, 0] = -float("inf")
        # k and v as slices of one projection's output
        both = torch.cat([k.reshape(len(k), -1), v.reshape(len(v), -1)], 1).to(DEV)
        half = both.shape[1] // 2
        kd, vd = both[:, :half].view(shape), both[:, half:].view(shape)
        if new == [1] * 5:
            c.write(kd[:5], vd[:5], ints(order), layer_begin=1)
        else:
            c.write(kd, vd, ints(order), ints(starts), layer_begin=1)
        m.write(order, starts, k.double().numpy(), v.double().numpy(), layer_begin=1)
        assert c.poll_status() == 0
        same_contents(c, m)


def test_write_ties_and_extremes():
    """Halves of the magnitude and other exact ties round to even; subnormal and very large magnitudes."""
    for dtype in (torch.float16, torch.bfloat16):
        for fmt in ("int8", "e4m3"):
            c, m = make(heads=1, dim=64, pages=8, seqs=1, seq_pages=8, pt=16, fmt=fmt, dtype=dtype)
            x = torch.zeros(96, 1, 1, 64)
            x[:16] = torch.linspace(-1, 1, 64)
            x[0, 0, 0, 0], x[16:32] = 254.0, (torch.arange(1024).reshape(16, 1, 1, 64) - 512) / 4.0
            x[16, 0, 0, 0] = 127.0
            x[32:48] = torch.arange(1024).reshape(16, 1, 1, 64) * 2.0 ** -24
            x[48:64] = (torch.arange(1024).reshape(16, 1, 1, 64) - 512) * (2.0 ** 90 if dtype == torch.bfloat16 else 100.0)
            x[64:80] = -0.0
            x[80:96] = float("nan")
            x = x.to(dtype)
            c.resize(ints([0]), ints([96]))
            m.resize([0], [96])
            c.write(x.to(DEV), (x * 0.5).to(DEV), ints([0]), ints([0, 96]))
            m.write([0], [0, 96], x.double().numpy(), (x * 0.5).double().numpy())
            assert c.poll_status() == 0
            same_contents(c, m)


def test_write_refusals():
    c, m = make(pages=20, seqs=4, seq_pages=4, pt=16, heads=2)
    x = torch.randn(8, 1, 2, 128, device=DEV).half()
    y = torch.randn(8, 1, 2, 128, device=DEV).half()
    c.resize(ints([0, 1]), ints([20, 5]))
    m.resize([0, 1], [20, 5])
    c.write(x, x, ints([0, 1]), ints([0, 4, 8]))
    m.write([0, 1], [0, 4, 8], x.double().cpu().numpy(), x.double().cpu().numpy())
    same_contents(c, m)
    for seqs, starts in (([0, 9], [0, 4, 8]), ([0, -1], [0, 4, 8]), ([0, 1], [0, 4, 9]), ([0, 1], [0, 4, 2]),
                         ([1, 3], [0, 0, 3]), ([1], [0, 6])):
        c.write(x, x, ints(seqs), ints(starts))
        assert c.poll_status() == -8, (seqs, starts)
    m.write([0], [0, 4], x.double().cpu().numpy(), x.double().cpu().numpy())
    same_contents(c, m)
    # the first entry of a sequence counts
    c.write(torch.cat([x[:4], y[:4]]), torch.cat([x[:4], y[:4]]), ints([0, 0]), ints([0, 4, 8]))
    assert c.poll_status() == 0
    same_contents(c, m)
    # a page that a fork shares is not written
    c.resize(ints([0]), ints([32]))
    m.resize([0], [32])
    c.fork(ints([0]), ints([2]))
    m.fork([0], [2])
    before = c.codes.clone()
    c.write(y[:1], y[:1], ints([2]))
    assert c.poll_status() == -10 and torch.equal(before, c.codes)
    for bad in (x.float(), x[:, :, :1], x.cpu(), x.transpose(2, 3), torch.zeros(8, 2, 2, 128, device=DEV).half()):
        with pytest.raises(ValueError):
            c.write(bad, bad, ints([0]), ints([0, 8]))
    with pytest.raises(ValueError):
        c.write(x, x, torch.zeros(1, dtype=torch.int64, device=DEV), ints([0, 8]))
    with pytest.raises(ValueError):
        c.write(x, x, ints([0, 1]), ints([0, 8]))


# --------------------------------------------------------------------------- #
# attention
# --------------------------------------------------------------------------- #
CASES = [  # dim, heads, group, pt, fmt, dtype
    (128, 2, 1, 64, "int8", torch.float16), (128, 1, 8, 16, "e4m3", torch.bfloat16),
    (128, 2, 5, 32, "int8", torch.bfloat16), (64, 1, 71, 64, "int8", torch.float16),
    (64, 3, 12, 128, "e4m3", torch.float16), (64, 2, 1, 16, "int8", torch.bfloat16),
    (128, 1, 16, 256, "e4m3", torch.float16), (128, 1, 128, 64, "int8", torch.bfloat16),
]


@pytest.mark.parametrize("dim,heads,group,pt,fmt,dtype", CASES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (20, 4), (100, 40)])
def test_single_tokens(dim, heads, group, pt, fmt, dtype, window, sinks):
    lens = [1, 16, 17, 130, 255, 64]
    c, m = make(layers=2, heads=heads, dim=dim, group=group, pt=pt, fmt=fmt, dtype=dtype, pages=60,
                seq_pages=-(-256 // pt))
    fill(c, m, lens)
    order = [3, 0, 5, 1, 4, 2]
    attend(c, m, order, list(range(7)), window=window, sinks=sinks, tail=0)
    attend(c, m, order[:4], list(range(5)), layer_begin=1, window=window, sinks=sinks, scale=0.3)


@pytest.mark.parametrize("dim,heads,group,pt,fmt,dtype", CASES[:5])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 4)])
def test_several_tokens(dim, heads, group, pt, fmt, dtype, window, sinks):
    lens = [7, 40, 200, 33, 64]
    new = [7, 1, 5, 0, 30]
    c, m = make(layers=1, heads=heads, dim=dim, group=group, pt=pt, fmt=fmt, dtype=dtype, pages=60,
                seq_pages=-(-256 // pt))
    fill(c, m, lens)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
    a = attend(c, m, [0, 1, 2, 3, 4], starts, max_new=30, window=window, sinks=sinks, slack=0.0)
    assert a.shape[0] == starts[-1] + 3


def test_rows_that_see_nothing():
    c, m = make(pages=20, seqs=4, seq_pages=8, pt=16, heads=2, group=3)
    fill(c, m, [0, 3, 100])
    # sequence 0 is empty; sequence 1 is given more new tokens than it has
    attend(c, m, [0, 1, 2], [0, 1, 6, 8])
    # everything but the last page is trimmed: those keys are not seen
    c.trim(ints([2]), 0, 4)
    m.trim([2], 0, 4)
    attend(c, m, [2, 0], [0, 2, 3])
    attend(c, m, [2], [0, 1], window=4, tail=0)


@pytest.mark.parametrize("lens", [[5000], [3000, 1], [1, 2999, 40, 700]])
@pytest.mark.parametrize("group,fmt", [(1, "int8"), (8, "e4m3"), (16, "int8")])
def test_long_sequences_are_split_and_merged(lens, group, fmt):
    c, m = make(heads=1, dim=64, group=group, pt=32, pages=200, seq_pages=160, seqs=4, fmt=fmt)
    fill(c, m, lens)
    n = len(lens)
    first = attend(c, m, list(range(n)), list(range(n + 1)), tail=0)
    again = attend(c, m, list(range(n)), list(range(n + 1)), tail=0)
    assert np.array_equal(first, again)                    # the order of the sums is fixed


def test_many_short_sequences():
    n = 700
    c, m = make(heads=1, dim=64, group=2, pt=16, pages=3000, seqs=n, seq_pages=4)
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 60, n)]
    fill(c, m, lens)
    attend(c, m, list(range(n)), list(range(n + 1)), tail=0)


def test_magnitudes_far_apart_and_peaked_scores():
    """Value blocks from 2^-12 to 2^10, zero blocks, scores of a few hundred."""
    for dtype in (torch.float16, torch.bfloat16):
        c, m = make(heads=2, dim=128, group=4, pt=16, pages=30, seq_pages=12, dtype=dtype)
        fill(c, m, [190, 45, 16])
        rng = np.random.default_rng(8)
        m.amax[:, :, :, 1] = np.float32(2.0 ** rng.integers(-12, 11, m.amax[:, :, :, 1].shape))
        m.amax[:, ::4, :, 1] = 0
        c.amax.copy_(torch.from_numpy(m.amax))
        attend(c, m, [0, 1, 2], [0, 1, 2, 3], tail=0)
        m.amax[:, :, :, 1] = 3.0
        m.amax[:, :, :, 0] *= 20
        c.amax.copy_(torch.from_numpy(m.amax))
        attend(c, m, [0, 1, 2], [0, 1, 2, 3], tail=0)


def test_a_bad_query_stays_in_its_row():
    for dtype in (torch.float16, torch.bfloat16):
        c, m = make(heads=1, group=4, dtype=dtype)
        fill(c, m, [50, 300])
        q = torch.randn(2, 1, 4, 128).to(dtype).to(DEV)
        good = c.attention(q, ints([0, 1])).clone()
        q[1, 0, 2, 7] = float("nan")
        bad = c.attention(q, ints([0, 1]))
        assert torch.isnan(bad[1, 0, 2]).all()
        keep = torch.ones(2, 1, 4, dtype=torch.bool)
        keep[1, 0, 2] = False
        assert torch.equal(bad[keep.to(DEV)], good[keep.to(DEV)])


def test_attention_refusals():
    c, m = make(heads=2, group=2, pages=20, seqs=3)
    fill(c, m, [50, 20])
    q = torch.randn(4, 1, 4, 128, device=DEV).half()
    for seqs, starts in (([7], [0, 1]), ([0, -1], [0, 1, 2]), ([0], [0, 5]), ([0, 1], [0, 3, 2])):
        out = torch.full_like(q, 3.0)
        c.attention(q, ints(seqs), ints(starts), out=out)
        assert c.poll_status() == -8
    c.table[0, 0] = 1000                                    # a page the pool does not have
    c.attention(q[:1], ints([0]))
    assert c.poll_status() == -8
    for bad in (q.float(), q[:, :, :3], q.cpu()):
        with pytest.raises(ValueError):
            c.attention(bad, ints([1]), ints([0, 1]))
    with pytest.raises(ValueError):
        c.attention(q, ints([1]), ints([0, 1]), out=torch.empty(4, 1, 4, 128, device=DEV))
    from paper_2402_09398_b200 import binding as B
    with pytest.raises(B.LessError):
        c.attention(q, ints([1]), ints([0, 1]), window=-1)
    with pytest.raises(B.LessError):
        c.attention(q, ints([0, 1]))                        # four rows for two sequences


def test_strided_queries():
    c, m = make(heads=2, group=2)
    fill(c, m, [70, 200])
    wide = torch.randn(2, 3 * 4 * 128, device=DEV).half()
    q = wide[:, 512:1024].view(2, 1, 4, 128)
    assert torch.equal(c.attention(q, ints([0, 1])), c.attention(q.contiguous(), ints([0, 1])))


# --------------------------------------------------------------------------- #
# together
# --------------------------------------------------------------------------- #
def test_a_generation():
    """Prompts, steps with a window, a fork, an end and a compaction, as a server would run them."""
    c, m = make(layers=2, heads=2, dim=64, group=3, pt=16, pages=60, seqs=6, seq_pages=12, fmt="int8")
    rng = np.random.default_rng(11)

    def step(seqs, new, layer_by_layer):
        lens = [int(m.lens[s]) + k for s, k in zip(seqs, new)]
        assert m.resize(seqs, lens)
        c.resize(ints(seqs), ints(lens))
        starts = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
        k, v = (torch.from_numpy(rng.normal(size=(starts[-1], 2, 2, 64))).half() for _ in range(2))
        for b, e in ((0, 1), (1, 2)) if layer_by_layer else ((0, 2),):
            c.write(k[:, b:e].to(DEV).contiguous(), v[:, b:e].to(DEV).contiguous(), ints(seqs), ints(starts), layer_begin=b)
        m.write(seqs, starts, k.double().numpy(), v.double().numpy())
        same_contents(c, m)
        attend(c, m, seqs, starts, max_new=max(new), window=40, sinks=4, seed=int(rng.integers(1 << 30)))

    step([0, 1, 2], [50, 7, 90], False)
    for _ in range(3):
        step([0, 1, 2], [1, 1, 1], True)
    m.fork([1, 2], [3, 4])
    c.fork(ints([1, 2]), ints([3, 4]))
    step([4, 3, 0], [1, 2, 3], False)
    m.resize([2], [0])
    c.resize(ints([2]), ints([0]))
    m.trim([0, 4], 4, 40)
    c.trim(ints([0, 4]), 4, 40)
    m.compact()
    c.compact()
    same_contents(c, m)
    step([0, 1, 3, 4], [1, 1, 1, 1], True)
    assert c.poll_status() == 0


def test_captured_step_allocates_and_attends():
    """One captured decode step, replayed: lengths advance on the device, pages are taken as they are needed."""
    c, m = make(heads=2, dim=128, group=2, pt=16, pages=30, seqs=3, seq_pages=8)
    fill(c, m, [15, 31, 5])
    m.resize([0, 1, 2], [15, 31, 5])
    seqs = ints([0, 1, 2])
    k, v = (torch.randn(3, 1, 2, 128, device=DEV).half() for _ in range(2))
    q = torch.randn(3, 1, 4, 128, device=DEV).half()
    out = torch.empty_like(q)
    want_lens = torch.empty(3, dtype=torch.int32, device=DEV)

    def step():
        torch.add(c.lens, 1, out=want_lens)
        c.resize(seqs, want_lens)
        c.write(k, v, seqs)
        c.attention(q, seqs, out=out)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for i in range(20):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape).half())
        graph.replay()
        torch.cuda.synchronize()
        assert m.resize([0, 1, 2], [16 + i, 32 + i, 6 + i])
        m.write([0, 1, 2], [0, 1, 2, 3], k.double().cpu().numpy(), v.double().cpu().numpy())
        same_contents(c, m)
        want, bound = m.attention(q.double().cpu().numpy(), [0, 1, 2], [0, 1, 2, 3])
        err = np.abs(out.double().cpu().numpy() - want)
        assert (err <= 2.0 ** -11 * np.abs(want) + bound + 2.0 ** -24).all()
    assert c.poll_status() == 0


def test_two_caches_on_two_streams():
    a, ma = make(heads=2, group=4)
    b, mb = make(heads=2, group=4, fmt="e4m3")
    fill(a, ma, [600, 20], seed=1)
    fill(b, mb, [20, 700], seed=2)
    q = torch.randn(2, 1, 8, 128, device=DEV).half()
    seqs = ints([0, 1])
    wa, wb = a.attention(q, seqs).clone(), b.attention(q, seqs).clone()
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        ga, gb = torch.empty_like(q), torch.empty_like(q)
        sa.wait_stream(torch.cuda.current_stream())
        sb.wait_stream(torch.cuda.current_stream())
        a.attention(q, seqs, out=ga, stream=sa)
        b.attention(q, seqs, out=gb, stream=sb)
        torch.cuda.synchronize()
        assert torch.equal(ga, wa) and torch.equal(gb, wb)
