"""Attention of many new tokens over the paged cache (tensor-core kernel), against the model of pages_ref.py."""
import numpy as np
import pytest
import torch

from test_gpu_pages import DEV, HALF_STEP, attend, fill, ints, make, same_contents, same_maps

pytestmark = pytest.mark.gpu


def starts_of(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()


@pytest.mark.parametrize("dim,heads,group,pt,fmt,dtype", [
    (128, 1, 1, 64, "int8", torch.float16), (128, 1, 1, 16, "e4m3", torch.bfloat16),
    (64, 1, 1, 128, "int8", torch.bfloat16), (64, 2, 1, 32, "e4m3", torch.float16)])
@pytest.mark.parametrize("length,new", [(128, 128), (33, 33), (300, 40), (700, 700), (129, 129), (513, 257)])
def test_one_prompt(dim, heads, group, pt, fmt, dtype, length, new):
    c, m = make(layers=1, heads=heads, dim=dim, group=group, pt=pt, fmt=fmt, dtype=dtype, pages=-(-720 // pt) + 2,
                seq_pages=-(-720 // pt), seqs=1)
    fill(c, m, [length])
    attend(c, m, [0], [0, new], max_new=new)


@pytest.mark.parametrize("dim,heads,group,pt,fmt,dtype", [
    (128, 2, 4, 64, "int8", torch.bfloat16), (64, 1, 71, 64, "int8", torch.float16),
    (128, 1, 5, 32, "e4m3", torch.float16), (64, 3, 8, 16, "e4m3", torch.bfloat16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (37, 5), (150, 20), (100000, 3)])
def test_ragged_chunks(dim, heads, group, pt, fmt, dtype, window, sinks):
    """Long and short chunks, single tokens and an empty entry in one call: both kernels, each its own rows."""
    lens, new = [400, 90, 300, 20, 260], [130, 90, 1, 0, 70]
    c, m = make(layers=2, heads=heads, dim=dim, group=group, pt=pt, fmt=fmt, dtype=dtype, pages=100,
                seq_pages=-(-400 // pt))
    fill(c, m, lens)
    order = [2, 0, 3, 4, 1]
    attend(c, m, order, starts_of([new[i] for i in order]), max_new=max(new), layers=1, layer_begin=1, window=window,
           sinks=sinks)


def test_result_does_not_depend_on_the_hint():
    c, m = make(heads=1, group=2, pages=30)
    fill(c, m, [300, 200])
    for hint in (1, 16, 17, 100, 1 << 30, None):
        attend(c, m, [0, 1], [0, 60, 70], max_new=hint)


def test_more_tokens_than_the_sequence_has():
    c, m = make(heads=2, group=1, pages=30)
    fill(c, m, [0, 50, 20])
    attend(c, m, [0, 1, 2], [0, 40, 140, 540], max_new=400)


def test_trimmed_pages_are_not_seen():
    c, m = make(heads=1, group=2, pt=16, pages=60, seq_pages=30, fmt="e4m3")
    fill(c, m, [400, 130])
    c.trim(ints([0]), 20, 130)
    m.trim([0], 20, 130)
    attend(c, m, [0, 1], [0, 50, 100], max_new=50)
    attend(c, m, [0, 1], [0, 50, 100], max_new=50, window=60, sinks=20)


def test_scores_that_grow_and_value_magnitudes_far_apart():
    """Keys that get larger along the sequence (the reference moves many times), zero value blocks among others."""
    for dtype in (torch.float16, torch.bfloat16):
        c, m = make(heads=1, dim=128, group=4, pt=16, pages=60, seqs=2, seq_pages=40, dtype=dtype)
        fill(c, m, [600, 300])
        rng = np.random.default_rng(4)
        for s, n in ((0, 600), (1, 300)):
            for b in range(-(-n // 16)):
                m.amax[:, m.table[s, b], :, 0] = np.float32(0.5 * (1 + b))
                m.amax[:, m.table[s, b], :, 1] = np.float32(0.0 if b % 7 == 3 else 2.0 ** rng.integers(-9, 6))
        c.amax.copy_(torch.from_numpy(m.amax))
        attend(c, m, [0, 1], [0, 64, 364], max_new=300)
        m.amax[..., 1, :] = 0                               # all values are zero
        c.amax.copy_(torch.from_numpy(m.amax))
        got = attend(c, m, [0, 1], [0, 64, 364], max_new=300)
        assert (got[:364] == 0).all()


def test_same_bits_again_and_after_a_replay():
    c, m = make(heads=2, group=4, pages=40, dtype=torch.bfloat16)
    fill(c, m, [500, 700, 64])
    q = torch.randn(400, 1, 8, 128, device=DEV).bfloat16()
    seqs, starts = ints([0, 1, 2]), ints([0, 100, 399, 400])
    want = c.attention(q, seqs, starts, max_new=299).clone()
    assert torch.equal(want, c.attention(q, seqs, starts, max_new=299))
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.attention(q, seqs, starts, max_new=299, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_a_bad_query_stays_in_its_row_of_a_tile():
    c, m = make(heads=1, group=1, dtype=torch.bfloat16)
    fill(c, m, [200])
    q = torch.randn(200, 1, 1, 128, device=DEV).bfloat16()
    good = c.attention(q, ints([0]), ints([0, 200])).clone()
    q[77, 0, 0, 3] = float("inf")
    bad = c.attention(q, ints([0]), ints([0, 200]))
    keep = torch.arange(200, device=DEV) != 77
    assert torch.equal(bad[keep], good[keep]) and not torch.isfinite(bad[77]).all()


@pytest.mark.parametrize("dim,heads,group,new,window", [(128, 1, 4, 12, 0), (64, 2, 71, 1, 0), (128, 1, 128, 1, 500), (64, 1, 1, 300, 0)])
def test_keys_split_over_ctas(dim, heads, group, new, window):
    """Few rows, many keys: the key tiles of an item go to several CTAs, whose parts are joined."""
    lens = [3000, 1, 700]
    c, m = make(heads=heads, dim=dim, group=group, pt=64, pages=70, seqs=3, seq_pages=48, dtype=torch.bfloat16)
    fill(c, m, lens)
    n = [min(new, k) for k in lens]
    first = attend(c, m, [0, 1, 2], starts_of(n), max_new=new, window=window, sinks=3 if window else 0)
    again = attend(c, m, [0, 1, 2], starts_of(n), max_new=new, window=window, sinks=3 if window else 0)
    assert np.array_equal(first, again)


@pytest.mark.parametrize("skip", [1, 17, 700])
@pytest.mark.parametrize("new", [[3, 1], [90, 40]])
def test_rows_before_the_first_entry(skip, new):
    """starts[0] > 0: the rows before it belong to nobody; they are not read, and the output keeps its own."""
    lens = [100, 45]
    c, m = make(heads=2, group=4, pt=16, pages=40)
    fill(c, m, lens)
    want_k = np.random.default_rng(3).normal(size=(sum(new), 1, 2, 128)).astype(np.float16)
    want_v = np.random.default_rng(4).normal(size=(sum(new), 1, 2, 128)).astype(np.float16)
    pad = lambda x: torch.cat([torch.full((skip, *x.shape[1:]), float("nan"), dtype=c.dtype), torch.from_numpy(x)]).to(DEV)
    starts = starts_of(new)
    late = ints([skip + s for s in starts])
    c.write(pad(want_k), pad(want_v), ints([0, 1]), late)
    m.write([0, 1], starts, want_k.astype(np.float64), want_v.astype(np.float64))
    same_contents(c, m)
    q = np.random.default_rng(5).normal(size=(sum(new), 1, 8, 128)).astype(np.float16)
    out = torch.full((skip + sum(new), 1, 8, 128), 7.0, dtype=c.dtype, device=DEV)
    c.attention(pad(q), ints([0, 1]), late, max_new=max(new), out=out)
    assert (out[:skip] == 7.0).all()
    want, bound = m.attention(q.astype(np.float64), [0, 1], starts)
    err = np.abs(out[skip:].double().cpu().numpy() - want)
    assert (err <= HALF_STEP[c.dtype] * np.abs(want) + bound + 2.0 ** -24).all()
    assert c.poll_status() == 0


@pytest.mark.parametrize("new", [12, 300])                  # 12: keys are split over CTAs
@pytest.mark.parametrize("order", ["zero first", "small first", "large first", "zero among", "mixed"])
def test_value_magnitudes_of_any_distance(order, new):
    """A block's share of the probabilities does not depend on the size of its values, its values not on other blocks'."""
    c, m = make(heads=1, dim=64, group=4, pt=16, pages=130, seqs=1, seq_pages=130, dtype=torch.bfloat16)
    fill(c, m, [2000])
    rng = np.random.default_rng(8)
    b = np.arange(125)
    e = {"zero first": np.where(b < 3, -np.inf, -30.0), "small first": np.where(b < 60, -95.0, 40.0),
         "large first": np.where(b < 60, 40.0, -95.0), "zero among": np.where(b % 5 == 2, -np.inf, -30.0 - b % 3),
         "mixed": rng.integers(-99, 90, 125).astype(float)}[order]
    m.amax[0, m.table[0, :125], 0, 1, 0] = np.float32(np.exp2(e))
    c.amax.copy_(torch.from_numpy(m.amax))
    q = torch.from_numpy(rng.normal(size=(new, 1, 4, 64))).bfloat16()
    got = c.attention(q.to(DEV), ints([0]), ints([0, new]), max_new=new).double().cpu().numpy()
    want, bound = m.attention(q.double().numpy(), [0], [0, new])
    assert (np.abs(got - want) <= HALF_STEP[c.dtype] * np.abs(want) + bound).all()


def test_more_entries_than_a_grid_dimension_and_than_the_bitmap():
    """70 000 sequences, nearly all of them empty, all in one call; lists with duplicates among them."""
    n = 70000
    c, m = make(heads=1, dim=64, group=1, pt=16, pages=80, seqs=n, seq_pages=8)
    live, lens = [0, 65536, 7, 65535, n - 1], [100, 70, 16, 128, 1]
    c.resize(ints(live + [7, 0]), ints(lens + [99, 3]))
    assert m.resize(live + [7, 0], lens + [99, 3])
    same_maps(c, m)
    rng = np.random.default_rng(2)
    k, v = (rng.normal(size=(sum(lens), 1, 1, 64)).astype(np.float16) for _ in range(2))
    c.write(torch.from_numpy(k).to(DEV), torch.from_numpy(v).to(DEV), ints(live), ints(starts_of(lens)))
    m.write(live, starts_of(lens), k.astype(np.float64), v.astype(np.float64))
    c.fork(ints([0, 65536]), ints([1, 66000]))
    m.fork([0, 65536], [1, 66000])
    same_contents(c, m)
    for src, dst in (([0, 0], [5, 5]), ([0, 9], [9, 11])):  # a destination twice; one that is a source
        assert c.poll_status() == 0
        c.fork(ints(src), ints(dst))
        assert c.poll_status() == -10
        same_maps(c, m)
    order = rng.permutation(n)
    new = np.ones(n, int)
    new[np.isin(order, [0, 65536, 66000])] = 70
    attend(c, m, order.tolist(), starts_of(new), max_new=70)


def test_results_belong_to_the_stream_that_writes_them():
    c, m = make(heads=2, group=2, pages=20)
    fill(c, m, [200])
    q = torch.randn(1, 1, 4, 128, device=DEV).half()
    want = c.attention(q, ints([0]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.attention(q, ints([0]), stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    place = got.data_ptr()
    del got                                                 # back to that stream's memory, not to the current one's
    assert torch.empty_like(want).data_ptr() != place
    with torch.cuda.stream(side):
        assert torch.empty_like(want).data_ptr() == place


def test_a_sequence_listed_twice():
    c, m = make(heads=2, group=4, pages=30)
    fill(c, m, [300, 200])
    attend(c, m, [1, 0, 1, 1], starts_of([1, 1, 1, 1]), max_new=1, tail=0)
    attend(c, m, [1, 0, 1, 0], starts_of([60, 3, 60, 80]), max_new=80, window=50, sinks=3)


def test_offsets_beyond_32_bits():
    """The same contents at the end of a pool of 5 GB and in a small one: the same bits."""
    from paper_2402_09398_b200 import binding as B
    lens, far = [500, 77, 130], 20000 - 20
    caches = []
    for pages in (20000, 20):
        c = B.PagedCache(2, 8, 128, pages, 4, 8, group=4, page_tokens=64, dtype=torch.bfloat16)
        c.refs[:pages - 20] = 1
        c.codes[:, pages - 20:] = 0                         # bytes that no token owns compare equal
        c.amax[:, pages - 20:] = 0
        c.resize(ints([0, 1, 2]), ints(lens))
        caches.append(c)
    big, small = caches
    assert big.codes.numel() > 2 ** 32 and torch.equal(big.table[:3] - far * (big.table[:3] >= 0).int(), small.table[:3])
    starts = ints(starts_of(lens))
    k, v = (torch.randn(sum(lens), 2, 8, 128, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn(sum(lens), 2, 32, 128, device=DEV).bfloat16()
    for c in caches:
        c.write(k, v, ints([0, 1, 2]), starts)
        c.fork(ints([1]), ints([3]))
        c.resize(ints([3, 2]), ints([78, 131]))
        c.write(k[:2], v[:2], ints([3, 2]))
    assert torch.equal(big.lens, small.lens)

    def same(pages):
        if pages:
            assert torch.equal(big.refs[far:], small.refs)
            assert torch.equal(big.codes[:, far:], small.codes) and torch.equal(big.amax[:, far:], small.amax)
        for args in ((q[:4], ints([0, 1, 2, 3]), None, 1), (q, ints([0, 1, 2]), starts, 500)):
            a, b = (c.attention(*args) for c in caches)
            assert torch.isfinite(b).all() and torch.equal(a, b)
        assert [c.poll_status() for c in caches] == [0, 0]

    same(True)
    big.refs[:far] = 0
    for c in caches:
        c.resize(ints([1]), ints([0]))
        c.compact()
    assert int(big.table.max()) < 20
    same(False)
