"""What the paged cache does beside an error: which entries of a call are carried out, and which calls after it."""
import numpy as np
import pytest
import torch

from test_gpu_pages import DEV, ints, make, same_contents, same_maps

pytestmark = pytest.mark.gpu
BOUNDS, STATE = -8, -10


def rows(rng, n, heads, dtype=torch.float16, dim=128):
    return torch.from_numpy(rng.normal(size=(n, 2, heads, dim))).to(dtype)


@pytest.mark.parametrize("bad,code", [(-1, BOUNDS), (70, BOUNDS), (64, STATE)])   # no sequence; one whose page is shared
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("at", [0, 30, 63])
def test_write_carries_out_every_entry_but_the_refused_one(bad, code, many, at):
    n, heads = 64, 3
    c, m = make(layers=2, heads=heads, dim=128, pages=700, seqs=66, seq_pages=10, pt=16)
    rng = np.random.default_rng(at)
    new = [int(x) for x in rng.integers(1, 60, n)] if many else [1] * n
    lens = [int(x) + k for x, k in zip(rng.integers(0, 80, n), new)]
    c.resize(ints(range(n)), ints(lens))
    m.resize(list(range(n)), lens)
    c.resize(ints([64]), ints([32]))
    m.resize([64], [32])
    c.fork(ints([64]), ints([65]))
    m.fork([64], [65])
    # sequence `at`'s rows are the refused entry's: it keeps what it has
    seqs = list(range(n))
    seqs[at] = bad
    starts = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
    for k in range(20):
        kk, vv = rows(rng, starts[-1], heads), rows(rng, starts[-1], heads)
        c.write(kk.to(DEV), vv.to(DEV), ints(seqs), ints(starts) if many else None)
        keep = [i for i in range(n) if i != at]
        for i in keep:
            m.write([i], [0, new[i]], *(x[starts[i]:starts[i + 1]].double().numpy() for x in (kk, vv)))
        if k % 5 == 4:                                     # a write that follows goes on, others wait
            c.resize(ints([0]), ints([0]))
            c.write(vv.to(DEV), kk.to(DEV), ints(seqs), ints(starts) if many else None)
            # (an entry with more tokens than its sequence has is out of bounds before its page is looked at)
            assert c.poll_status() == (BOUNDS if new[at] > 32 else code) and c.poll_status() == 0
            for i in range(n):
                for b in range((lens[i] - new[i]) // 16 if i != at else 10 ** 9, -(-lens[i] // 16)):
                    page, inner = m.table[i, b], 0
                    assert np.array_equal(c.codes[:, page].cpu().numpy(), m.codes[:, page]), (i, b)
                    assert np.array_equal(c.amax[:, page].double().cpu().numpy(), m.amax[:, page])
            same_maps(c, m)


def test_trim_carries_out_every_entry_but_the_refused_one():
    n = 900
    for k in range(10):
        c, m = make(heads=1, dim=64, pages=n * 4, seqs=n, seq_pages=4, pt=16)
        c.resize(ints(range(n)), ints([64] * n))
        m.resize(list(range(n)), [64] * n)
        order = np.random.default_rng(k).permutation(n).tolist()
        c.trim(ints([n] + order[:-1]), 0, 20)
        m.trim(order[:-1], 0, 20)
        c.trim(ints(order[-1:]), 0, 20)                    # goes on as well
        m.trim(order[-1:], 0, 20)
        c.compact()                                        # does not
        same_maps(c, m)
        assert c.poll_status() == BOUNDS and c.poll_status() == 0


def test_other_calls_wait_until_the_error_of_a_write_has_been_read():
    c, m = make(heads=2, pages=20, seqs=5, seq_pages=4, pt=16)
    c.resize(ints([0, 1]), ints([20, 30]))
    m.resize([0, 1], [20, 30])
    x = torch.ones(1, 1, 2, 128, device=DEV).half()
    c.write(x, x, ints([9]))
    c.fork(ints([0]), ints([2]))
    c.write(x, x, ints([0]))                               # the fork has seen the error: from now on nothing is written
    c.trim(ints([1]), 0, 1)
    c.resize(ints([3]), ints([5]))
    same_maps(c, m)
    assert (c.codes == 0).all() and c.poll_status() == BOUNDS and c.poll_status() == 0
    c.write(x, x, ints([0]))
    assert (c.codes != 0).any() and c.poll_status() == 0


def test_starts_that_descend_are_reported():
    """Also where the entry in question is one that a search for rows never meets."""
    c, m = make(heads=1, group=71, dim=64, pages=300, seqs=4, seq_pages=64, pt=16)
    c.resize(ints([0, 1, 2, 3]), ints([1000] * 4))
    x = torch.zeros(1000, 1, 1, 64, device=DEV).half()
    q = torch.zeros(1000, 1, 71, 64, device=DEV).half()
    assert c.poll_status() == 0
    for starts in ([0, 1000, 0, 500, 1000], [0, 0, 1000, 999, 1000], [500, 0, 1000, 1000, 1000]):
        c.write(x, x, ints([0, 1, 2, 3]), ints(starts))
        assert c.poll_status() == BOUNDS, starts
        c.attention(q, ints([0, 1, 2, 3]), ints(starts), max_new=1000)
        assert c.poll_status() == BOUNDS, starts
        c.attention(q, ints([0, 1, 2, 3]), ints(starts), max_new=1)
        assert c.poll_status() == BOUNDS, starts


def test_entries_that_overlap_more_often_than_can_be_counted():
    """starts 0, 1024, 0, 1024, ...: 2^32 items of eight rows.  Nothing is done (an index of an item would be any number)."""
    c, m = make(layers=16, heads=8, group=8, dim=64, pages=64, seqs=1, seq_pages=64, pt=16)
    c.resize(ints([0]), ints([1000]))
    q = torch.zeros(1024, 16, 64, 64, device=DEV).half()
    n = 1 << 16
    out = torch.full_like(q, 3.0)
    c.attention(q, torch.zeros(n, dtype=torch.int32, device=DEV), ints([0, 1024] * (n // 2) + [0]), max_new=1, out=out)
    assert c.poll_status() == BOUNDS
    assert (out == 3.0).all()


@pytest.mark.parametrize("n", [2048, 2049, 5000])
@pytest.mark.parametrize("many", [False, True])
def test_first_entry_of_a_sequence_counts_in_long_lists(n, many):
    """Also beside entries that name no sequence; a list of more than 2048 entries is looked up in another way."""
    c, m = make(layers=1, heads=1, dim=64, pages=n, seqs=n, seq_pages=1, pt=16)
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(2, 17, n)]
    c.resize(ints(range(n)), ints(lens))
    m.resize(list(range(n)), lens)
    seqs = rng.integers(0, n, n)
    seqs[rng.integers(0, n, 3)] = (-1, n, 2 ** 31 - 1)
    k, v = (torch.from_numpy(rng.normal(size=(n, 1, 1, 64))).half() for _ in range(2))
    c.write(k.to(DEV), v.to(DEV), ints(seqs), ints(range(n + 1)) if many else None)
    first = [i for i in np.unique(seqs, return_index=True)[1] if 0 <= seqs[i] < n]
    for i in first:
        m.write([int(seqs[i])], [0, 1], k[i:i + 1].double().numpy(), v[i:i + 1].double().numpy())
    same_contents(c, m)
    assert c.poll_status() == BOUNDS


@pytest.mark.parametrize("call", ["write", "attention", "resize"])
def test_inputs_may_be_dropped_while_another_stream_waits_to_read_them(call):
    c, m = make(heads=2, group=2, pages=40, seqs=4, seq_pages=12)
    rng = np.random.default_rng(1)
    k, v = (torch.from_numpy(rng.normal(size=(300, 1, 2, 128))).half() for _ in range(2))
    q = torch.from_numpy(rng.normal(size=(300, 1, 4, 128))).half().to(DEV)
    seqs, starts = ints([0, 1]), ints([0, 100, 300])
    c.resize(seqs, ints([100, 200]))
    m.resize([0, 1], [100, 200])
    c.write(k.to(DEV), v.to(DEV), seqs, starts)
    m.write([0, 1], [0, 100, 300], k.double().numpy(), v.double().numpy())
    want = c.attention(q, seqs, starts, max_new=200)
    side = torch.cuda.Stream()
    kd, vd, qd, lens = v.to(DEV), k.to(DEV), q.clone(), ints([150, 200])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)                     # some 50 ms
    if call == "write":
        c.write(kd, vd, seqs, starts, stream=side)
        m.write([0, 1], [0, 100, 300], v.double().numpy(), k.double().numpy())
    elif call == "attention":
        got = c.attention(qd, seqs, starts, max_new=200, stream=side)
    else:
        c.resize(seqs, lens, stream=side)
        m.resize([0, 1], [150, 200])
    old = [t.data_ptr() for t in (kd, vd, qd, lens)]
    shapes = [(t.shape, t.dtype) for t in (kd, vd, qd, lens)]
    del kd, vd, qd, lens
    new = [torch.zeros(s, dtype=d, device=DEV) for s, d in shapes for _ in range(2)]     # on the current stream, at once
    side.synchronize()
    if call == "attention":
        assert torch.equal(got, want)
    else:
        same_contents(c, m)
    used = {"write": old[:2], "attention": old[2:3], "resize": old[3:]}[call]
    assert not set(used) & {t.data_ptr() for t in new}
    assert c.poll_status() == 0


def test_calls_on_a_named_stream_can_be_captured():
    c, m = make(heads=2, group=2, pages=40, seqs=4, seq_pages=12)
    k = torch.randn(2, 1, 2, 128, device=DEV).half()
    q, seqs, lens = torch.randn(2, 1, 4, 128, device=DEV).half(), ints([0, 1]), ints([0, 0])
    out = torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        lens.add_(1)
        c.resize(seqs, lens, stream=side)
        c.write(k, k.neg(), seqs, stream=side)             # the graph's own memory, dropped at once
        c.attention(q, seqs, out=out, stream=side)
    for i in range(1, 40):
        graph.replay()
        m.resize([0, 1], [i, i])
        m.write([0, 1], [0, 1, 2], k.double().cpu().numpy(), -k.double().cpu().numpy())
    torch.cuda.synchronize()
    same_contents(c, m)
    assert torch.equal(out, c.attention(q, seqs)) and c.poll_status() == 0
