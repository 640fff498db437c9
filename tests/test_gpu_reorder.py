"""Reordering on the GPU: LESS's own state (less_reorder) and the paged cache (less_pages_reorder), against plain copies
and the model of pages_ref.py, exactly."""
import numpy as np
import pytest
import torch

from test_gpu_pages import DEV, fill, ints, make, same_contents, same_maps

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- #
# LESS's state
# --------------------------------------------------------------------------- #
def context(batch, layers=2, heads=3, slots=(5, 6), rank=8, dim=128, hidden=64, group=1, flags=0):
    from paper_2402_09398_b200 import binding as B
    g = torch.Generator().manual_seed(batch)
    shapes = {"w_phi1": (layers, heads * group, dim, hidden), "w_phi2": (layers, heads * group, hidden, rank),
              "w_psi1": (layers, heads, dim, hidden), "w_psi2": (layers, heads, hidden, rank),
              "w_psi3": (layers, heads, rank, rank)}
    w = {k: (torch.randn(s, generator=g) * 0.1).half().to(DEV) for k, s in shapes.items()}
    return B.LessContext(batch, layers, heads, dim, rank, hidden, *slots, 0, w, group=group, flags=flags)


def scramble(ctx, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = ctx.state_tensors()
    for k, t in st.items():
        if t.dtype == torch.int32:
            t.copy_(torch.randint(0, ctx.N + 1, t.shape, generator=g, device=DEV, dtype=torch.int32))
        else:
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
    return st


def snapshot(st):
    return {k: t.clone() for k, t in st.items()}


@pytest.mark.parametrize("batch,beams,kw", [
    (1, 1, {}), (4, 4, dict(layers=1, heads=8)), (6, 2, {}), (6, 3, dict(heads=1, layers=1)), (40, 8, dict(slots=(3, 10))),
    (64, 64, dict(layers=1, heads=2)), (5, 5, dict(dim=64, group=3, rank=16)), (12, 4, dict(slots=(100, 101), layers=3)),
    (100, 1, {}), (130, 130, dict(layers=1, heads=1))])
def test_state_follows_its_parents(batch, beams, kw):
    ctx = context(batch, **kw)
    rng = np.random.default_rng(batch)
    for turn in range(4):
        st = scramble(ctx, turn)
        before = snapshot(st)
        first = np.arange(batch) // beams * beams
        if turn == 3:                                      # a cycle through every row of a group
            parents = first + (np.arange(batch) - first + 1) % beams
        else:
            parents = first + rng.integers(0, beams, batch)
        ctx.reorder(ints(parents), beams=beams)
        for k in st:
            assert torch.equal(st[k], before[k][torch.from_numpy(parents).to(DEV)]), (k, turn)
    assert ctx.poll_status() == 0
    ctx.close()


def test_a_parent_of_another_group_changes_nothing():
    ctx = context(6)
    st = scramble(ctx)
    before = snapshot(st)
    for parents in ([0, 1, 2, 3, 4, 6], [0, 1, 2, 3, 4, -1], [0, 1, 3, 3, 3, 3]):
        ctx.reorder(ints(parents), beams=3)
        assert all(torch.equal(st[k], before[k]) for k in st)
        assert ctx.poll_status() == -8
    ctx.close()
    ctx = context(6)
    st = scramble(ctx)
    before = snapshot(st)
    ctx.reorder(ints([5, 4, 3, 2, 1, 0]))                  # one group is all
    assert all(torch.equal(st[k], before[k].flip(0)) for k in st) and ctx.poll_status() == 0
    with pytest.raises(ValueError):
        ctx.reorder(ints([0, 1, 2]))
    from paper_2402_09398_b200 import binding as B
    for beams in (0, 4, 4000):
        with pytest.raises(B.LessError):
            ctx.reorder(ints([0] * 6), beams=beams)
    ctx.close()


def test_record_views_are_the_exported_records():
    ctx = context(2)
    st = scramble(ctx)
    recs = ctx.export_state(range(ctx.instances))
    for i, r in enumerate(recs):
        b, l, h = i // 6, i // 3 % 2, i % 3
        n = r["count"]
        assert n == int(st["count"][b, l, h])
        for k in ("pos", "acc", "K", "V", "psi"):
            assert np.array_equal(st[k][b, l, h, :n].cpu().numpy(), r[k]), k
        assert np.array_equal(st["H"][b, l, h].cpu().numpy(), r["H"])
        assert np.array_equal(st["z"][b, l, h].cpu().numpy(), r["z"])
    ctx.close()


@pytest.mark.parametrize("kw", [dict(layers=1, heads=4), dict(layers=2, heads=16, hidden=512), dict(group=4, hidden=128),
                                dict(flags=2), dict(layers=1, heads=8, hidden=512, small="1")])
@pytest.mark.parametrize("captured", [False, True])
def test_steps_and_reorderings_back_to_back(monkeypatch, kw, captured):
    """Decode steps (of a few heads: as one launch) with reorderings between them, launched without a pause, against the
    same calls with a wait behind each: bit for bit."""
    kw = dict(kw)
    small = kw.pop("small", "0")
    monkeypatch.setenv("LESS_SMALL_STEP", small)
    batch, beams, steps = 4 if small == "1" else 8, 4, 24
    rng = np.random.default_rng(1)
    parents = [ints(np.arange(batch) // beams * beams + rng.integers(0, beams, batch)) for _ in range(steps)]
    results = []
    for wait in (True, False):
        ctx = context(batch, slots=(6, 6), **kw)
        L, H, G = ctx.cfg.layers, ctx.cfg.heads, ctx.group
        g = torch.Generator(device=DEV).manual_seed(3)
        outs = []
        qkv = [[torch.randn((batch, L, h, 128), generator=g, device=DEV).half() for h in (H * G, H, H)]
               for _ in range(steps)]
        torch.cuda.synchronize()
        for t in range(2):                                 # the first calls are direct
            outs.append(ctx.decode_step(*qkv[t]).clone())
            ctx.reorder(parents[t], beams=beams)

        def rest():
            for t in range(2, steps):
                outs.append(ctx.decode_step(*qkv[t]))
                if wait:
                    torch.cuda.synchronize()
                ctx.reorder(parents[t], beams=beams)
                if wait:
                    torch.cuda.synchronize()
        if captured and not wait:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                rest()
            graph.replay()
        else:
            rest()
        torch.cuda.synchronize()
        assert ctx.poll_status() == 0
        results.append(([o.clone() for o in outs], snapshot(ctx.state_tensors())))
        ctx.close()
    (a, sa), (b, sb) = results
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    live = torch.arange(12, device=DEV) < sa["count"][..., None]
    for k in sa:
        x, y = sa[k], sb[k]
        if k in ("pos", "acc"):
            x, y = x[live], y[live]
        elif k in ("K", "V", "psi"):
            x, y = x[live], y[live]
        assert torch.equal(x, y), k


# --------------------------------------------------------------------------- #
# the paged cache
# --------------------------------------------------------------------------- #
def model_reorder(m, seqs, parents):
    """The model's answer; False = refused."""
    n = len(seqs)
    rows, lens = m.table[seqs].copy(), m.lens[seqs].copy()
    refs = m.refs.copy()
    for row in rows:
        for p in row[row >= 0]:
            refs[p] -= 1
    heir = {}
    for i, a in enumerate(parents):
        if a == i or (a not in heir):
            heir[a] = i
    new, need = rows[parents].copy(), []
    for i, a in enumerate(parents):
        tail, part = lens[a] // m.pt, lens[a] % m.pt
        if part and new[i, tail] >= 0 and heir[a] != i:
            need.append((i, tail, new[i, tail], -(-part // 16)))
            new[i, tail] = -1
        for p in new[i][new[i] >= 0]:
            refs[p] += 1
    free = np.nonzero(refs == 0)[0]
    if len(need) > len(free):
        return False
    for (i, tail, src, used), dst in zip(need, free):
        new[i, tail], refs[dst] = dst, 1
        m.codes[:, dst, :, :, :used * 16 * m.D] = m.codes[:, src, :, :, :used * 16 * m.D]
        m.amax[:, dst, :, :, :used] = m.amax[:, src, :, :, :used]
    m.table[seqs], m.lens[seqs], m.refs[:] = new, lens[parents], refs
    return True


def everything(cache, model):
    same_maps(cache, model)
    assert np.array_equal(cache.codes.cpu().numpy(), model.codes)
    assert np.array_equal(cache.amax.double().cpu().numpy(), model.amax, equal_nan=True)


def test_groups_that_live_on_are_left_alone():
    ctx = context(40, slots=(50, 51))
    st = scramble(ctx)
    before = snapshot(st)
    parents = list(range(40))
    for turn in range(3):
        if turn == 1:
            parents[8:16] = [9, 9, 10, 15, 12, 13, 8, 8]
        if turn == 2:
            parents[39] = 32
        st = scramble(ctx, turn)
        before = snapshot(st)
        ctx.reorder(ints(parents), beams=8)
        assert all(torch.equal(st[k], before[k][torch.tensor(parents, device=DEV)]) for k in st)
    assert ctx.poll_status() == 0
    ctx.close()


@pytest.mark.parametrize("seed", range(8))
def test_a_search_in_the_paged_cache(seed):
    """Growth by a token, choice of parents, growth again: families share and part."""
    rng = np.random.default_rng(seed)
    pt, beams = [16, 32, 64, 128][seed % 4], [2, 3, 5][seed % 3]
    groups = 3
    n = groups * beams
    c, m = make(layers=2, heads=[1, 3][seed % 2], dim=[64, 128][seed // 4], pages=150, seqs=n + 3, seq_pages=6, pt=pt,
                fmt=["int8", "e4m3"][seed % 2])
    seqs = rng.permutation(n + 3)[:n].tolist()
    lens = np.repeat(rng.integers(0, 3 * pt, groups), beams)
    first = seqs[::beams]
    c.resize(ints(first), ints(lens[::beams]))
    assert m.resize(first, lens[::beams].tolist())
    m.codes[:] = rng.integers(0, 120, m.codes.shape)
    m.amax[:] = np.float32(rng.uniform(1, 2, m.amax.shape))
    c.codes.copy_(torch.from_numpy(m.codes))
    c.amax.copy_(torch.from_numpy(m.amax))
    parents = np.arange(n) // beams * beams               # at first all beams become copies of their group's first one
    for step in range(2 * pt // 3 + 8):
        c.reorder(ints(seqs), ints(parents))
        assert model_reorder(m, seqs, parents)
        if step % 7 == 0:
            everything(c, m)
        lens = np.minimum(m.lens[seqs] + 1, 6 * pt)
        c.resize(ints(seqs), ints(lens))
        assert m.resize(seqs, lens.tolist())
        if step == 5:
            c.trim(ints(seqs[:beams]), 0, pt)
            m.trim(seqs[:beams], 0, pt)
        parents = np.arange(n) // beams * beams + rng.integers(0, beams, n)
        if step % 5 == 4:
            parents = np.arange(n)
            parents[0], parents[n - 1] = n - 1, 0          # across groups, of other lengths
    everything(c, m)
    assert c.poll_status() == 0


def test_refusals_change_nothing():
    c, m = make(pages=12, seqs=7, seq_pages=4, pt=16)
    fill(c, m, [20, 33, 16, 0, 5])
    everything(c, m)
    for seqs, parents, code in (([0, 1, 7], [0, 1, 2], -8), ([0, 1, -1], [0, 1, 2], -8), ([0, 1, 2], [0, 1, 3], -8),
                                ([0, 1, 2], [0, -1, 2], -8), ([0, 1, 0], [0, 1, 2], -10)):
        c.reorder(ints(seqs), ints(parents))
        everything(c, m)
        c.resize(ints([4]), ints([6]))                    # until the status is read, nothing changes
        same_maps(c, m)
        assert c.poll_status() == code and c.poll_status() == 0
    # 2 + 3 + 1 + 1 pages are held, 5 free: seven copies of sequence 1 release 4 and need 6 last pages
    c2, m2 = make(pages=8, seqs=7, seq_pages=4, pt=16)
    fill(c2, m2, [33, 16, 0, 0, 0, 0, 0])
    assert not model_reorder(m2, list(range(7)), [0] * 7)
    c2.reorder(ints(range(7)), ints([0] * 7))
    everything(c2, m2)
    from paper_2402_09398_b200 import binding as B
    assert c2.poll_status() == B.LESS_ERR_PAGES_EXHAUSTED
    c2.reorder(ints(range(6)), ints([0] * 6))             # five last pages are free, one by release
    assert model_reorder(m2, list(range(6)), [0] * 6)
    everything(c2, m2)
    assert c2.poll_status() == 0
    with pytest.raises(ValueError):
        c2.reorder(ints([0, 1]), ints([0]))
    with pytest.raises(B.LessError):
        c2.reorder(ints([0] * 8), ints([0] * 8))


def test_many_entries_and_wide_tables():
    rng = np.random.default_rng(2)
    for n, seq_pages, pt in ((3000, 9, 16), (70, 700, 16), (1, 5, 64)):
        c, m = make(layers=1, heads=1, dim=64, pages=n * 4 + 800, seqs=n, seq_pages=seq_pages, pt=pt)
        lens = np.zeros(n, int)
        lens[::4] = rng.integers(0, 3 * pt, len(lens[::4]))
        lens[0] = min(seq_pages, 700) * pt - 3
        fill(c, m, lens.tolist())
        order = rng.permutation(n).tolist()
        for _ in range(2):
            parents = (rng.integers(0, n, n) // 4 * 4).tolist()
            parents[-1] = 0
            c.reorder(ints(order), ints(parents))
            assert model_reorder(m, order, parents)
            everything(c, m)
        assert c.poll_status() == 0


def test_more_sequences_than_the_bitmap_tells():
    c, m = make(layers=1, heads=1, dim=64, pages=64, seqs=65600, seq_pages=2, pt=16)
    order = [65599, 3, 65537, 1, 0]
    c.resize(ints(order), ints([20, 3, 16, 0, 31]))
    assert m.resize(order, [20, 3, 16, 0, 31])
    c.reorder(ints(order), ints([4, 4, 0, 0, 1]))
    assert model_reorder(m, order, [4, 4, 0, 0, 1])
    same_maps(c, m)
    c.reorder(ints([65599, 3, 65599]), ints([0, 1, 2]))
    same_maps(c, m)
    assert c.poll_status() == -10


def test_reorder_captured_with_the_writes_of_a_step():
    """resize, write and reorder of a step in one graph, replayed: as the model has it."""
    n = 6
    c, m = make(layers=1, heads=2, pages=60, seqs=n, seq_pages=5, pt=32)
    lens = [40, 40, 40, 70, 70, 70]
    fill(c, m, lens, seed=3)
    parents, lens_t, seqs = ints([0, 0, 1, 5, 5, 3]), ints(lens), ints(range(n))
    k, v = (torch.randn(n, 1, 2, 128, device=DEV).half() for _ in "kv")

    def step():
        lens_t.add_(1)
        c.resize(seqs, lens_t)
        c.write(k, v, seqs)
        c.reorder(seqs, parents)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(12):
        if turn:
            graph.replay()
        lens = [x + 1 for x in lens]
        assert m.resize(list(range(n)), lens)
        m.write(list(range(n)), list(range(n + 1)), k.double().cpu().numpy(), v.double().cpu().numpy())
        assert model_reorder(m, list(range(n)), [0, 0, 1, 5, 5, 3])
        same_contents(c, m)
    assert c.poll_status() == 0
