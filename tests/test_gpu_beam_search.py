"""Beam search as it is used: attention, selection, reordering, growth and write of every step, over the paged cache and over
LESS's own state, against the models of each part fed with the same inputs."""
import numpy as np
import pytest
import torch

import beams_ref
from test_gpu_pages import DEV, ints, make, same_contents
from test_gpu_pages_shared import attend, reach
from test_gpu_reorder import context, model_reorder

pytestmark = pytest.mark.gpu


def chosen(choice, logits, scores, ended, end, beams):
    want = beams_ref.select(logits.double().cpu().numpy(), scores.double().cpu().numpy(), ended.cpu().numpy(), end, beams,
                            65504.0)
    assert np.array_equal(choice.tokens.cpu().numpy(), want[1]) and np.array_equal(choice.parents.cpu().numpy(), want[2])
    assert np.array_equal(choice.ended.cpu().numpy(), want[3])
    return want[2].ravel().tolist()


@pytest.mark.parametrize("group,fmt", [(1, "int8"), (4, "e4m3")])
def test_search_over_the_paged_cache(group, fmt):
    from paper_2402_09398_b200 import binding as B
    groups, beams, heads, dim, vocab, pt = 3, 4, 2, 64, 500, 16
    n = groups * beams
    rng = np.random.default_rng(group)
    c, m = make(layers=1, heads=heads, dim=dim, pages=220, seqs=n + 2, seq_pages=reach(1, 1, heads, dim, pt), group=group,
                pt=pt, fmt=fmt)
    g = torch.Generator(device=DEV).manual_seed(5)
    embed = torch.randn(vocab, 3, heads * dim, generator=g, device=DEV).half()
    head = torch.randn(heads * group * dim, vocab, generator=g, device=DEV) * 0.3
    seqs = rng.permutation(n + 2)[:n].tolist()
    lens = np.repeat([37, 80, 5], beams)
    # the prompts, once each, and a fork for every beam
    firsts, others = seqs[::beams], [s for i, s in enumerate(seqs) if i % beams]
    c.resize(ints(firsts), ints(lens[::beams]))
    m.resize(firsts, lens[::beams].tolist())
    starts = np.concatenate([[0], np.cumsum(lens[::beams])]).astype(int).tolist()
    k, v = (torch.randn(starts[-1], 1, heads, dim, generator=g, device=DEV).half() for _ in "kv")
    c.write(k, v, ints(firsts), ints(starts))
    m.write(firsts, starts, k.double().cpu().numpy(), v.double().cpu().numpy())
    src = [s for s in firsts for _ in range(beams - 1)]
    c.fork(ints(src), ints(others))
    m.fork(src, others)
    sel = B.BeamSelect(groups, beams, vocab, dtype=torch.float16, end_token=7)
    scores = torch.full((groups, beams), -float("inf"), device=DEV)
    scores[:, 0] = 0.0
    ended = torch.zeros(groups, beams, dtype=torch.bool, device=DEV)
    bounds, s_t, b_t = list(range(0, n + 1, beams)), ints(seqs), ints(range(0, n + 1, beams))
    q = torch.randn(n, 1, heads * group, dim, generator=g, device=DEV).half()
    for step in range(24):
        out = c.shared_attention(q, s_t, b_t, max_group=beams)
        if step % 6 == 0:
            attend(c, m, seqs, bounds, tail=0, q=q.cpu(), max_group=beams)
        logits = (out.reshape(groups, beams, -1).float() @ head).half()
        if step == 18:
            logits[1:, 0, 7] = 60.0                        # the best beams of two texts end
        choice = c.beam_step(sel, logits, scores, s_t, ended)
        assert model_reorder(m, seqs, chosen(choice, logits, scores, ended, 7, beams))
        scores, ended = choice.scores, choice.ended
        grown = m.lens[seqs] + 1
        c.resize(s_t, ints(grown))
        assert m.resize(seqs, grown.tolist())
        e = embed[choice.tokens.view(-1).long().clamp(min=0)]
        kv = [e[:, i].reshape(n, 1, heads, dim).contiguous() for i in (0, 1)]
        c.write(kv[0], kv[1], s_t)
        m.write(seqs, list(range(n + 1)), kv[0].double().cpu().numpy(), kv[1].double().cpu().numpy())
        q = e[:, 2].reshape(n, 1, heads, 1, dim).expand(n, 1, heads, group, dim).reshape(n, 1, heads * group, dim).contiguous()
    same_contents(c, m)
    assert c.poll_status() == 0 and ended.any()


@pytest.mark.parametrize("small_step", ["0", "1"])
def test_search_over_less_state(monkeypatch, small_step):
    """Against a second context whose rows are exchanged by records through the host."""
    from paper_2402_09398_b200 import binding as B
    monkeypatch.setenv("LESS_SMALL_STEP", small_step)
    groups, beams, vocab, L, H = 1, 4, 300, 1, 3
    n = groups * beams
    a, b = (context(n, layers=L, heads=H, slots=(4, 5), hidden=128) for _ in "ab")
    sel = B.BeamSelect(groups, beams, vocab, dtype=torch.float16, end_token=2)
    g = torch.Generator(device=DEV).manual_seed(1)
    head = torch.randn(L * H * 128, vocab, generator=g, device=DEV)
    embed = torch.randn(vocab, 3, L, H, 128, generator=g, device=DEV).half()
    scores = torch.zeros(groups, beams, device=DEV)
    ended = torch.zeros(groups, beams, dtype=torch.bool, device=DEV)
    tokens = torch.arange(n, device=DEV)
    per = L * H
    for step in range(20):
        q, k, v = (embed[tokens, i].contiguous() for i in range(3))
        out, twin = a.decode_step(q, k, v), b.decode_step(q, k, v)
        assert torch.equal(out, twin)
        logits = (out.reshape(groups, beams, -1) @ head).half()
        choice = a.beam_step(sel, logits, scores, ended)
        parents = chosen(choice, logits, scores, ended, 2, beams)
        recs = b.export_state(range(n * per))
        b.import_state(range(n * per), [recs[p * per + i] for p in parents for i in range(per)])
        scores, ended, tokens = choice.scores, choice.ended, choice.tokens.view(-1).long().clamp(min=0)
    assert a.poll_status() == 0 and b.poll_status() == 0
    with pytest.raises(ValueError):
        a.beam_step(B.BeamSelect(1, 3, vocab), logits[:, :3], scores[:, :3])
    a.close(), b.close()
