"""Beam search's selection on the GPU against the 64-bit model of beams_ref.py: tokens, parents and ends exactly, scores
to half a step of fp32 plus the error of a sum (kernel comment: below 2.8e-6 of a logarithm)."""
import numpy as np
import pytest
import torch

import beams_ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def make(groups, beams, vocab, keep=None, dtype=torch.float16, end_token=-1):
    from paper_2402_09398_b200 import binding as B
    return B.BeamSelect(groups, beams, vocab, keep=keep, dtype=dtype, end_token=end_token)


def random_inputs(groups, beams, vocab, dtype, seed=0, pad=0, shift=0):
    """logits with `pad` elements between rows, the first row `shift` elements behind an aligned address."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.randn(groups * beams * (vocab + pad) + shift, generator=g) * 2.5
    flat = flat.to(dtype).to(DEV)
    logits = flat[shift:].view(groups, beams, vocab + pad)[:, :, :vocab]
    scores = (-5.0 * torch.rand((groups, beams), generator=g)).to(DEV)
    return logits, scores


def check(sel, logits, scores, ended=None, got=None):
    got = sel.select(logits, scores, ended) if got is None else got
    want = beams_ref.select(logits.double().cpu().numpy(), scores.double().cpu().numpy(),
                            None if ended is None else ended.cpu().numpy(), sel.desc.end_token, sel.keep,
                            torch.finfo(sel.dtype).max)
    assert np.array_equal(got.tokens.cpu().numpy(), want[1])
    assert np.array_equal(got.parents.cpu().numpy(), want[2])
    assert np.array_equal(got.ended.cpu().numpy(), want[3])
    a, b = got.scores.double().cpu().numpy(), want[0]
    some = np.isfinite(b)
    assert np.array_equal(some, np.isfinite(a))
    assert (np.abs(a[some] - b[some]) <= np.abs(b[some]) * 2.0 ** -24 + 2.8e-6).all()
    return got


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("groups,beams,vocab,keep", [(1, 4, 32000, 4), (3, 5, 50257, 10), (2, 1, 1, 1), (2, 3, 2, 8),
                                                     (1, 64, 700, 128), (7, 2, 4097, 33), (40, 8, 1003, 16),
                                                     (1, 1, 300001, 32), (1, 3, 129, 128), (300, 3, 63, 3)])
def test_selection(dtype, groups, beams, vocab, keep):
    sel = make(groups, beams, vocab, keep, TYPES[dtype], end_token=vocab // 2)
    check(sel, *random_inputs(groups, beams, vocab, TYPES[dtype], seed=vocab))


@pytest.mark.parametrize("groups,beams,vocab", [(700, 3, 700), (5000, 1, 90), (130, 16, 3), (2, 2, 400000), (33, 62, 40)])
def test_many_rows_and_long_ones(groups, beams, vocab):
    """More rows than are counted, rows of which a CTA takes several, rows of which many CTAs take a stretch."""
    sel = make(groups, beams, vocab, dtype=torch.float16, end_token=vocab - 1)
    logits, scores = random_inputs(groups, beams, vocab, torch.float16, seed=groups)
    g = torch.Generator().manual_seed(1)
    ended = (torch.rand((groups, beams), generator=g) < 0.2).to(DEV)
    scores[torch.rand((groups, beams), generator=g).to(DEV) < 0.3] = -float("inf")
    check(sel, logits, scores, ended)
    check(sel, logits, scores)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 7), (13, 2)])
def test_rows_at_any_address(dtype, pad, shift):
    for vocab in (5, 8, 1000, 9001):
        sel = make(2, 3, vocab, 5, TYPES[dtype])
        check(sel, *random_inputs(2, 3, vocab, TYPES[dtype], seed=pad, pad=pad, shift=shift))


def test_largest_beam_sums_do_not_overflow_an_index():
    """Rows whose elements lie beyond 2^31."""
    rows, vocab = 3, 1001
    stride = (1 << 30) + 24
    flat = torch.empty(2 * stride + vocab, dtype=torch.float16, device=DEV)
    logits = flat.as_strided((1, rows, vocab), (rows * stride, stride, 1))
    logits.copy_(torch.randn(1, rows, vocab))
    check(make(1, rows, vocab, 6), logits, torch.tensor([[-1.0, -1.5, -0.5]], device=DEV))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_beams_that_do_not_exist_or_have_ended(dtype):
    groups, beams, vocab = 6, 5, 2000
    sel = make(groups, beams, vocab, 9, TYPES[dtype], end_token=7)
    logits, scores = random_inputs(groups, beams, vocab, TYPES[dtype], seed=4)
    ended = torch.zeros(groups, beams, dtype=torch.bool, device=DEV)
    scores[0, 1:] = -float("inf")
    scores[1] = -float("inf")                             # nobody
    ended[2, ::2] = True
    ended[3] = True                                       # five candidates for nine places
    scores[4, 2], scores[4, 3] = float("nan"), float("inf")
    ended[4, 4] = True
    ended[5, 0] = True
    scores[5, 0] = -float("inf")
    logits[2, 0] = float("nan")                           # not looked at
    logits[5, 2] = -float("inf")
    logits[5, 3, 3:] = float("nan")
    got = check(sel, logits, scores, ended)
    assert got.tokens[1].eq(-1).all() and got.parents[1].tolist() == [5, 6, 7, 8, 9, 9, 9, 9, 9]


@pytest.mark.parametrize("dtype", list(TYPES))
def test_ties_and_crowds(dtype):
    """Equal logits, ascending and descending rows, equal beams: more at the bar than a list holds."""
    groups, beams, vocab = 7, 3, 30011
    sel = make(groups, beams, vocab, 11, TYPES[dtype])
    logits = torch.zeros(groups, beams, vocab, dtype=TYPES[dtype], device=DEV)
    up = torch.arange(vocab, device=DEV, dtype=torch.float64) / vocab * 4
    logits[1] = up.to(TYPES[dtype])
    logits[2] = up.flip(0).to(TYPES[dtype])
    logits[3, :, ::2] = -0.0
    logits[4] = torch.randn(vocab, generator=torch.Generator().manual_seed(5)).to(TYPES[dtype])
    logits[5, 0, 12345], logits[5, 1, 12345], logits[5, 2, 9] = 1.0, 1.0, 1.0
    logits[6, :, :9000] = -float("inf")                   # first tiles without candidates
    scores = torch.full((groups, beams), -0.5, device=DEV)
    check(sel, logits, scores)
    scores[4] = torch.tensor([-0.5, -0.5 - 2.0 ** -24, -0.5 + 2.0 ** -24], device=DEV)   # the order hangs on these
    check(sel, logits, scores)
    scores[4] = torch.tensor([-0.5, -0.5, -0.5 + 2.0 ** -24], device=DEV)
    check(sel, logits, scores)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("peak", [3.0, 9.0, 20.0, 36.0])
def test_order_of_beams_whose_peaks_come_late(dtype, peak):
    """The same logits in two orders, the largest among the first ones or far behind them (where it is added relative to a
    reference up to 2^52 smaller), and scores that differ by some 1e-7: the order is that of the 64-bit values."""
    groups, vocab = 320, 20000                            # a stretch a row
    g = torch.Generator().manual_seed(int(peak))
    logits = torch.randn(groups, 1, vocab, generator=g).repeat(1, 2, 1)
    logits[:, 0, 15000] = peak + 3 * torch.rand(groups, generator=g)
    logits[:, 1, 15000] = logits[:, 0, 5]
    logits[:, 1, 5] = logits[:, 0, 15000]
    first = torch.randint(24, 60, (groups,), generator=g)
    apart = torch.randint(1, 24, (groups,), generator=g) * (2 * torch.randint(0, 2, (groups,), generator=g) - 1)
    scores = -0.5 - torch.stack([first, first + apart], 1) * 2.0 ** -24
    sel = make(groups, 2, vocab, 2, TYPES[dtype])
    check(sel, logits.to(TYPES[dtype]).to(DEV), scores.to(DEV))


def test_crowds_with_many_kept():
    sel = make(2, 2, 40000, 128, torch.float32)
    logits = torch.zeros(2, 2, 40000, device=DEV)
    logits[1] = torch.arange(40000, device=DEV).float() * 1e-4
    check(sel, logits, torch.zeros(2, 2, device=DEV))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_infinities_and_extremes(dtype):
    most = torch.finfo(TYPES[dtype]).max
    sel = make(6, 2, 5000, 4, TYPES[dtype])
    logits, scores = random_inputs(6, 2, 5000, TYPES[dtype], seed=9)
    logits[0, 0, 17] = float("inf")
    logits[0, 0, 4000] = most                             # as large as the infinity counts
    logits[1] = -most
    logits[2, 0, :8] = most
    logits[2, 1, 4990:] = most
    logits[3, 0] = logits[3, 0].clamp(max=0)
    logits[3, 0, 4999] = 60000.0                          # the reference moves late
    logits[4, :, 1::2] = float("nan")
    logits[5] = -float("inf")
    logits[5, 1, 4999] = -most
    check(sel, logits, scores)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_masked_beginnings_and_references_that_move(dtype):
    """Stretches that begin with masked or NaN logits, references far below what follows, the type's lowest values beside
    masked ones."""
    most = torch.finfo(TYPES[dtype]).max
    vocab = 70001                                         # several tiles of 16-byte pieces
    sel = make(9, 2, vocab, 12, TYPES[dtype], end_token=0)
    logits, scores = random_inputs(9, 2, vocab, TYPES[dtype], seed=2)
    scores = scores[:1].repeat(9, 1).contiguous()
    logits[0, 0, :40000] = -float("inf")
    logits[0, 1, :69990] = float("nan")
    logits[1, :, :50000] -= 3000.0                        # rises by more than the reference reaches
    logits[2, :, ::3] = -float("inf")
    logits[2, :, 1::3] = -most
    logits[3] = -float("inf")
    logits[3, 0, 69999] = -most
    logits[3, 1, 5] = -most
    logits[4] = -most
    logits[4, 0, 60000:] = -float("inf")
    logits[5] = logits[5] * 1e-3 + 40000.0                # all rounded to few values
    logits[6, :, 30000] = float("inf")
    logits[6, 1, 60000] = most
    logits[7] = torch.linspace(-20, 20, vocab).to(TYPES[dtype])
    logits[8] = torch.linspace(0, -90, vocab).to(TYPES[dtype])
    check(sel, logits, scores)


@pytest.mark.parametrize("seed", range(4))
def test_beams_closer_than_fp32_tells_apart(seed):
    """The same logits in every beam, scores a few steps of 64-bit arithmetic's visible distance apart: the order is that of
    the scores, of equal ones that of the beams."""
    g = torch.Generator().manual_seed(seed)
    beams, vocab = 8, 20000
    sel = make(4, beams, vocab, 16, torch.float32)
    logits = (torch.randn(4, 1, vocab, generator=g) * 3).expand(4, beams, vocab).contiguous().to(DEV)
    steps = torch.randint(-2, 3, (4, beams), generator=g)
    scores = (-1.0 + steps * 2.0 ** -23).to(DEV)
    check(sel, logits, scores)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("seed", range(6))
def test_equal_beams_at_different_addresses(dtype, seed):
    """Rows of the same logits, each at another alignment: exact ties, the lowest beam first."""
    beams, vocab = 7, [501, 8191, 20001][seed % 3]
    sel = make(2, beams, vocab, 30, TYPES[dtype])
    g = torch.Generator().manual_seed(seed)
    logits = (torch.randn(2, 1, vocab, generator=g) * 2.5).to(TYPES[dtype]).expand(2, beams, vocab).contiguous().to(DEV)
    check(sel, logits, torch.full((2, beams), -1.0, device=DEV))


def test_captured_and_on_a_stream():
    groups, beams, vocab = 5, 4, 3000
    sel = make(groups, beams, vocab, dtype=torch.bfloat16, end_token=3)
    logits, scores = random_inputs(groups, beams, vocab, torch.bfloat16)
    ended = torch.zeros(groups, beams, dtype=torch.bool, device=DEV)
    want = check(sel, logits, scores, ended)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = sel.select(logits, scores, ended, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sel.select(logits, scores, ended)
    for seed in range(3):
        l2, s2 = random_inputs(groups, beams, vocab, torch.bfloat16, seed=20 + seed)
        logits.copy_(l2)
        scores.copy_(s2)
        graph.replay()
        check(sel, logits, scores, ended, got=out)
