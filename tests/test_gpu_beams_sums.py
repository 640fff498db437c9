"""The sums of beam search's selection over the whole range of logits, against beams_ref.py within the bounds of
test_gpu_beams.py: a term is off by at most 2^-22 (exponential) + 6 * 2^-24 (additions) + |x| 2^-23.4 of itself, x the
distance in bits from the reference, so a score by less than 2.8e-6 as long as the terms that count lie within 23 bits."""
import numpy as np
import pytest
import torch

from test_gpu_beams import DEV, TYPES, check, make

pytestmark = pytest.mark.gpu
FAR = {"fp16": [1e3, 4099.0, 2.1e4, 4e4, 6e4], "bf16": [7e4, 1e5, 1e6, 1e7, 1e8, 1e9, 1e10, 1e20, 1e30],
       "fp32": [7e4, 1e5, 1e6, 1e7, 1e8, 1e9, 1e10, 1e20, 1e30]}


def body(n, vocab, seed=0):
    return torch.randn(n, vocab, generator=torch.Generator().manual_seed(seed)) * 2.5


def one_beam(dtype, logits, copies, keep=3):
    """Rows as texts of one beam each, `copies` times: few rows are cut into stretches, many are not."""
    logits = logits.to(TYPES[dtype]).to(DEV).repeat(copies, 1)[:, None].contiguous()
    n, vocab = logits.shape[0], logits.shape[2]
    check(make(n, 1, vocab, keep, TYPES[dtype]), logits, torch.full((n, 1), -0.25, device=DEV))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("copies", [1, 50])
def test_large_logits(dtype, sign, copies):
    """Rows around a large value, and wholly at one."""
    rows = body(2 * len(FAR[dtype]), 20011)
    for i, far in enumerate(FAR[dtype]):
        rows[2 * i] += sign * far
        rows[2 * i + 1] = sign * far
    one_beam(dtype, rows, copies)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("copies", [1, 50])
def test_masks_that_are_finite(dtype, copies):
    """Tokens masked with a finite value: the first ones, all but the last, every third; and one that is forced."""
    rows = body(4 * len(FAR[dtype]), 20011, seed=1)
    for i, far in enumerate(FAR[dtype]):
        rows[4 * i, :12000] = -far
        rows[4 * i + 1, :20010] = -far
        rows[4 * i + 2, ::3] = -far
        rows[4 * i + 3, 17000] = far
    one_beam(dtype, rows, copies)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_equal_beams_of_large_logits(dtype, sign):
    """Beams whose order hangs on the second summation."""
    far = FAR[dtype] + ([] if dtype == "fp16" else [2.0 ** 31, 2.0 ** 33, 1.5 * 2.0 ** 33, 2.0 ** 34, 1e11, 1e12, 1e15])
    vocab = 20011
    rows = body(3 * len(far), vocab, seed=2)
    for i, x in enumerate(far):
        rows[3 * i] += sign * x
        rows[3 * i + 1] = sign * x
        rows[3 * i + 2] = sign * x
        rows[3 * i + 2, ::2] = sign * x * (1 - sign * 2.0 ** -7)    # two values, far apart from 1e5 on
    logits = rows.to(TYPES[dtype])[:, None].expand(-1, 2, -1).contiguous().to(DEV)
    check(make(len(rows), 2, vocab, 4, TYPES[dtype]), logits, torch.full((len(rows), 2), -0.5, device=DEV))


def beside_ended(dtype, rows, keep=2, seed=0):
    """Every row as a beam beside one that has ended, whose score is that of the row's first candidate up to three steps of
    fp32: the order is that of the 64-bit values."""
    rows = rows.to(TYPES[dtype])
    n, vocab = rows.shape
    logits = torch.zeros(n, 2, vocab, dtype=TYPES[dtype])
    logits[:, 0] = rows
    x = rows.double().numpy()
    top = x.max(-1)
    value = -0.0625 + (top - (top + np.log(np.exp(x - top[:, None]).sum(-1))))
    step = np.random.default_rng(seed).integers(-3, 4, n)
    score = value.astype(np.float32)
    score = score + step.astype(np.float32) * np.spacing(np.abs(score))
    near = np.abs(score.astype(np.float64) - value) < 1e-9          # than the second summation tells apart
    score = np.where(near, score + np.spacing(np.abs(score)), score)
    scores = torch.tensor([[-0.0625, float(s)] for s in score])
    ended = torch.tensor([[False, True]]).repeat(n, 1)
    check(make(n, 2, vocab, keep, TYPES[dtype], end_token=vocab - 1), logits.to(DEV), scores.to(DEV), ended.to(DEV))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("where", ["first", "last"])
def test_a_peak_at_either_end(dtype, where):
    """A row whose probability lies in its first or last element, before or behind the whole 16 bytes."""
    groups, vocab = 64, 50257
    g = torch.Generator().manual_seed(3)
    peak = (30 + 150 * torch.rand(groups, generator=g)) * (2 * torch.randint(0, 2, (groups,), generator=g) - 1)
    rows = peak[:, None] - 16 + torch.randn(groups, vocab, generator=g)
    rows[:, 0 if where == "first" else -1] = peak
    beside_ended(dtype, rows)
    # the same logits, the peak in the midst of the second beam's
    logits = rows.to(TYPES[dtype])[:, None].repeat(1, 2, 1)
    at = 0 if where == "first" else vocab - 1
    logits[:, 1, at], logits[:, 1, 30000] = logits[:, 0, 30000], logits[:, 0, at]
    first = torch.randint(24, 60, (groups,), generator=g)
    apart = torch.randint(1, 24, (groups,), generator=g) * (2 * torch.randint(0, 2, (groups,), generator=g) - 1)
    scores = -0.5 - torch.stack([first, first + apart], 1) * 2.0 ** -24
    check(make(groups, 2, vocab, 2, TYPES[dtype]), logits.to(DEV), scores.to(DEV))


def climbing(dtype, groups, seed):
    """Rows in which a thread meets logits far above its reference (39 of at most 40) before one that moves it: the former
    have most of the probability.  `first` is the reference, `mid` the former, `last` the latter.  (x is 56.3 there: half a
    step of it, 2^-19, times ln 2 1.3e-6, log2 e in fp32 39 * 1.93e-8, a term 6e-7: 2.7e-6 of four fifths of the sum.)"""
    g = torch.Generator().manual_seed(seed)
    per = 8 if dtype != "fp32" else 4                     # elements of 16 bytes; 256 threads, a first tile of four of each
    stride, vocab = 256 * per, 24 * 256 * per
    first = ((20 + 150 * torch.rand(groups, generator=g)) * (2 * torch.randint(0, 2, (groups,), generator=g) - 1)).to(TYPES[dtype]).float()
    mid, last = (first + 39.0).to(TYPES[dtype]).float(), (first + 42.0).to(TYPES[dtype]).float()
    rows = first[:, None] - 10 + torch.randn(groups, vocab, generator=g).clamp(max=4)
    rows[:, 77] = first
    for piece in range(6, 16):
        at = piece * stride + 5 * per
        rows[:, at:at + per] = mid[:, None]
    rows[:, 20 * stride + 5 * per] = last
    return rows


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("copies", [1, 10])
def test_references_that_move_under_much_of_a_sum(dtype, copies):
    one_beam(dtype, climbing(dtype, 64, 0), copies)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("seed", range(3))
def test_order_where_references_move_under_much_of_a_sum(dtype, seed):
    beside_ended(dtype, climbing(dtype, 320, seed), seed=seed)      # a stretch a row


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("keep", [2, 4, 6])
def test_order_of_beams_with_others_between(dtype, keep):
    """Beams of one value but for some 1e-6, whose sums have errors of different bounds: a peak that comes late, one that is
    the first tile's, and ended ones, which have none, among them."""
    groups, beams = 320, 6
    rows = climbing(dtype, groups, 7).to(TYPES[dtype])
    vocab = rows.shape[1]
    logits = torch.zeros(groups, beams, vocab, dtype=TYPES[dtype])
    logits[:, 0], logits[:, 2], logits[:, 4] = rows, rows.flip(1), rows.roll(1000, 1)
    x = rows.double().numpy()
    top = x.max(-1)
    value = -0.0625 + (top - (top + np.log(np.exp(x - top[:, None]).sum(-1))))
    rng = np.random.default_rng(keep)
    live = np.float32(-0.0625) + rng.integers(-60, 61, (groups, 3)).astype(np.float32) * np.float32(2.0 ** -27)
    near = (value[:, None] + rng.uniform(-1.5e-6, 1.5e-6, (groups, 3))).astype(np.float32)
    scores = torch.zeros(groups, beams)
    scores[:, ::2], scores[:, 1::2] = torch.from_numpy(live), torch.from_numpy(near)
    ended = torch.zeros(groups, beams, dtype=torch.bool)
    ended[:, 1::2] = True
    check(make(groups, beams, vocab, keep, TYPES[dtype], end_token=vocab - 1), logits.to(DEV), scores.to(DEV), ended.to(DEV))


def test_the_last_token_of_the_last_beam():
    """64 beams of 2^26 tokens, the last beam ended with the last token."""
    vocab = 1 << 26
    sel = make(1, 64, vocab, 4, torch.float16, end_token=vocab - 1)
    logits = torch.empty(1, 64, vocab, dtype=torch.float16, device=DEV)   # of beams that are not looked at
    scores = torch.full((1, 64), -float("inf"), device=DEV)
    ended = torch.zeros(1, 64, dtype=torch.bool, device=DEV)
    scores[0, 63], ended[0, 63] = -2.0, True
    scores[0, 7], ended[0, 7] = -2.0, True
    got = sel.select(logits, scores, ended)
    assert got.tokens.tolist() == [[vocab - 1, vocab - 1, -1, -1]] and got.parents.tolist() == [[7, 63, 2, 3]]
    assert got.scores.tolist() == [[-2.0, -2.0, -float("inf"), -float("inf")]]
    assert got.ended.tolist() == [[True, True, False, False]]
