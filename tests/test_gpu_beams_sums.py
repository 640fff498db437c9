"""The sums of beam search's selection over the whole range of logits, against beams_ref.py within the bounds of
test_gpu_beams.py: a term is off by at most 2^-22 (exponential) + 6 * 2^-24 (additions) + |x| 2^-23.4 of itself, x the
distance in bits from the reference, so a score by less than 2.8e-6 as long as the terms that count lie within 23 bits."""
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
