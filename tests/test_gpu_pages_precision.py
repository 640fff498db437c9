"""Attention over the paged cache where a row's probabilities, or the magnitudes of its values, lie far apart: both kernels
against the 64-bit model, with a bound that scales with what a row adds up, not with the largest value of the cache."""
import numpy as np
import pytest
import torch

from test_gpu_pages import DEV, HALF_STEP, fill, ints, make

pytestmark = pytest.mark.gpu


def expected(m, q, seqs, starts, many):
    """(out, bound), float64 [rows, 1, heads * group, D]; `many`: the entries are the many-token kernel's.

    With p_j a probability, v_j and a_j a key's value and value magnitude, o the output, every p_j is off by a factor of
    at most 1 + d_j in both sums, so the output by sum p_j d_j (|v_j| + |o|) / sum p:
      d_j = D / 16 accumulations of 8 (fp32, may truncate: 2^-22) of at most reach_j = scale * sum |q| |k_j|
          + |z_j| 2^-21 (factors, sum and difference of the exponent in fp32)
          + 2^-17 (exponential: polynomial 2^-18.5; log2 a_v, below 128, to half a step of 2^-17; the fp32 sums)
          + bf16 queries as fp16 over a power of two: 2^-25 of the row's largest, times scale * sum |k_j|
    Rounding P = p_j a_j (times a power of two of the row) to fp16 moves it by 2^-11 at most, where a rest is kept (few
    rows, fp16 output) by 2^-21; below 2^-14 by 2^-25.  A tile of T keys (32, many 64) is rounded with its own largest P at
    2^-7 or more, and at 2^6.5 or more if it is the largest of the row so far: the T keys of a tile lose at most T 2^-18
    of the tile's largest p_j a_j, that is of the sum over its keys, and beside the largest of the row T 2^-31 of that, but
    no more than themselves (a rounding to zero)."""
    scale, T = m.D ** -0.5, 64 if many else 32
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for i, s in enumerate(seqs):
        n, new = int(m.lens[s]), starts[i + 1] - starts[i]
        j = np.arange(n)
        see = j <= (n - new + np.arange(new))[:, None]
        for h in range(m.H):
            k, _ = m.rows(0, s, h, 0, n)
            v, _ = m.rows(0, s, h, 1, n)
            a = m.amax[0, m.table[s, j // m.pt], h, 1, j % m.pt // 16]
            for g in range(m.G):
                qq = q[starts[i]:starts[i + 1], 0, h * m.G + g]
                z = np.where(see, qq @ k.T * scale, -np.inf)
                p = np.exp(z - z.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o = p @ v
                d = m.D // 16 * 2.0 ** -22 * (np.abs(qq) @ np.abs(k).T * scale) + 2.0 ** -17
                d += np.where(see, np.abs(z), 0.0) * 2.0 ** -21
                if m.bf16:
                    d += 2.0 ** -25 * scale * np.abs(qq).max(1)[:, None] * np.abs(k).sum(1)
                e = (p * d) @ np.abs(v) + (p * d).sum(1, keepdims=True) * np.abs(o)
                e += 2.0 ** (-11 if many or m.bf16 else -21) * (p @ np.abs(v))
                pa = p * a
                top = pa.max(1, keepdims=True)
                least = np.minimum(2.0 ** -31 * top, np.sort(pa, 1)[:, -2:-1]) if n > 1 else 0.0
                e += T * (2.0 ** -18 * (pa.sum(1, keepdims=True) - top) + least)
                out[starts[i]:starts[i + 1], 0, h * m.G + g] = o
                bound[starts[i]:starts[i + 1], 0, h * m.G + g] = e
    return out, bound


def check(c, m, q, seqs, starts, many):
    one = all(b - a == 1 for a, b in zip(starts, starts[1:]))
    got = c.attention(q.to(DEV), ints(seqs), None if one else ints(starts), max_new=max(np.diff(starts)))
    got = got.double().cpu().numpy()
    want, bound = expected(m, q.double().numpy(), seqs, starts, many)
    least = 2.0 ** -25 if c.dtype == torch.float16 else 0.0     # half the smallest fp16
    err, tol = np.abs(got - want), HALF_STEP[c.dtype] * np.abs(want) + bound + least
    at = np.unravel_index(np.argmax(err / (tol + 1e-300)), err.shape)
    assert np.isfinite(got).all()
    assert (err <= tol).all(), (at, got[at], want[at], tol[at])
    assert c.poll_status() == 0


def push(c, m):
    c.codes.copy_(torch.from_numpy(m.codes))
    c.amax.copy_(torch.from_numpy(m.amax))


# few rows: the step kernel, whose items are split where they are long; more: the many-token kernel
SHAPES = [(1, 1, False), (1, 8, False), (1, 16, False), (4, 8, True), (150, 2, True)]


def queries(rng, new, m, dtype, first):
    """Random queries whose first component (the one that meets large keys below) is `first`."""
    q = rng.normal(size=(new, 1, m.H * m.G, m.D))
    q[..., 0] = first
    return torch.from_numpy(q).to(dtype)


def set_first(m, s, tokens, which, code):
    """The first dimension's code of the tokens' keys (0) or values (1)."""
    for j in np.atleast_1d(tokens):
        m.codes[:, m.table[s, j // m.pt], :, which, j % m.pt // 16 * 16 * m.D + m.at[which][j % 16, 0]] = code


@pytest.mark.parametrize("dim,fmt,dtype", [(64, "int8", torch.float16), (64, "e4m3", torch.bfloat16), (128, "int8", torch.bfloat16),
                                           (128, "e4m3", torch.float16)])
@pytest.mark.parametrize("new,group,many", SHAPES)
def test_values_far_larger_than_those_attended_to(dim, fmt, dtype, new, group, many):
    """Blocks of huge values that get no probability to speak of do not take bits from the others, wherever they stand."""
    c, m = make(heads=1, dim=dim, group=group, pt=16, pages=70, seqs=1, seq_pages=70, fmt=fmt, dtype=dtype)
    fill(c, m, [1000])
    rng = np.random.default_rng(3)
    set_first(m, 0, np.arange(1000), 0, 0)
    for b in range(63):
        m.amax[:, m.table[0, b], :, 1] = np.float32(2.0 ** rng.integers(-3, 2))
        if b % 9 in (0, 5) and 16 * (b + 1) <= 1000 - new:       # keys that turn away from every query: p = e^-50 or less
            m.amax[:, m.table[0, b], :, 1] = np.float32(2.0 ** (24 + b % 4))
            set_first(m, 0, np.arange(16 * b, 16 * b + 16), 0, 0x81 if fmt == "int8" else 0xfe)    # -top
    push(c, m)
    q = queries(rng, new, m, dtype, 20.0 * dim ** 0.5)
    check(c, m, q, [0], [0, new], many)


@pytest.mark.parametrize("dim,fmt,dtype", [(64, "int8", torch.float16), (64, "e4m3", torch.bfloat16), (128, "int8", torch.bfloat16),
                                           (128, "e4m3", torch.float16)])
@pytest.mark.parametrize("new,group,many", SHAPES)
@pytest.mark.parametrize("order", ["small first", "large first", "mixed"])
def test_values_of_any_magnitude(dim, fmt, dtype, new, group, many, order):
    """Value blocks from 2^-90 to 2^90 (bf16) or over what fp16 holds; the sum is that of the large ones, to its own bound."""
    c, m = make(heads=1, dim=dim, group=group, pt=16, pages=70, seqs=1, seq_pages=70, fmt=fmt, dtype=dtype)
    fill(c, m, [1000])
    rng = np.random.default_rng(6)
    b, far = np.arange(63), 90.0 if dtype == torch.bfloat16 else 13.0
    e = {"small first": np.where(b < 30, -far, far), "large first": np.where(b < 30, far, -far),
         "mixed": rng.integers(-int(far), int(far) + 1, 63).astype(float)}[order]
    m.amax[0, m.table[0, :63], 0, 1, 0] = np.float32(np.exp2(e))
    push(c, m)
    check(c, m, torch.from_numpy(rng.normal(size=(new, 1, group, dim))).to(dtype), [0], [0, new], many)
    # and where all that a row sees is small
    m.amax[0, m.table[0, :63], 0, 1, 0] = np.float32(np.exp2(rng.integers(-99, -90, 63) if dtype == torch.bfloat16 else -8.0))
    push(c, m)
    check(c, m, torch.from_numpy(rng.normal(size=(new, 1, group, dim))).to(dtype), [0], [0, new], many)


def weak_tokens_beside_a_strong_one(dim, fmt, dtype, new, group, many, bits):
    """The first token's values are zeros, so that what comes out is the share of all the others, 2^-bits of its own each."""
    n = 4000
    c, m = make(heads=1, dim=dim, group=group, pt=64, pages=64, seqs=1, seq_pages=64, fmt=fmt, dtype=dtype)
    fill(c, m, [n])
    rng = np.random.default_rng(bits)
    set_first(m, 0, np.arange(n), 0, 0)
    page = m.table[0, 0]
    code = bits * np.log(2.0) / (20.0 * m.amax[0, page, 0, 0, 0]) * (127 if fmt == "int8" else 448)
    set_first(m, 0, 0, 0, round(code) if fmt == "int8" else int(np.searchsorted(m.val[:127], code)))
    m.codes[:, page, :, 1, m.at[1][0]] = 0
    m.amax[:, m.table[0, :63], :, 1] *= 2.0 ** min(14, bits - 8)       # so that fp16 can hold what comes out
    push(c, m)
    check(c, m, queries(rng, new, m, dtype, 20.0 * dim ** 0.5), [0], [0, new], many)


TYPES = [(64, "int8", torch.float16), (64, "e4m3", torch.bfloat16), (128, "int8", torch.bfloat16), (128, "e4m3", torch.float16)]


@pytest.mark.parametrize("dim,fmt,dtype", TYPES)
@pytest.mark.parametrize("new,group,many", SHAPES[:3])
@pytest.mark.parametrize("bits", [12, 20, 27, 34])
def test_first_token_that_holds_nearly_all_probability(dim, fmt, dtype, new, group, many, bits):
    weak_tokens_beside_a_strong_one(dim, fmt, dtype, new, group, many, bits)


@pytest.mark.parametrize("dim,fmt,dtype", TYPES)
@pytest.mark.parametrize("new,group,many", SHAPES[:3])
def test_strong_tokens_now_and_then(dim, fmt, dtype, new, group, many):
    """The reference goes up and down many times, also by more than the sums have room for."""
    strong_tokens_now_and_then(dim, fmt, dtype, new, group, many)


def strong_tokens_now_and_then(dim, fmt, dtype, new, group, many):
    n = 3000
    c, m = make(heads=1, dim=dim, group=group, pt=16, pages=190, seqs=1, seq_pages=190, fmt=fmt, dtype=dtype)
    fill(c, m, [n])
    rng = np.random.default_rng(9)
    top = 127 if fmt == "int8" else 0x7e
    set_first(m, 0, np.arange(n), 0, 0)
    for j in rng.integers(0, n - new, 25):                     # 4 to 120 bits above the others
        set_first(m, 0, j, 0, int(rng.integers(top // 12, top + 1)))
    set_first(m, 0, 40, 0, top)
    m.amax[:, m.table[0, :188], :, 1] *= 2.0 ** 6
    push(c, m)
    check(c, m, queries(rng, new, m, dtype, 24.0 * dim ** 0.5), [0], [0, new], many)


@pytest.mark.parametrize("dim,fmt,dtype", TYPES)
@pytest.mark.parametrize("new,group,many", SHAPES[3:])
@pytest.mark.parametrize("bits", [12, 20, 27, 34])
def test_many_tokens_first_token_that_holds_nearly_all_probability(dim, fmt, dtype, new, group, many, bits):
    weak_tokens_beside_a_strong_one(dim, fmt, dtype, new, group, many, bits)


@pytest.mark.parametrize("dim,fmt,dtype", TYPES)
@pytest.mark.parametrize("new,group,many", SHAPES[3:])
def test_many_tokens_strong_tokens_now_and_then(dim, fmt, dtype, new, group, many):
    strong_tokens_now_and_then(dim, fmt, dtype, new, group, many)


@pytest.mark.parametrize("dim,fmt,dtype", TYPES)
@pytest.mark.parametrize("group,many", [(1, False), (8, False), (16, False), (40, True), (128, True)])
def test_a_row_that_is_one_key(dim, fmt, dtype, group, many):
    """One key, or one with nearly all probability: the largest P of a row is a power of two, so that the result is the value
    but for 2^-15 (the bound of `expected` without the rounding of P) and the output's own rounding."""
    n = 30
    c, m = make(heads=1, dim=dim, group=group, pt=16, pages=2 * n, seqs=n, seq_pages=2, fmt=fmt, dtype=dtype)
    fill(c, m, [1] * n)
    rng = np.random.default_rng(group)
    q = torch.from_numpy(rng.normal(size=(n, 1, group, dim))).to(dtype)
    got = c.attention(q.to(DEV), ints(range(n))).double().cpu().numpy()
    want = np.stack([m.rows(0, s, 0, 1, 1)[0] for s in range(n)])[:, :, None]
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -14))) - (10 if dtype == torch.float16 else 7))
    assert (np.abs(got - want) <= step / 2 + 2.0 ** -15 * np.abs(want)).all()
    assert c.poll_status() == 0
