"""The write into blocks whose magnitudes are any fp32 number, as a cache may hold that its owner has filled."""
import numpy as np
import pytest
import torch

from test_gpu_pages import DEV, ints, make, same_contents

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,fmt,dtype", [(64, "int8", torch.float16), (128, "int8", torch.bfloat16), (64, "e4m3", torch.bfloat16),
                                           (128, "e4m3", torch.float16)])
@pytest.mark.parametrize("new", [1, 9])
@pytest.mark.parametrize("grows", [False, True])
def test_quotients_beside_a_tie(dim, fmt, dtype, new, grows):
    """The older magnitude is such that a code (where the new tokens are larger), or a new value (where they are not), falls
    beside a tie, nearer than fp32 can tell."""
    n, heads, kept = 60, 4, 7
    c, m = make(heads=heads, dim=dim, pages=n, seqs=n, seq_pages=1, pt=16, fmt=fmt, dtype=dtype)
    c.resize(ints(range(n)), ints([kept + new] * n))
    m.resize(list(range(n)), [kept + new] * n)
    rng = np.random.default_rng(dim + new)
    val = np.sort(m.val[:127]) if fmt == "e4m3" else np.arange(128.0)
    ties = (val[1:] + val[:-1]) / 2
    top = val[-1]
    m.codes[:] = rng.integers(0, 256, m.codes.shape)
    if fmt == "e4m3":
        m.codes[m.codes % 128 == 127] = 3
    else:
        m.codes[m.codes == 128] = 3
    x = rng.normal(size=(n * new, 1, heads, dim, 2)) * 0.3
    x = torch.from_numpy(x.clip(-1, 1)).to(dtype)
    for s in range(n):
        page = m.table[s, 0]
        for h in range(heads):
            for which in (0, 1):
                if grows:
                    x[s * new, 0, h, 5, which] = big = 1.5
                    code = abs(m.val[m.codes[0, page, h, which, m.at[which][rng.integers(kept), rng.integers(dim)]]])
                    below = ties[ties < code]
                    ratio = below[rng.integers(len(below))] / code if len(below) else 0.4      # of old to new magnitude
                    old = np.float32(big * ratio)
                else:
                    v = abs(float(x[s * new, 0, h, rng.integers(dim), which]))
                    old = np.float32(v * top / ties[np.searchsorted(ties, v * top / 3.5) + rng.integers(0, 2)])
                old = np.nextafter(old, np.float32(rng.choice([0, 100])))
                m.amax[0, page, h, which, 0] = max(old, np.float32(1.1)) if not grows else old
    c.codes.copy_(torch.from_numpy(m.codes))
    c.amax.copy_(torch.from_numpy(m.amax))
    k, v = x[..., 0].contiguous(), x[..., 1].contiguous()
    starts = list(range(0, n * new + 1, new))
    c.write(k.to(DEV), v.to(DEV), ints(range(n)), ints(starts) if new > 1 else None)
    m.write(list(range(n)), starts, k.double().numpy(), v.double().numpy())
    same_contents(c, m)
    assert c.poll_status() == 0
