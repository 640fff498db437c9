"""The kernel that joins the parts of a row over shared pages, where two rows share a warp: of one all parts count, of the
other some or none."""
import numpy as np
import pytest
import torch

from test_gpu_pages import DEV, ints
from test_gpu_pages_shared import attend, family

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [1, 3])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_rows_with_and_without_parts(dtype, group):
    """Groups of 37 and 35 rows or more with a long text in common, between them entries that share nothing, odd numbers of rows."""
    tails = [1 + 7 * i % 60 for i in range(37)]
    c, m, seqs, b = family([(3001, tails), (0, [9]), (700, tails[:35]), (5, [3])], dim=64, pt=32, heads=1, group=group, dtype=dtype)
    want = attend(c, m, seqs, b, max_group=1000)
    attend(c, m, seqs, b, tail=0, max_group=1000)
    attend(c, m, seqs, b, new=[1 + i % 3 for i in range(len(seqs))], max_group=1000)
    q = torch.from_numpy(np.random.default_rng(1).normal(size=want.shape)).to(dtype).to(DEV)
    starts = ints(list(range(len(seqs) + 1)))
    got = [c.shared_attention(q, ints(seqs), ints(b), starts, max_new=1, max_group=1000)[:len(seqs)] for _ in range(20)]
    assert all(torch.equal(x, got[0]) for x in got)
    assert np.array_equal(got[0].double().cpu().numpy(), want[:len(seqs)]) and c.poll_status() == 0
