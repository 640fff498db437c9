"""Attention over shared pages without a GPU: refusals of the C entry point (nothing is launched)."""
import pytest

from test_pages_host import BAD, LAYERS, MISALIGNED, NULL, SMALL, desc


@pytest.fixture(scope="module")
def B():
    from paper_2402_09398_b200 import build, binding
    build.build()
    binding.lib()
    return binding


def test_arguments(B):
    p = 4096

    def call(lb=0, lc=1, n=2, seqs=p, starts=None, rows=2, new=1, ng=1, groups=p, most=2, q=p, qs=1024, window=0, sinks=0,
             scale=0.1, out=p, **kw):
        return B.less_pages_shared_attention(desc(B, **kw), lb, lc, n, seqs, starts, rows, new, ng, groups, most, q, qs,
                                             window, sinks, scale, out, None)
    assert call(lb=2) == LAYERS and call(lc=3) == LAYERS
    assert call(rows=1) == BAD and call(new=0) == BAD and call(window=-1) == BAD and call(sinks=-1) == BAD
    assert call(scale=0.0) == BAD and call(scale=float("nan")) == BAD
    assert call(qs=1016) == BAD and call(qs=1028) == MISALIGNED and call(q=4104) == MISALIGNED
    assert call(out=None) == NULL and call(seqs=None) == NULL and call(groups=None) == NULL
    assert call(groups=4098) == MISALIGNED
    assert call(ng=0) == BAD and call(ng=3) == BAD and call(ng=-1) == BAD and call(most=0) == BAD
    assert call(n=4, rows=4) == BAD                        # more entries than sequences
    assert call(n=0, rows=0, ng=0, seqs=None, groups=None, q=None, out=None) == 0
    for kw, code in ((dict(codes=None), NULL), (dict(refs=4100), MISALIGNED), (dict(workspace_bytes=1 << 20), SMALL),
                     (dict(head_dim=32), BAD)):
        assert call(**kw) == code
