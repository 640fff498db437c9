"""Beam search's selection without a GPU: refusals of the C entry points, the ctypes mirror, the model itself."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

import beams_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, NULL, MISALIGNED, SMALL = -1, -2, -3, -4


@pytest.fixture(scope="module")
def B():
    from paper_2402_09398_b200 import build, binding
    build.build()
    binding.lib()
    return binding


def desc(B, **kw):
    f = dict(groups=2, beams=4, vocab=1000, keep=4, end_token=-1, flags=0, workspace=4096, workspace_bytes=1 << 30)
    f.update(kw)
    return B.less_beams(*(f[n] for n, _ in B.less_beams._fields_))


def test_struct_matches_the_header(B, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in B.less_beams._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "less.h"\nint main(void) {\n  printf("%zu\\n", sizeof(less_beams));\n' +
                   "".join(f'  printf("%zu\\n", offsetof(less_beams, {n}));\n' for n in names) + "  return 0;\n}\n")
    subprocess.run([gcc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True,
                                          text=True).stdout.split()]
    assert got == [C.sizeof(B.less_beams)] + [getattr(B.less_beams, n).offset for n in names]


def test_descriptions(B):
    good = B.less_beams_workspace_bytes(desc(B))
    assert good > 0 and good % 256 == 0
    assert B.less_beams_workspace_bytes(desc(B, groups=50)) > good
    p = 4096
    for bad in (dict(groups=0), dict(beams=0), dict(beams=65), dict(vocab=0), dict(vocab=2 ** 26 + 1), dict(keep=0), dict(keep=129), dict(flags=3),
                dict(flags=4), dict(end_token=-2), dict(end_token=1000), dict(groups=1 << 20)):
        assert B.less_beams_workspace_bytes(desc(B, **bad)) == 0, bad
        assert B.less_beam_select(desc(B, **bad), p, 1000, p, None, p, p, p, p, None) == BAD, bad
    assert B.less_beams_workspace_bytes(desc(B, beams=64, keep=128, vocab=2 ** 26, end_token=5)) > good


def test_arguments(B):
    p = 4096

    def call(d=None, logits=p, stride=1000, scores=p, ended=None, s=p, t=p, r=p, e=None, **kw):
        return B.less_beam_select(desc(B, **kw) if d is None else d, logits, stride, scores, ended, s, t, r, e, None)
    for name in ("logits", "scores", "s", "t", "r"):
        assert call(**{name: None}) == NULL, name
    assert call(workspace=None) == NULL and B.less_beam_select(None, p, 1000, p, None, p, p, p, p, None) == NULL
    assert call(stride=999) == BAD and call(ended=p) == BAD and call(stride=1 << 50) == BAD
    assert call(logits=p + 1) == MISALIGNED and call(logits=p + 2, flags=2) == MISALIGNED
    assert call(workspace=4096 + 16) == MISALIGNED and call(workspace_bytes=100) == SMALL
    for name in ("scores", "s", "t", "r"):
        assert call(**{name: p + 2}) == MISALIGNED, name


def test_holder_refuses_before_the_device(B):
    import torch
    with pytest.raises(ValueError):
        B.BeamSelect(1, 2, 100, dtype=torch.float64)
    with pytest.raises(B.LessError):
        B.BeamSelect(1, 65, 100)
    with pytest.raises(B.LessError):
        B.BeamSelect(1, 2, 100, end_token=100)


def test_the_model():
    x = np.array([[[0.0, 1.0, 1.0], [2.0, -np.inf, np.nan]]])
    s, t, p, e = beams_ref.select(x, np.array([[0.0, -0.5]]), np.array([[False, False]]), 1, 5, 65504.0)
    lse = np.log(1 + 2 * np.exp(1.0))
    assert np.allclose(s[0], [-0.5, 1 - lse, 1 - lse, -lse, -np.inf])
    assert t[0].tolist() == [0, 1, 2, 0, -1] and p[0].tolist() == [1, 0, 0, 0, 1] and e[0].tolist() == [0, 1, 0, 0, 0]
