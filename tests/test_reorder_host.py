"""Reordering without a GPU: refusals of the C entry points (nothing is launched) and the ctypes mirrors."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from test_pages_host import desc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, NULL, MISALIGNED, SMALL = -1, -2, -3, -4


@pytest.fixture(scope="module")
def B():
    from paper_2402_09398_b200 import build, binding
    build.build()
    binding.lib()
    return binding


def test_struct_matches_the_header(B, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in B.less_state._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "less.h"\nint main(void) {\n  printf("%zu\\n", sizeof(less_state));\n' +
                   "".join(f'  printf("%zu\\n", offsetof(less_state, {n}));\n' for n in names) +
                   '  printf("%d\\n", LESS_KERNEL_COUNT);\n  return 0;\n}\n')
    subprocess.run([gcc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True,
                                          text=True).stdout.split()]
    assert got == [C.sizeof(B.less_state)] + [getattr(B.less_state, n).offset for n in names] + [len(B.KERNEL_NAMES)]


def test_without_a_context(B):
    assert B.less_reorder(None, 1, 4096, None) == NULL
    assert B.less_state_view(None)[0] == NULL


def test_paged(B):
    d, p = desc(B, seqs=20000), 4096
    assert B.less_pages_reorder(d, -1, p, p, None) == BAD and B.less_pages_reorder(d, 8193, p, p, None) == BAD
    assert B.less_pages_reorder(desc(B), 4, p, p, None) == BAD
    assert B.less_pages_reorder(d, 1, None, p, None) == NULL and B.less_pages_reorder(d, 1, p, None, None) == NULL
    assert B.less_pages_reorder(d, 1, 4098, p, None) == MISALIGNED and B.less_pages_reorder(d, 1, p, 4097, None) == MISALIGNED
    assert B.less_pages_reorder(d, 0, None, None, None) == 0
    for kw, code in ((dict(codes=None), NULL), (dict(refs=4100), MISALIGNED), (dict(workspace_bytes=1 << 20), SMALL),
                     (dict(head_dim=32), BAD)):
        assert B.less_pages_reorder(desc(B, **kw), 1, p, p, None) == code
