"""The paged cache without a GPU: refusals of the C entry points (nothing is launched), the ctypes mirror of
less_pages, and the reference model itself."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

import pages_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, NULL, MISALIGNED, SMALL, LAYERS = -1, -2, -3, -4, -6


@pytest.fixture(scope="module")
def B():
    from paper_2402_09398_b200 import build, binding
    build.build()
    binding.lib()
    return binding


def desc(B, **kw):
    f = dict(layers=2, heads=4, group=2, head_dim=128, page_tokens=64, pages=10, seqs=3, seq_pages=5, flags=0,
             codes=4096, amax=4096, table=4096, lens=4096, refs=4096, workspace=4096, workspace_bytes=1 << 30)
    f.update(kw)
    return B.less_pages(*(f[n] for n, _ in B.less_pages._fields_))


def test_struct_matches_the_header(B, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in B.less_pages._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "less.h"\nint main(void) {\n  printf("%zu\\n", sizeof(less_pages));\n' +
                   "".join(f'  printf("%zu\\n", offsetof(less_pages, {n}));\n' for n in names) + "  return 0;\n}\n")
    subprocess.run([gcc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True,
                                          text=True).stdout.split()]
    assert got == [C.sizeof(B.less_pages)] + [getattr(B.less_pages, n).offset for n in names]


def test_workspace_and_description(B):
    good = B.less_pages_workspace_bytes(desc(B))
    assert good > 48 << 20
    assert B.less_pages_workspace_bytes(desc(B, pages=100000)) > good
    for bad in (dict(layers=0), dict(heads=0), dict(group=0), dict(group=129), dict(head_dim=96), dict(page_tokens=8),
                dict(page_tokens=48), dict(page_tokens=512), dict(pages=0), dict(seqs=0), dict(seq_pages=0),
                dict(flags=4), dict(seq_pages=1 << 25), dict(pages=(1 << 28) + 1), dict(heads=40000, group=2),
                dict(seqs=1 << 23, seq_pages=1 << 10)):
        assert B.less_pages_workspace_bytes(desc(B, **bad)) == 0, bad
        assert B.less_pages_reset(desc(B, **bad), None) == BAD, bad


def calls(B, d):
    p = 4096
    return [lambda: B.less_pages_reset(d, None), lambda: B.less_pages_resize(d, 1, p, p, None),
            lambda: B.less_pages_fork(d, 1, p, p, None), lambda: B.less_pages_trim(d, 1, p, 0, 1, None),
            lambda: B.less_pages_compact(d, None),
            lambda: B.less_pages_write(d, 0, 1, 1, p, None, 1, p, 512, p, 512, None),
            lambda: B.less_pages_attention(d, 0, 1, 1, p, None, 1, 1, p, 1024, 0, 0, 0.1, p, None),
            lambda: B.less_pages_poll_status(d, None)]


@pytest.mark.parametrize("kw,code", [(dict(codes=None), NULL), (dict(amax=None), NULL), (dict(table=None), NULL),
                                     (dict(lens=None), NULL), (dict(refs=None), NULL), (dict(workspace=None), NULL),
                                     (dict(codes=4104), MISALIGNED), (dict(refs=4100), MISALIGNED),
                                     (dict(workspace=4096 + 16), MISALIGNED), (dict(workspace_bytes=1 << 20), SMALL),
                                     (dict(head_dim=32), BAD)])
def test_bad_descriptions_are_refused_by_every_call(B, kw, code):
    for c in calls(B, desc(B, **kw)):
        assert c() == code


def test_bad_arguments(B):
    d, p = desc(B), 4096
    assert B.less_pages_resize(d, -1, p, p, None) == BAD and B.less_pages_resize(d, 4, p, p, None) == BAD
    assert B.less_pages_resize(d, 1, None, p, None) == NULL and B.less_pages_resize(d, 1, p, 4098, None) == MISALIGNED
    assert B.less_pages_resize(d, 0, None, None, None) == 0
    assert B.less_pages_fork(d, 4, p, p, None) == BAD and B.less_pages_fork(d, 1, p, None, None) == NULL
    assert B.less_pages_fork(d, 0, None, None, None) == 0
    assert B.less_pages_trim(d, 1, p, -1, 5, None) == BAD and B.less_pages_trim(d, 1, p, 0, 0, None) == BAD
    assert B.less_pages_trim(d, 1, None, 0, 5, None) == NULL

    def write(lb=0, lc=1, n=1, seqs=p, starts=None, rows=1, k=p, ks=512, v=p, vs=512):
        return B.less_pages_write(d, lb, lc, n, seqs, starts, rows, k, ks, v, vs, None)
    assert write(lb=-1) == LAYERS and write(lc=0) == LAYERS and write(lb=1, lc=2) == LAYERS
    assert write(lc=0x7fffffff) == LAYERS
    assert write(rows=2) == BAD and write(n=-1) == BAD and write(ks=504) == BAD and write(vs=0) == BAD
    assert write(ks=516) == MISALIGNED and write(k=4104) == MISALIGNED and write(v=None) == NULL
    assert write(starts=4097, rows=3) == MISALIGNED
    assert write(n=0, rows=0, seqs=None, k=None, v=None) == 0

    def attn(lb=0, lc=1, n=1, seqs=p, starts=None, rows=1, new=1, q=p, qs=1024, window=0, sinks=0, scale=0.1, out=p):
        return B.less_pages_attention(d, lb, lc, n, seqs, starts, rows, new, q, qs, window, sinks, scale, out, None)
    assert attn(lb=2) == LAYERS and attn(lc=3) == LAYERS
    assert attn(rows=2) == BAD and attn(new=0) == BAD and attn(window=-1) == BAD and attn(sinks=-1) == BAD
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attn(scale=scale) == BAD
    assert attn(qs=1016) == BAD and attn(qs=1028) == MISALIGNED and attn(q=4104) == MISALIGNED
    assert attn(out=None) == NULL and attn(out=4104) == MISALIGNED
    assert attn(n=0, rows=0, seqs=None, q=None, out=None) == 0
    assert "free pages" in B.less_strerror(B.LESS_ERR_PAGES_EXHAUSTED)


def test_holder_refuses_before_the_device(B):
    import torch
    with pytest.raises(ValueError):
        B.PagedCache(1, 1, 64, 4, 1, 4, fmt="fp8")
    with pytest.raises(ValueError):
        B.PagedCache(1, 1, 64, 4, 1, 4, dtype=torch.float32)
    with pytest.raises(B.LessError):
        B.PagedCache(1, 1, 80, 4, 1, 4)


@pytest.mark.parametrize("D", [64, 128])
def test_stored_order_covers_a_tile_once(D):
    for values in (False, True):
        at = pages_ref.places(D, values)
        assert sorted(at.ravel().tolist()) == list(range(16 * D))


def test_codes_of_the_model():
    import torch
    for fmt, t in (("int8", torch.int8), ("e4m3", torch.float8_e4m3fn)):
        val = pages_ref.code_values(fmt)
        want = torch.arange(256, dtype=torch.int64).to(torch.uint8).view(t).double().numpy()
        assert np.array_equal(val, want, equal_nan=True)
        ok = ~np.isnan(val) & ~((fmt == "e4m3") & (np.arange(256) == 128))
        assert np.array_equal(pages_ref.encode(val[ok], fmt), np.arange(256, dtype=np.uint8)[ok])
    x = np.random.default_rng(0).uniform(-448, 448, 5000).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(pages_ref.encode(x.astype(np.float64), "e4m3"), want)
    assert pages_ref.encode(np.array([0.5, 1.5, 2.5, -0.5]), "int8").tolist() == [0, 2, 2, 0]


def test_attention_of_more_items_than_can_be_counted(B):
    d, p = desc(B, heads=64, group=2), 4096

    def attn(rows, lc):
        return B.less_pages_attention(d, 0, lc, 4, p, p, rows, 1, p, 2 * 64 * 2 * 128, 0, 0, 0.1, p, None)
    assert attn(1 << 29, 1) == BAD and attn(1 << 27, 1) == BAD and attn(1 << 26, 2) == BAD


@pytest.mark.parametrize("starts", [None, 4096])
def test_write_of_more_entries_than_sequences(B, starts):
    assert B.less_pages_write(desc(B), 0, 1, 4, 4096, starts, 4, 4096, 512, 4096, 512, None) == BAD
