"""Host-side checks of the head operators' C ABI that need no GPU: sizes and
arguments are refused before any device is touched, and the binding mirrors the
header."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def lib():
    from paper_2608_13144_gb300.build import build
    build()
    from paper_2608_13144_gb300 import _lib
    return _lib.load()


def describe(**kw):
    from paper_2608_13144_gb300._lib import Adapted
    v = dict(type=0, d=16, classes=8, adapters=2, rank=4, reserved=0, tokens=4, x=4096, ldx=16, W=4096, ldw=16, A=4096,
             B=4096, adapter=4096, scales=None)
    v.update(kw)
    return Adapted(**v)


def test_adapted_sizes(lib):
    for backward in (0, 1):
        assert lib.lipcache_adapted_workspace(C.byref(describe()), backward) >= 0
        for bad in (dict(type=2), dict(d=0), dict(d=65537), dict(classes=0), dict(classes=65537), dict(adapters=-1),
                    dict(adapters=4097), dict(rank=0), dict(rank=129), dict(tokens=-1), dict(tokens=(1 << 24) + 1),
                    dict(reserved=1)):
            assert lib.lipcache_adapted_workspace(C.byref(describe(**bad)), backward) == -1, bad
            assert lib.lipcache_last_error()
    assert lib.lipcache_adapted_workspace(None, 0) == -1


def test_adapted_arguments(lib):
    big = 1 << 40  # a workspace size; the refusals come before any use
    def fwd(p, y=4096, ldy=8, ws=4096, n=big):
        return lib.lipcache_adapted_logits(C.byref(p), None, y, ldy, ws, n, None)
    for bad in (dict(x=None), dict(W=None), dict(A=None), dict(B=None), dict(adapter=None), dict(ldx=15),
                dict(ldw=15), dict(x=4097), dict(W=4098)):
        assert fwd(describe(**bad)) == 1, bad
    assert fwd(describe(), y=None) == 1
    assert fwd(describe(), ldy=7) == 1
    assert fwd(describe(), ws=4097) == 1
    assert fwd(describe(), ws=None) == 1
    assert fwd(describe(), n=-1) == 1
    assert fwd(describe(tokens=0, x=None, W=None), y=None, ws=None, n=0) == 0
    assert lib.lipcache_adapted_logits_backward(C.byref(describe()), None, 8, 4096, 16, 4096, 4096, 4096, big, None) == 1
    assert lib.lipcache_adapted_logits_backward(C.byref(describe()), 4096, 7, 4096, 16, 4096, 4096, 4096, big, None) == 1
    assert lib.lipcache_adapted_logits_backward(C.byref(describe()), 4096, 8, 4096, 15, 4096, 4096, 4096, big, None) == 1


def test_cross_entropy_arguments(lib):
    def ce(ty=0, z=4096, ldz=8, n=2, c=8, t=4096, loss=4096, dz=8192, ldd=8):
        return lib.lipcache_cross_entropy(ty, z, ldz, n, c, t, None, loss, dz, ldd, None)
    for bad in (dict(ty=7), dict(z=None), dict(ldz=7), dict(n=-1), dict(c=0), dict(c=(1 << 24) + 1), dict(t=None),
                dict(ldd=7), dict(z=4097), dict(dz=4096, ldd=9)):
        assert ce(**bad) == 1, bad
    assert ce(n=0, z=None, t=None) == 0
    assert ce(loss=None, dz=None) == 0  # nothing asked for


def test_orthogonalize_arguments(lib):
    coef = (C.c_double * 3)(1.5, -0.5, 0.0)
    assert lib.lipcache_orthogonalize_workspace(0, 1, 64, 64) > 0
    for bad in ((2, 1, 64, 64), (0, -1, 64, 64), (0, 65536, 64, 64), (0, 1, 0, 64), (0, 1, 64, 0), (0, 1, 65537, 4),
                (0, 1, 20000, 20000)):
        assert lib.lipcache_orthogonalize_workspace(*bad) == -1, bad
    big = 1 << 40

    def o(ty=0, g=4096, ld=8, b=1, m=8, n=8, steps=1, c=coef, eps=1e-7, out=8192, ws=4096, nb=big):
        return lib.lipcache_orthogonalize(ty, g, ld, b, m, n, steps, c, eps, out, ws, nb, None)
    for bad in (dict(ty=3), dict(g=None), dict(out=None), dict(ld=7), dict(steps=0), dict(steps=33), dict(c=None),
                dict(eps=0.0), dict(eps=2.0), dict(g=4097), dict(ws=4100), dict(ws=None), dict(nb=16),
                dict(out=4096, ld=9)):
        assert o(**bad) == 1, bad
    for v in (float("nan"), float("inf"), 65.0):
        assert o(c=(C.c_double * 3)(1.5, v, 0.0)) == 1
    assert o(b=0, g=None, out=None, ws=None, nb=0) == 0

    def st(wt=0, gt=0, w=4096, g=4096, m=4096, ow=4096, om=4096, lr=0.1, beta=0.9, decay=0.0):
        return lib.lipcache_orthogonal_step(wt, gt, w, g, m, ow, om, 1, 8, 8, lr, beta, 1, decay, 1, coef, 1e-7, 4096,
                                            big, None)
    for bad in (dict(wt=2), dict(gt=2), dict(w=None), dict(g=None), dict(m=None), dict(ow=None), dict(om=None),
                dict(lr=float("nan")), dict(beta=-0.1), dict(beta=1.1), dict(decay=float("inf")), dict(m=4098)):
        assert st(**bad) == 1, bad


def test_arrays_of_32_bits_are_aligned(lib):
    big = 1 << 40
    for ty in (0, 1):
        for bad in (dict(adapter=4098), dict(adapter=4097), dict(scales=4098)):
            p = describe(type=ty, **bad)
            assert lib.lipcache_adapted_logits(C.byref(p), None, 4096, 8, 4096, big, None) == 1, bad
            assert lib.lipcache_adapted_logits_backward(C.byref(p), 4096, 8, 4096, 16, 4096, 4096, 4096, big, None) == 1, bad
        assert lib.lipcache_adapted_logits(C.byref(describe(type=ty)), 4098, 4096, 8, 4096, big, None) == 1
        for target, weight, loss in ((4098, None, 4096), (4096, 4098, 4096), (4096, None, 4097)):
            assert lib.lipcache_cross_entropy(ty, 4096, 8, 2, 8, target, weight, loss, 8192, 8, None) == 1


def test_operator_errors_argument(lib):
    assert lib.lipcache_operator_errors(None, None) == 1


def test_struct_layout_matches_header(tmp_path):
    from paper_2608_13144_gb300 import _lib
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = [f[0] for f in _lib.Adapted._fields_]
    body = "\n".join(f'  printf("{n} %zu\\n", offsetof(lipcache_adapted, {n}));' for n in names)
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "lipcache.h"\nint main(void) {\n'
                   f'{body}\n  printf("sizeof %zu\\n", sizeof(lipcache_adapted));\n  return 0;\n}}\n')
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True,
                                                       text=True).stdout.splitlines())
    for n in names:
        assert int(out[n]) == getattr(_lib.Adapted, n).offset, n
    assert int(out["sizeof"]) == C.sizeof(_lib.Adapted)
