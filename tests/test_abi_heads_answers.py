"""Host-side checks of the C entries of log_probs, distill and layer_norm that
need no GPU: sizes and arguments are refused before any device is touched."""
import math

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2608_13144_gb300.build import build
    build()
    from paper_2608_13144_gb300 import _lib
    return _lib.load()


TEMPERATURES = [dict(T=0.0), dict(T=-1.0), dict(T=9e-4), dict(T=1001.0), dict(T=math.nan), dict(T=math.inf)]
ROWS = [dict(ty=2), dict(z=None), dict(ldz=7), dict(n=-1), dict(n=(1 << 24) + 1), dict(c=0), dict(c=(1 << 24) + 1), dict(z=4097)]


def test_log_probs_arguments(lib):
    def call(ty=0, z=4096, ldz=8, n=2, c=8, t=4096, k=2, T=1.0, lp=4096, ent=4096, norm=4096, top=4096, index=4096):
        return lib.lipcache_log_probs(ty, z, ldz, n, c, t, k, T, lp, ent, norm, top, index, None)
    for bad in ROWS + TEMPERATURES + [dict(t=None), dict(k=-1), dict(k=129), dict(top=None), dict(index=None), dict(t=4098),
                                      dict(lp=4098), dict(ent=4097), dict(norm=4098), dict(top=4099), dict(index=4098)]:
        assert call(**bad) == 1, bad
        assert lib.lipcache_last_error()
    assert call(n=0, z=None, t=None, lp=None, top=None) == 0
    assert call(k=0, lp=None, ent=None, norm=None, top=None, index=None, t=None) == 0  # nothing asked for


def test_log_probs_backward_arguments(lib):
    def call(ty=0, z=4096, ldz=8, n=2, c=8, norm=4096, t=4096, g=4096, h=4096, T=1.0, dz=8192, ldd=8):
        return lib.lipcache_log_probs_backward(ty, z, ldz, n, c, norm, t, g, h, T, dz, ldd, None)
    for bad in ROWS + TEMPERATURES + [dict(norm=None), dict(dz=None), dict(t=None), dict(ldd=7), dict(dz=4096, ldd=9),
                                      dict(dz=8194), dict(norm=4098), dict(t=4097), dict(g=4098), dict(h=4098)]:
        assert call(**bad) == 1, bad
    assert call(n=0, z=None, norm=None, dz=None) == 0


def test_distill_arguments(lib):
    def call(ty=0, z=4096, ldz=8, n=2, c=8, k=2, top=4096, index=4096, w=4096, T=1.0, loss=4096, dz=8192, ldd=8):
        return lib.lipcache_distill(ty, z, ldz, n, c, k, top, index, w, T, loss, dz, ldd, None)
    for bad in ROWS + TEMPERATURES + [dict(k=0), dict(k=129), dict(top=None), dict(index=None), dict(ldd=7),
                                      dict(dz=4096, ldd=9), dict(dz=8193), dict(top=4098), dict(index=4098), dict(w=4097),
                                      dict(loss=4098)]:
        assert call(**bad) == 1, bad
    assert call(n=0, z=None, top=None, index=None) == 0
    assert call(loss=None, dz=None) == 0  # nothing asked for


def test_layer_norm_arguments(lib):
    sizes = [dict(ty=2), dict(n=-1), dict(n=(1 << 24) + 1), dict(d=0), dict(d=65_537)]

    def fwd(ty=0, x=4096, ldx=8, n=2, d=8, w=4096, b=4096, eps=1e-5, y=8192, ldy=8, stats=4096):
        return lib.lipcache_layer_norm(ty, x, ldx, n, d, w, b, eps, y, ldy, stats, None)
    for bad in sizes + [dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7), dict(x=4097), dict(y=4098), dict(w=4098),
                        dict(b=4097), dict(stats=4098), dict(eps=0.0), dict(eps=1.5), dict(eps=math.nan)]:
        assert fwd(**bad) == 1, bad
    assert fwd(n=0, x=None, y=None) == 0
    for bad in sizes:
        a = dict(ty=0, n=2, d=8)
        a.update(bad)
        assert lib.lipcache_layer_norm_workspace(a["ty"], a["n"], a["d"]) == -1, bad
    assert lib.lipcache_layer_norm_workspace(0, 0, 8) == 0
    assert lib.lipcache_layer_norm_workspace(1, 500, 65_536) >= 2 * 65_536 * 4
    assert lib.lipcache_layer_norm_workspace(1, 2, 65_536) == 0  # few rows need none


def test_layer_norm_workspace_is_what_blocks_write(lib):
    """Two sums a column of each block: of an SM's blocks, or of clusters that share a wide row, not more."""
    for d, blocks in ((8, 3 * 152), (256, 3 * 152), (257, 2 * 152), (512, 2 * 152), (1000, 152), (8192, 152), (8193, 76),
                      (20_000, 38), (40_000, 19), (65_536, 19)):
        for ty in (0, 1):
            assert lib.lipcache_layer_norm_workspace(ty, 1 << 20, d) <= blocks * 2 * d * 4, d
            assert lib.lipcache_layer_norm_workspace(ty, 10, d) in (0, 10 * 2 * d * 4), d


def test_layer_norm_backward_arguments(lib):
    big = 1 << 40  # a workspace size; the refusals come before any use

    def call(ty=0, dy=4096, lddy=8, x=4096, ldx=8, n=2000, d=8, stats=4096, w=4096, dx=8192, lddx=8, dw=4096, db=4096,
             ws=4096, nb=big):
        return lib.lipcache_layer_norm_backward(ty, dy, lddy, x, ldx, n, d, stats, w, dx, lddx, dw, db, ws, nb, None)
    for bad in (dict(ty=5), dict(n=-1), dict(d=0), dict(d=65_537), dict(dy=None), dict(x=None), dict(stats=None), dict(lddy=7),
                dict(ldx=7), dict(lddx=7), dict(dy=4098), dict(x=4097), dict(dx=8194), dict(stats=4098), dict(w=4098),
                dict(dw=4098), dict(db=4097), dict(ws=None), dict(ws=4100), dict(nb=16), dict(nb=-1)):
        assert call(**bad) == 1, bad
    assert call(dx=None, dw=None, db=None) == 0  # nothing asked for
    assert call(n=0, dy=None, x=None, stats=None, dw=None, db=None) == 0
