"""Host-side checks of the gated layer and the checkpoints: sizes, and arguments that are rejected before any launch.
Nothing runs on a GPU here."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2010_14298_amd", "libfqt.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libfqt.so not built")

FAKE = 0x1000  # never dereferenced: validation fails first
WS = 1 << 50


@pytest.fixture(scope="module")
def lib():
    from paper_2010_14298_amd import fqt
    return fqt.load()


def op(q=FAKE, e=FAKE, k_major=0):
    from paper_2010_14298_amd import fqt
    return ctypes.byref(fqt.Fp8(q, e, k_major))


def kept(q=FAKE, e=FAKE):
    from paper_2010_14298_amd import fqt
    return ctypes.byref(fqt.Kept(q, e))


def test_sizes(lib):
    assert [lib.fqt_fp8_kept_pitch(c) for c in (-1, 0, 1, 32, 33, 1 << 31)] == [0, 0, 32, 32, 64, 0]
    assert lib.fqt_fp8_gated_forward_workspace(300, 1000, 64, 0, 1) >= 300 * 1024
    assert lib.fqt_fp8_gated_forward_workspace(300, 1000, 64, 1, 0) >= 300 * 1024 + 128 * 1024
    # few rows that keep nothing are read as they are
    assert lib.fqt_fp8_gated_forward_workspace(1, 1000, 64, 0, 0) == 0
    assert lib.fqt_fp8_gated_forward_workspace(1, 1000, 64, 0, 1) > 0
    assert lib.fqt_fp8_gated_forward_workspace(1, 1000, 64, 1, 0) >= 128 * 1024
    assert lib.fqt_fp8_gated_backward_workspace(300, 1000, 64) >= 300 * 128 + 128 * 384
    for bad in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (8, 8, 1 << 29), (1 << 31, 8, 8), (8, 8, -1)):
        assert lib.fqt_fp8_gated_forward_workspace(*bad, 1, 1) == 0 and lib.fqt_fp8_gated_backward_workspace(*bad) == 0


def test_layernorm8_arguments(lib):
    def fwd(x=FAKE, t=0, rows=4, cols=8, ldx=8, eps=1e-5, y=FAKE, ldy=8, gamma=None, k=kept(), r=FAKE):
        return lib.fqt_layernorm_forward8(x, t, rows, cols, ldx, gamma, None, eps, y, ldy, k, r, None)
    for bad in (dict(x=None), dict(t=3), dict(rows=0), dict(cols=0), dict(rows=1 << 31), dict(ldx=-1), dict(ldy=7),
                dict(x=FAKE + 2), dict(eps=-1e-5), dict(eps=float("nan")), dict(gamma=FAKE + 2), dict(k=None),
                dict(k=kept(None)), dict(k=kept(FAKE, None)), dict(k=kept(FAKE + 8)), dict(r=None), dict(r=FAKE + 2)):
        assert fwd(**bad) == 1, bad

    def bwd(g=FAKE, k=kept(), t=0, rows=4, cols=8, r=FAKE, gx=FAKE, gg=FAKE, gb=FAKE, ws=FAKE, n=WS, ld=8):
        return lib.fqt_layernorm_backward8(g, ld, k, t, rows, cols, r, None, gx, ld, gg, gb, ws, n, None)
    for bad in (dict(g=None), dict(k=None), dict(k=kept(None)), dict(k=kept(FAKE + 4)), dict(r=None), dict(gx=None),
                dict(t=-1), dict(rows=0), dict(ld=7), dict(r=FAKE + 1)):
        assert bwd(**bad) == 1, bad
    assert bwd(ws=None) == 4 and bwd(n=16) == 4 and bwd(ws=FAKE + 4) == 4 and bwd(gg=None, n=16) == 4


def test_gated_arguments(lib):
    def fwd(X=FAKE, t=0, N=4, i=8, ldx=8, W=op(), h=8, act=0, H=FAKE, ldh=8, Xt=op(), a=kept(), b=kept(), ws=FAKE, n=WS):
        return lib.fqt_fp8_gated_forward(X, t, N, i, ldx, W, h, act, H, ldh, Xt, a, b, ws, n, None)
    for bad in (dict(X=None), dict(t=9), dict(N=0), dict(N=1 << 31), dict(i=0), dict(ldx=-1), dict(W=None),
                dict(W=op(None)), dict(W=op(FAKE, FAKE, 2)), dict(h=0), dict(h=1 << 29), dict(act=3), dict(act=-1),
                dict(H=None), dict(ldh=7), dict(Xt=op(FAKE, FAKE, 1)), dict(Xt=op(None)), dict(a=kept(None)),
                dict(b=kept(FAKE, None)), dict(b=kept(FAKE + 4))):
        assert fwd(**bad) == 1, bad
    assert fwd(ws=None) == 4 and fwd(n=64) == 4 and fwd(ws=FAKE + 8) == 4 and fwd(i=(1 << 23) + 1) == 2
    # nothing kept: the next check fails, the workspace's
    assert fwd(Xt=None, a=None, b=None, W=op(FAKE, FAKE, 1), n=64) == 4

    def bwd(G=FAKE, t=0, N=4, h=8, ldg=8, a=kept(), b=kept(), X=op(), W=op(), i=8, sr=1, gw=FAKE, gx=FAKE, ldgx=8,
            ws=FAKE, n=WS):
        return lib.fqt_fp8_gated_backward(G, t, N, h, ldg, a, b, X, W, i, sr, 0, gw, gx, ldgx, ws, n, None)
    for bad in (dict(G=None), dict(t=4), dict(N=0), dict(h=0), dict(h=1 << 29), dict(ldg=-1), dict(a=None), dict(b=None),
                dict(a=kept(FAKE, None)), dict(b=kept(FAKE + 8)), dict(X=None), dict(W=None), dict(gw=None, gx=None),
                dict(sr=2), dict(ldgx=7), dict(i=0), dict(gw=FAKE + 2)):
        assert bwd(**bad) == 1, bad
    assert bwd(ws=None) == 4 and bwd(n=64) == 4
    assert bwd(N=(1 << 23) + 1) == 2 and bwd(h=(1 << 22) + 1) == 2
    # what is not contracted may be longer, what is not formed needs no operand: the workspace's check fails
    assert bwd(N=(1 << 23) + 1, gw=None, X=None, n=64) == 4 and bwd(h=(1 << 22) + 1, gx=None, W=None, n=64) == 4
