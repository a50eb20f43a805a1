"""Host-side checks of the operators around the layers: sizes of operands and workspaces, and arguments that are
rejected before any launch.  Nothing runs on a GPU here."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2010_14298_amd", "libfqt.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libfqt.so not built")

FAKE = 0x1000  # never dereferenced: validation fails first
WS = 1 << 40


@pytest.fixture(scope="module")
def lib():
    from paper_2010_14298_amd import fqt
    return fqt.load()


def op(q=FAKE, e=FAKE, k_major=0):
    from paper_2010_14298_amd import fqt
    return ctypes.byref(fqt.Fp8(q, e, k_major))


def test_sizes(lib):
    assert [lib.fqt_fp8_pitch(k) for k in (0, 1, 128, 129)] == [0, 128, 128, 256]
    assert lib.fqt_fp8_exp_bytes(5, 128) == 20 and lib.fqt_fp8_exp_bytes(5, 513) == 40
    assert lib.fqt_fp8_exp_bytes(0, 128) == 0
    assert lib.fqt_layernorm_backward_workspace(0, 4) == 0
    assert lib.fqt_layernorm_backward_workspace(100, 64) >= 2 * 64 * 4
    # the operands of the activations, or of both quantizations of the gradient
    assert lib.fqt_fp8_linear_forward_workspace(300, 1000, 64) >= 300 * 1024
    assert lib.fqt_fp8_linear_backward_workspace(300, 1000, 64) >= 300 * 128 + 64 * 384
    assert lib.fqt_fp8_linear_forward_workspace(1, 0, 1) == 0 and lib.fqt_fp8_gemm_workspace(1, 1, 0) == 0
    assert lib.fqt_grad_norm_clip_workspace(0) == 0
    assert lib.fqt_grad_norm_clip_workspace(1000) > lib.fqt_grad_norm_clip_workspace(1)


def test_layernorm_arguments(lib):
    def fwd(x=FAKE, t=0, rows=4, cols=8, ldx=8, eps=1e-5, y=FAKE, ldy=8, gamma=None):
        return lib.fqt_layernorm_forward(x, t, rows, cols, ldx, gamma, None, eps, y, ldy, None, None, None)
    for bad in (dict(x=None), dict(t=3), dict(rows=0), dict(cols=0), dict(rows=1 << 31), dict(ldx=-1), dict(ldy=7),
                dict(x=FAKE + 2), dict(t=1, x=FAKE + 1), dict(eps=-1e-5), dict(eps=float("inf")), dict(gamma=FAKE + 2)):
        assert fwd(**bad) == 1, bad

    def bwd(g=FAKE, x=FAKE, t=0, rows=4, cols=8, mean=FAKE, gx=FAKE, gg=FAKE, gb=FAKE, ws=FAKE, n=WS, ld=8):
        return lib.fqt_layernorm_backward(g, ld, x, 8, t, rows, cols, mean, FAKE, None, gx, ld, gg, gb, ws, n, None)
    for bad in (dict(g=None), dict(x=None), dict(mean=None), dict(gx=None), dict(t=-1), dict(rows=0), dict(ld=7)):
        assert bwd(**bad) == 1, bad
    assert bwd(ws=None) == 4 and bwd(n=16) == 4 and bwd(ws=FAKE + 4) == 4 and bwd(gg=None, n=16) == 4


def test_fp8_arguments(lib):
    def quant(x=FAKE, t=0, rows=4, cols=8, ld=8, tile=0, sr=0, a=op(), b=op()):
        return lib.fqt_fp8_quantize(x, t, rows, cols, ld, tile, sr, 0, a, b, None)
    for bad in (dict(x=None), dict(t=5), dict(rows=0), dict(cols=0), dict(tile=2), dict(sr=-1), dict(a=None, b=None),
                dict(a=op(None)), dict(b=op(FAKE, None)), dict(a=op(FAKE + 8)), dict(a=op(FAKE, FAKE + 2)), dict(ld=-1),
                dict(a=op(FAKE, FAKE, 1)), dict(b=op(FAKE, FAKE, 2))):
        assert quant(**bad) == 1, bad

    def gemm(A=op(), B=op(), M=4, N=8, K=8, t=0, relu=0, mask=None, ldm=8, C=FAKE, ldc=8, ws=FAKE, n=WS):
        return lib.fqt_fp8_gemm(A, B, M, N, K, t, relu, mask, ldm, C, ldc, ws, n, None)
    for bad in (dict(A=None), dict(B=op(None)), dict(B=op(FAKE, FAKE, 2)), dict(M=0), dict(K=0), dict(N=1 << 31), dict(t=4), dict(relu=2),
                dict(mask=FAKE + 1), dict(C=None), dict(ldc=7)):
        assert gemm(**bad) == 1, bad

    # longer contractions than a tile's offsets reach
    assert gemm(K=(1 << 23) + 1) == 2

    def fwd(X=FAKE, t=0, N=4, i=8, ldx=8, W=op(), o=8, relu=0, Y=FAKE, ldy=8, Xt=None, ws=FAKE, n=WS):
        return lib.fqt_fp8_linear_forward(X, t, N, i, ldx, W, o, relu, Y, ldy, Xt, ws, n, None)
    for bad in (dict(X=None), dict(W=None), dict(N=0), dict(o=0), dict(relu=3), dict(Y=None), dict(ldy=7),
                dict(Xt=op(None)), dict(Xt=op(FAKE, FAKE, 1)), dict(t=9)):
        assert fwd(**bad) == 1, bad
    assert fwd(ws=None) == 4 and fwd(n=64) == 4 and fwd(i=(1 << 23) + 1) == 2

    def bwd(G=FAKE, t=0, N=4, o=8, X=op(), W=op(), i=8, sr=1, r=None, gw=FAKE, gx=FAKE, ldgx=8, ws=FAKE, n=WS):
        return lib.fqt_fp8_linear_backward(G, t, N, o, 8, X, W, i, sr, 0, r, 8, gw, gx, ldgx, ws, n, None)
    for bad in (dict(G=None), dict(gw=None, gx=None), dict(X=None), dict(W=None), dict(sr=2), dict(r=FAKE + 1),
                dict(ldgx=7), dict(i=0)):
        assert bwd(**bad) == 1, bad
    assert bwd(ws=None) == 4 and bwd(n=64) == 4 and bwd(N=(1 << 23) + 1) == 2
    # what is not formed needs no operand: the next check fails, the workspace's
    assert bwd(gw=None, X=None, n=64) == 4 and bwd(gx=None, W=None, n=64) == 4


def test_clip_arguments(lib):
    def clip(g=(FAKE,), o=None, n=(10,), t=(0,), count=1, max_norm=1.0, ws=FAKE, nb=WS, norm=None):
        arr = (ctypes.c_uint64 * max(1, len(g)))(*[p or 0 for p in g])
        outs = (ctypes.c_uint64 * len(o))(*[p or 0 for p in o]) if o is not None else None
        return lib.fqt_grad_norm_clip(arr, outs, (ctypes.c_int64 * len(n))(*n), (ctypes.c_int32 * len(t))(*t), count,
                                      max_norm, norm, ws, nb, None)
    for bad in (dict(count=0), dict(count=-1), dict(max_norm=0.0), dict(max_norm=float("nan")), dict(t=(3,)),
                dict(n=(-1,)), dict(g=(None,)), dict(g=(FAKE + 2,)), dict(o=(None,)), dict(o=(FAKE + 1,)),
                dict(norm=FAKE + 2)):
        assert clip(**bad) == 1, bad
    assert clip(ws=None) == 4 and clip(nb=64) == 4
    # more chunks than the table's 32-bit counters hold
    assert clip(g=(FAKE,) * 90, n=(1 << 40,) * 90, t=(0,) * 90, count=90) == 2
