"""The gated forward of few rows that keeps nothing, at widths that take its waves of a block several turns along K:
eight waves of a float32 block (and of a 16-bit one up to 1024 columns) make a second turn from 9 blocks of 128 on, the
sixteen of a wider 16-bit block from 17 on.  Tolerances: those of test_gpu_gated.py."""
import numpy as np
import pytest

from oracle import gated as G
from tests import test_gpu_gated as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = base.TYPES
# one block past 8, whole blocks, one element past 17 blocks, a few past 32, 47 of which the last is ragged
WIDTHS = [1025, 2048, 2177, 4100, 6000]


def serve(X, W8, act="silu", **how):
    """H of a call that keeps nothing, of rows that are read as they are (no workspace)."""
    H, kept, ws = base.fqt().fqt_fp8_gated_forward(X, W8, act=act, save=False, **how)
    assert kept is None and ws is None
    return H


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d_in", WIDTHS)
@pytest.mark.parametrize("N,hidden,act", [(1, 129, "silu"), (16, 37, "gelu_tanh"), (17, 200, "relu"), (33, 45, "silu"),
                                          (5, 1, "gelu_tanh")])
def test_long_rows(N, hidden, act, d_in, dtype):
    X = base.matrix(N + d_in, N, d_in, dtype)
    W, W8, _ = base.weights(hidden, hidden, d_in)
    base.check_forward(X, W, act, serve(X, W8, act), None, d_in)


@pytest.mark.parametrize("d_in", WIDTHS)
@pytest.mark.parametrize("N", [1, 16, 17, 40])
@pytest.mark.parametrize("dtype", TYPES)
def test_exact_sums_give_the_oracles_bits(dtype, N, d_in):
    """Whole numbers up to 4: sums below 2^24 are exact in any order, so H is the product of two of them rounded once.
    The first and last column of K count in every row and hidden unit."""
    rng = np.random.default_rng(N + d_in)
    hidden = 35
    x = rng.integers(-4, 5, (N, d_in)) * (rng.random((N, d_in)) < 0.1)
    w = rng.integers(-2, 3, (2 * hidden, d_in)) * (rng.random((2 * hidden, d_in)) < 0.2)
    x[:, [0, -1]], w[:, [0, -1]] = rng.integers(1, 5, (N, 2)), rng.integers(1, 3, (2 * hidden, 2))
    X = torch.from_numpy(x.astype(np.float32)).to(dtype).cuda()
    W8, _ = base.fqt().fqt_fp8_quantize(torch.from_numpy(w.astype(np.float32)).cuda(), tile=True)
    want = torch.from_numpy(G.gated_forward(x, w, "relu")["H"])
    assert float(want.abs().max()) < 2.0 ** 15
    assert torch.equal(serve(X, W8, "relu").cpu(), want.float().to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("N", [1, 9, 33])
def test_non_finite_rows_stay_in_their_rows(N, bad, dtype):
    """In any turn of any wave, the ragged last block's included: the row is NaN, the others keep their bits."""
    d_in, hidden = 2177, 70
    X = base.matrix(3, N, d_in, dtype)
    _, W8, _ = base.weights(4, hidden, d_in)
    for act in ("silu", "gelu_tanh", "relu"):
        want = serve(X, W8, act)
        assert torch.isfinite(want).all()
        for col in (7, 900, 1100, 2047, 2050, 2176):
            Y = X.clone()
            Y[N // 2, col] = bad
            H = serve(Y, W8, act)
            rows = torch.arange(N, device="cuda") != N // 2
            assert torch.equal(H[rows], want[rows]) and torch.isnan(H[N // 2]).all(), (act, col)


@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dtype,big", [(torch.float32, 2.0 ** 60), (torch.bfloat16, 2.0 ** 60), (torch.float16, 2.0 ** 7)])
@pytest.mark.parametrize("at", [0, 1030, 2176])
def test_saturated_activations(at, dtype, big, act):
    """Pre-activations of big and -big, wherever along K they come from: H is big^2 and next to 0."""
    X = torch.zeros((3, 2177), dtype=dtype, device="cuda")
    X[0, at], X[1, at] = big, -big
    W = torch.zeros((64, 2177), device="cuda")
    W[:, at] = 1.0
    W8, _ = base.fqt().fqt_fp8_quantize(W, tile=True)
    H = serve(X, W8, act)
    assert (H[0] == big * big).all() and (H[2] == 0).all()
    # |a s(a) b| with s(a) <= exp(-128): below 2^14 exp(-128) for 2^7, 0 for 2^60
    assert (H[1].abs() <= 2.0 ** -100).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [1, 9, 33])
@pytest.mark.parametrize("d_in", [200, 2177])
def test_strides_and_rows_behind_stay(d_in, N, dtype):
    """X and H inside larger buffers, NaN around X; one row over and over; weights column by column."""
    X = base.matrix(5, N, d_in, dtype)
    _, W8, _ = base.weights(6, 70, d_in)
    want = serve(X, W8)
    buf = torch.full((N + 1, d_in + 17), float("nan"), dtype=dtype, device="cuda")
    buf[:N, 5:d_in + 5] = X
    out = torch.full((N + 3, 79), 7.0, dtype=dtype, device="cuda")
    H = serve(buf[:N, 5:d_in + 5], W8, H=out[1:N + 1, 3:73])
    assert torch.equal(H, want)
    assert (out[0] == 7).all() and (out[N + 1:] == 7).all() and (out[:, :3] == 7).all() and (out[:, 73:] == 7).all()
    repeated = serve(X[:1].expand(N, d_in), W8)
    assert torch.equal(repeated, repeated[:1].expand(N, 70)) and torch.equal(repeated[0], want[0])
    turned = dict(q=W8["q"].t().contiguous().t(), exp=W8["exp"], K=W8["K"])
    assert torch.equal(base.fqt().fqt_fp8_gated_forward(X, turned, save=False)[0], want)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_row_has_the_same_bits_with_any_rows_beside_it(dtype):
    """As long as the rows are read as they are: a row's sums do not depend on which of the sixteen it is."""
    X = base.matrix(8, 33, 2177, dtype)
    _, W8, _ = base.weights(9, 100, 2177)
    want = serve(X, W8)
    for a, b in ((0, 1), (5, 6), (32, 33), (3, 20), (16, 33)):
        assert torch.equal(serve(X[a:b], W8), want[a:b])
