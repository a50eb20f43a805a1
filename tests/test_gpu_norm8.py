"""Layer norm with an 8-bit checkpoint against the float64 oracle.

Forward: Y and rstd as without a checkpoint (the same bits).  xh is off by e = 66 2^-24 (max|x| rstd + (1 + 2 max|x| rstd)
|xh|): a sum 64 additions deep in the mean and in the variance, where the mean's error enters twice; a code adds half a
step of the format at its block's scale.

Backward: xh is what the checkpoint holds.  grad_X = rstd (c - mean c - xh mean(c xh)): sums of at most 64 additions in
depth and a handful of roundings, 72 2^-24 of rstd (|c| + mean|c| + |xh| mean|c xh|), and its type's rounding; rows longer
than 16384 columns add one after the other in each thread, cols / 1024 more.  The parameters' gradients add rows one after
the other, rows + 64 at most."""
import numpy as np
import pytest

from oracle import feedforward as F
from oracle import gated as G

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 1), (1, 31), (2, 32), (3, 33), (5, 256), (7, 257), (300, 130), (40, 512), (33, 1000), (129, 1024), (20, 2048),
         (9, 4096), (6, 8192), (3, 16384), (2, 16385), (4, 20011), (600, 6001), (300, 9002)]


def fqt():
    from paper_2010_14298_amd import fqt as f
    f.load()
    return f


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def inputs(rows, cols, dtype, seed=0):
    rng = np.random.default_rng(seed + rows + cols)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.normal(0, 0.5, (rows, 1))) + rng.standard_normal((rows, 1))
    g = rng.standard_normal((rows, cols)) * np.where(rng.random((rows, 1)) < 0.1, 0.0, 1.0)
    v = [torch.from_numpy(t.astype(np.float32)).cuda() for t in
         (1 + 0.3 * rng.standard_normal(cols), 0.3 * rng.standard_normal(cols))]
    return torch.from_numpy(x).to(dtype).cuda(), torch.from_numpy(g).to(dtype).cuda(), v[0], v[1]


def values(k):
    return G.kept_values(k["q"].view(torch.uint8).cpu().numpy(), k["exp"].cpu().numpy(), k["cols"])


def check_checkpoint(k, x):
    rows, cols = x.shape
    xh, _, rstd = F.layernorm(x)
    depth = 66 + (cols // 1024 if cols > 16384 else 0)
    big = (np.abs(x).max(1) * rstd)[:, None]
    err = depth * U * (big + (1 + 2 * big) * np.abs(xh))
    q, exp = k["q"].view(torch.uint8).cpu().numpy(), k["exp"].cpu().numpy()
    nb = -(-cols // 32)
    assert q.shape == (rows, nb * 32) and exp.shape == (rows, nb) and (q[:, cols:] == 0).all()
    pad = ((0, 0), (0, nb * 32 - cols))
    top, slack = (np.pad(t, pad).reshape(rows, nb, 32).max(2) for t in (np.abs(xh), err))
    E = exp.astype(int) - 127
    assert np.all(top - slack <= 448.0 * 2.0 ** E)
    assert np.all((top + slack > 448.0 * 2.0 ** (E - 1.0)) | (top <= slack))
    scale = np.repeat(2.0 ** E, 32, axis=1)[:, :cols]
    step = 2.0 ** (np.floor(np.log2(np.maximum((np.abs(xh) + err) / scale, 2.0 ** -6))) - 3) * scale
    assert np.all(np.abs(values(k) - xh) <= err + 0.5 * step)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype):
    f = fqt()
    x, _, gamma, beta = inputs(rows, cols, dtype)
    Y, xh8, rstd = f.fqt_layernorm_forward8(x, gamma, beta)
    plain, _, r = f.fqt_layernorm_forward(x, gamma, beta)
    assert torch.equal(Y, plain) and torch.equal(rstd, r)
    check_checkpoint(xh8, host(x))
    Y, again, _ = f.fqt_layernorm_forward8(x)
    assert torch.equal(Y, f.fqt_layernorm_forward(x)[0])
    assert torch.equal(again["q"].view(torch.uint8), xh8["q"].view(torch.uint8))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(rows, cols, dtype):
    f = fqt()
    x, g, gamma, beta = inputs(rows, cols, dtype)
    _, xh8, rstd = f.fqt_layernorm_forward8(x, gamma, beta)
    gX, gg, gb, ws = f.fqt_layernorm_backward8(g, xh8, rstd, gamma)
    xh, gd, ga, r = values(xh8), host(g), host(gamma), host(rstd)
    wx, wg, wb = G.layernorm_backward8(gd, xh, r, ga)
    c = gd * ga
    depth = 72 + (cols // 1024 if cols > 16384 else 0)
    size = r[:, None] * (np.abs(c) + np.abs(c).mean(1, keepdims=True)
                         + np.abs(xh) * np.abs(c * xh).mean(1, keepdims=True))
    tol = depth * U * size
    assert np.all(np.abs(host(gX) - wx) <= tol + HALF[dtype] * (np.abs(wx) + tol) + TINY[dtype])
    assert np.all(np.abs(host(gg) - wg) <= (rows + 64) * U * np.abs(gd * xh).sum(0))
    assert np.all(np.abs(host(gb) - wb) <= (rows + 64) * U * np.abs(gd).sum(0))
    only, a, b, _ = f.fqt_layernorm_backward8(g, xh8, rstd, gamma, params=False)
    assert a is None and b is None and torch.equal(only, gX)
    out = torch.full((rows, cols + 5), 3.0, dtype=dtype, device="cuda")
    f.fqt_layernorm_backward8(g, xh8, rstd, gamma, grad_X=out[:, 2:cols + 2], ws=ws)
    assert torch.equal(out[:, 2:cols + 2], gX) and (out[:, :2] == 3).all() and (out[:, cols + 2:] == 3).all()


def test_many_rows():
    f = fqt()
    x, g, gamma, beta = inputs(5003, 96, torch.bfloat16)
    Y, xh8, rstd = f.fqt_layernorm_forward8(x, gamma, beta)
    check_checkpoint(xh8, host(x))
    gX, gg, gb, _ = f.fqt_layernorm_backward8(g, xh8, rstd, gamma)
    wx, wg, wb = G.layernorm_backward8(host(g), values(xh8), host(rstd), host(gamma))
    assert np.abs(host(gX) - wx).max() <= 2.0 ** -8 * np.abs(wx).max()
    assert np.all(np.abs(host(gg) - wg) <= 5067 * U * np.abs(host(g) * values(xh8)).sum(0))
    assert np.all(np.abs(host(gb) - wb) <= 5067 * U * np.abs(host(g)).sum(0))


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_and_repeated_rows(dtype):
    f = fqt()
    x, g, gamma, beta = inputs(37, 300, dtype)
    want = f.fqt_layernorm_forward8(x, gamma, beta)
    bx, bg = (torch.full((37, 311), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    bx[:, 3:303], bg[:, 5:305] = x, g
    got = f.fqt_layernorm_forward8(bx[:, 3:303], gamma, beta)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1]["exp"], want[1]["exp"])
    assert torch.equal(got[1]["q"].view(torch.uint8), want[1]["q"].view(torch.uint8))
    a = f.fqt_layernorm_backward8(g, want[1], want[2], gamma)
    b = f.fqt_layernorm_backward8(bg[:, 5:305], want[1], want[2], gamma)
    assert all(torch.equal(p, q) for p, q in zip(a[:3], b[:3]))
    one = f.fqt_layernorm_forward8(x[:1].expand(37, 300), gamma, beta)
    assert torch.equal(one[0], want[0][:1].expand(37, 300))


def test_constant_zero_and_non_finite_rows():
    """A row of one value has xh = 0 (scale byte 127); a NaN or an infinity makes its whole row NaN, and no other."""
    f = fqt()
    x, g, gamma, beta = inputs(6, 100, torch.float32)
    x[1], x[2], x[3, 50], x[4, 7] = 0.0, 2.5, float("nan"), float("inf")
    Y, xh8, rstd = f.fqt_layernorm_forward8(x, gamma, beta)
    assert (xh8["q"][1:3].float() == 0).all() and (xh8["exp"][1:3] == 127).all()
    assert (xh8["exp"][3:5] == 255).all() and torch.isnan(xh8["q"][3:5].float()).all()
    assert (xh8["exp"][[0, 5]] < 255).all()
    gX = f.fqt_layernorm_backward8(g, xh8, rstd, gamma)[0]
    assert torch.isnan(gX[3:5]).all() and torch.isfinite(gX[[0, 5]]).all()


def test_extreme_rows():
    """Rows of float32's smallest and largest magnitudes, eps 0: xh stays of order one."""
    f = fqt()
    x, _, _, _ = inputs(4, 64, torch.float32)
    x[1] *= 2.0 ** 60
    x[2] *= 2.0 ** -55
    _, xh8, _ = f.fqt_layernorm_forward8(x, eps=0.0)
    _, same, _ = f.fqt_layernorm_forward8(inputs(4, 64, torch.float32)[0], eps=0.0)
    assert torch.equal(xh8["q"].view(torch.uint8), same["q"].view(torch.uint8)) and torch.equal(xh8["exp"], same["exp"])


def test_gradients_against_differences():
    """The loss sum(G Y) by differences in float64: the checkpoint's noise of 2.6 % an element leaves the gradient's
    direction within 3 % (it enters once, and once through a mean)."""
    f = fqt()
    x, g, gamma, beta = inputs(6, 90, torch.float32)
    _, xh8, rstd = f.fqt_layernorm_forward8(x, gamma, beta)
    gX, gg, gb, _ = f.fqt_layernorm_backward8(g, xh8, rstd, gamma)
    xd, gd, ga, be = host(x), host(g), host(gamma), host(beta)

    def loss(x, ga, be):
        return float((gd * F.layernorm(x, ga, be)[0]).sum())
    rng = np.random.default_rng(0)
    for got, of, shape in ((gX, lambda d: loss(xd + d, ga, be), xd.shape), (gg, lambda d: loss(xd, ga + d, be), ga.shape),
                           (gb, lambda d: loss(xd, ga, be + d), be.shape)):
        num, kernel = [], []
        for _ in range(40):
            d = rng.standard_normal(shape)
            num.append((of(1e-6 * d) - of(-1e-6 * d)) / 2e-6)
            kernel.append(float((host(got) * d).sum()))
        num, kernel = np.array(num), np.array(kernel)
        assert num @ kernel / np.linalg.norm(num) / np.linalg.norm(kernel) > 0.99


def test_refusals():
    f = fqt()
    x, g, gamma, beta = inputs(5, 40, torch.bfloat16)
    _, xh8, rstd = f.fqt_layernorm_forward8(x, gamma, beta)
    for call in (lambda: f.fqt_layernorm_forward8(x.cpu()), lambda: f.fqt_layernorm_forward8(x, gamma[:39]),
                 lambda: f.fqt_layernorm_forward8(x.t()), lambda: f.fqt_layernorm_forward8(x, Y=x.float()),
                 lambda: f.fqt_layernorm_backward8(g[:4], xh8, rstd), lambda: f.fqt_layernorm_backward8(g, xh8, rstd[:4]),
                 lambda: f.fqt_layernorm_backward8(g[:, :39], xh8, rstd),
                 lambda: f.fqt_layernorm_backward8(g, dict(xh8, q=xh8["q"].cpu()), rstd),
                 lambda: f.fqt_layernorm_backward8(g, dict(xh8, exp=xh8["exp"][:, :1]), rstd),
                 lambda: f.fqt_layernorm_backward8(g, xh8, rstd.double()),
                 lambda: f.fqt_layernorm_backward8(g, xh8, rstd, ws=torch.empty(1 << 20, device="cuda"))):
        with pytest.raises(ValueError):
            call()
