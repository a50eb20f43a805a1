"""Layer norm forward and backward against the float64 oracle.

Tolerances, from float32 arithmetic (u = 2^-24) and the output type's rounding (half a unit in the last place: 2^-24,
2^-8, 2^-11 of the value, and half the smallest subnormal step of float16):

* mean: a sum of up to cols terms in a tree of at most 64 additions deep: 64 u mean|x|, and the division.
* rstd: that error of the mean enters the variance squared; the sum of squares has the same depth: 64 u rstd, and
  twice the mean's error over the deviation (rows whose deviation is far below their mean lose digits by nature).
* Y = (x - mean) rstd gamma + beta: 64 u (max|x| rstd |gamma| + |y| + |beta|) and rstd's relative error of |y - beta|.
* grad_X: rstd (c - a - xh b): 64 u rstd (|c| + mean|c| + |xh| mean|c xh| + |xh| max|xh|-weighted terms), bounded by
  192 u rstd (max|c| (1 + |xh|)^2 + mean|c| + |xh| mean|c xh|).
* grad_gamma, grad_beta: sums over the rows, each at most rows additions: u (rows + 64) sum|g| (|xh| + max|x| rstd).
"""
import numpy as np
import pytest

from oracle import feedforward as F

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 0.0, "bfloat16": 0.0, "float16": 2.0 ** -25}
EPS = 1e-5


def fqt():
    from paper_2010_14298_amd import fqt as f
    f.load()
    return f


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def inputs(rows, cols, dtype, seed=0, offset=1.0):
    rng = np.random.default_rng(seed)
    dt = getattr(torch, dtype)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.normal(0, 0.5, (rows, 1))) + offset * rng.standard_normal((rows, 1))
    g = rng.standard_normal((rows, cols)) * np.where(rng.random((rows, 1)) < 0.1, 0.0, 1.0)
    gamma = (1 + 0.3 * rng.standard_normal(cols)).astype(np.float32)
    beta = (0.3 * rng.standard_normal(cols)).astype(np.float32)
    return (torch.from_numpy(x).to(dt).cuda(), torch.from_numpy(g).to(dt).cuda(), torch.from_numpy(gamma).cuda(),
            torch.from_numpy(beta).cuda())


def check_forward(x, gamma, beta, Y, mean, rstd, eps=EPS):
    xd, dt = host(x), str(Y.dtype).split(".")[1]
    ga = host(gamma) if gamma is not None else np.ones(x.shape[1])
    be = host(beta) if beta is not None else np.zeros(x.shape[1])
    y, m, r = F.layernorm(xd, ga, be, eps)
    dm = 66 * U * np.abs(xd).mean(1)
    assert np.all(np.abs(host(mean) - m) <= dm)
    # relative: the variance's own sum, the square of the mean's error, eps's rounding; 1/sqrt and rounding
    dr = 66 * U + (dm * r) ** 2 + 2 * dm * r
    assert np.all(np.abs(host(rstd) - r) <= dr * r)
    top = np.abs(xd).max(1, keepdims=True)
    tol = 66 * U * (top * r[:, None] * np.abs(ga) + np.abs(y) + np.abs(be)) + dr[:, None] * np.abs(y - be)
    tol = tol + HALF[dt] * np.abs(y) + TINY[dt]
    assert np.all(np.abs(host(Y) - y) <= tol)


def check_backward(g, x, gamma, gx, gg, gb):
    gd, xd, dt = host(g), host(x), str(gx.dtype).split(".")[1]
    ga = host(gamma) if gamma is not None else np.ones(x.shape[1])
    wx, wg, wb = F.layernorm_backward(gd, xd, ga, EPS)
    xh, m, r = F.layernorm(xd, eps=EPS)
    c, r = np.abs(gd * ga), r[:, None]
    # xh itself is off by the error of the float32 mean and rstd that the forward hands over
    dx = 66 * U * (np.abs(xd).max(1, keepdims=True) * r + np.abs(xh)) + 132 * U * (np.abs(xd).mean(1, keepdims=True) * r) * np.abs(xh)
    cm, cx = c.mean(1, keepdims=True), (c * (np.abs(xh) + dx)).mean(1, keepdims=True)
    tol = r * (66 * U * (c + cm + np.abs(xh) * cx) + np.abs(xh) * (c * dx).mean(1, keepdims=True) + dx * cx)
    tol = tol + 132 * U * (1 + np.abs(xd).mean(1, keepdims=True) * r) * np.abs(wx) + HALF[dt] * np.abs(wx) + TINY[dt]
    assert np.all(np.abs(host(gx) - wx) <= tol)
    n = (g.shape[0] + 66) * U
    assert np.all(np.abs(host(gg) - wg) <= n * (np.abs(gd) * np.abs(xh)).sum(0) + (np.abs(gd) * dx).sum(0))
    assert np.all(np.abs(host(gb) - wb) <= n * np.abs(gd).sum(0))


SHAPES = [(1, 1), (1, 2), (3, 7), (1, 4096), (5, 64), (130, 255), (33, 257), (17, 513), (1000, 1024), (9, 1025),
          (300, 1001), (6, 2049), (40, 4096), (3, 4097), (11, 8191), (2, 16384), (2, 16385), (70, 20011)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward_and_backward(rows, cols, dtype):
    f = fqt()
    x, g, gamma, beta = inputs(rows, cols, dtype, seed=rows * 31 + cols)
    Y, mean, rstd = f.fqt_layernorm_forward(x, gamma, beta, eps=EPS)
    check_forward(x, gamma, beta, Y, mean, rstd)
    gx, gg, gb, _ = f.fqt_layernorm_backward(g, x, mean, rstd, gamma)
    check_backward(g, x, gamma, gx, gg, gb)
    # grad_X alone is the same
    only, none, _, _ = f.fqt_layernorm_backward(g, x, mean, rstd, gamma, params=False)
    assert none is None and torch.equal(only, gx)


def test_no_parameters():
    f = fqt()
    x, g, _, _ = inputs(37, 300, "float32", seed=9)
    Y, mean, rstd = f.fqt_layernorm_forward(x, eps=EPS)
    check_forward(x, None, None, Y, mean, rstd)
    gx, gg, gb, _ = f.fqt_layernorm_backward(g, x, mean, rstd)
    check_backward(g, x, None, gx, gg, gb)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strided_and_unaligned_rows(dtype):
    """Views into wider buffers at odd offsets; what lies outside the view is neither read into the result nor written."""
    f = fqt()
    x, g, gamma, beta = inputs(65, 500, dtype, seed=10)

    def view(t, off, pitch):
        buf = torch.full((65 * pitch + off + 8,), float("nan"), dtype=t.dtype, device="cuda")
        v = buf[off:off + 65 * pitch].view(65, pitch)[:, :500]
        v.copy_(t)
        return v
    xv, gv = view(x, 1, 507), view(g, 3, 501)
    buf = torch.full((65, 511), 7.0, dtype=x.dtype, device="cuda")
    Y, mean, rstd = f.fqt_layernorm_forward(xv, gamma, beta, eps=EPS, Y=buf[:, 5:505])
    check_forward(x, gamma, beta, Y, mean, rstd)
    assert (buf[:, :5] == 7).all() and (buf[:, 505:] == 7).all()
    buf2 = torch.full((65, 513), 7.0, dtype=x.dtype, device="cuda")
    gx, gg, gb, _ = f.fqt_layernorm_backward(gv, xv, mean, rstd, gamma, grad_X=buf2[:, 1:501])
    check_backward(g, x, gamma, gx, gg, gb)
    assert (buf2[:, :1] == 7).all() and (buf2[:, 501:] == 7).all()


def test_gradient_repeated_by_broadcasting():
    """A gradient whose rows are one row (pitch 0), as a sum's is."""
    f = fqt()
    x, g, gamma, beta = inputs(50, 384, "float32", seed=11)
    _, mean, rstd = f.fqt_layernorm_forward(x, gamma, beta, eps=EPS)
    e = g[:1].expand(50, 384)
    gx, gg, gb, _ = f.fqt_layernorm_backward(e, x, mean, rstd, gamma)
    check_backward(e, x, gamma, gx, gg, gb)


def test_constant_rows_and_large_offsets():
    f = fqt()
    x = torch.full((4, 1000), 3.25, device="cuda")
    x[1] = 0.0
    x[2] = -1e30
    x[3] = 1e4 + torch.randn(1000, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    Y, mean, rstd = f.fqt_layernorm_forward(x, eps=EPS)
    assert torch.isfinite(Y).all()
    check_forward(x[:2], None, None, Y[:2], mean[:2], rstd[:2])
    check_forward(x[3:], None, None, Y[3:], mean[3:], rstd[3:])


def test_non_finite_rows_stay_alone():
    f = fqt()
    x, g, gamma, beta = inputs(20, 700, "bfloat16", seed=12)
    bad = x.clone()
    bad[3, 17], bad[8, 0] = float("nan"), float("inf")
    Y0, m0, r0 = f.fqt_layernorm_forward(x, gamma, beta)
    Y1, m1, r1 = f.fqt_layernorm_forward(bad, gamma, beta)
    keep = [i for i in range(20) if i not in (3, 8)]
    assert torch.equal(Y0[keep], Y1[keep]) and torch.isnan(Y1[3]).all() and torch.isnan(Y1[8]).all()
    g0, _, _, _ = f.fqt_layernorm_backward(g, x, m0, r0, gamma)
    g1, _, _, _ = f.fqt_layernorm_backward(g, bad, m1, r1, gamma)
    assert torch.equal(g0[keep], g1[keep])


def test_gradient_against_differences():
    """Central differences of the oracle's forward: second-order error h^2 ~ 1e-8 and float32's."""
    f = fqt()
    x, g, gamma, beta = inputs(3, 40, "float32", seed=13)
    _, mean, rstd = f.fqt_layernorm_forward(x, gamma, beta, eps=EPS)
    gx, gg, gb, _ = f.fqt_layernorm_backward(g, x, mean, rstd, gamma)
    xd, gd, ga, be = host(x), host(g), host(gamma), host(beta)
    h = 1e-4

    def loss(a, b, c):
        return (F.layernorm(a, b, c, EPS)[0] * gd).sum()
    for i, j in ((0, 0), (1, 13), (2, 39)):
        d = np.zeros_like(xd)
        d[i, j] = h
        num = (loss(xd + d, ga, be) - loss(xd - d, ga, be)) / (2 * h)
        assert abs(num - host(gx)[i, j]) < 1e-5 * (1 + abs(num))
    for j in (0, 21, 39):
        d = np.zeros_like(ga)
        d[j] = h
        assert abs((loss(xd, ga + d, be) - loss(xd, ga - d, be)) / (2 * h) - host(gg)[j]) < 1e-5 * 10
        assert abs((loss(xd, ga, be + d) - loss(xd, ga, be - d)) / (2 * h) - host(gb)[j]) < 1e-5 * 10


def test_same_result_twice_and_on_another_stream():
    f = fqt()
    x, g, gamma, beta = inputs(3000, 1000, "float16", seed=14)
    a = f.fqt_layernorm_forward(x, gamma, beta)
    b = f.fqt_layernorm_backward(g, x, a[1], a[2], gamma)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a2 = f.fqt_layernorm_forward(x, gamma, beta)
        b2 = f.fqt_layernorm_backward(g, x, a2[1], a2[2], gamma)
    s.synchronize()
    for p, q in zip(a + b[:3], a2 + b2[:3]):
        assert torch.equal(p, q)


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes and 2^31 elements of input: the last rows against the same rows alone."""
    f = fqt()
    rows, cols = (1 << 21) + 37, 1027
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").normal_()
    Y, mean, rstd = f.fqt_layernorm_forward(x)
    tail = x[-300:].clone()
    Y2, m2, r2 = f.fqt_layernorm_forward(tail)
    assert torch.equal(Y[-300:], Y2) and torch.equal(mean[-300:], m2) and torch.equal(rstd[-300:], r2)
    gx, gg, gb, _ = f.fqt_layernorm_backward(x, x, mean, rstd)
    g2, _, _, _ = f.fqt_layernorm_backward(tail, tail, m2, r2)
    assert torch.equal(gx[-300:], g2)
    n = (rows + 66) * U
    want = sum(x[i:i + (1 << 18)].double().sum(0) for i in range(0, rows, 1 << 18))
    scale = sum(x[i:i + (1 << 18)].double().abs().sum(0) for i in range(0, rows, 1 << 18))
    assert ((gb.double() - want).abs() <= n * scale).all()


def test_refusals():
    f = fqt()
    x, g, gamma, beta = inputs(8, 32, "float32")
    _, mean, rstd = f.fqt_layernorm_forward(x)
    for bad in (lambda: f.fqt_layernorm_forward(x.cpu()), lambda: f.fqt_layernorm_forward(x.double()),
                lambda: f.fqt_layernorm_forward(x.t()), lambda: f.fqt_layernorm_forward(x, gamma[:31]),
                lambda: f.fqt_layernorm_forward(x, gamma.bfloat16()), lambda: f.fqt_layernorm_forward(x[0]),
                lambda: f.fqt_layernorm_forward(x, Y=torch.empty_like(x[:4])),
                lambda: f.fqt_layernorm_backward(g[:4], x, mean, rstd),
                lambda: f.fqt_layernorm_backward(g.half(), x, mean, rstd),
                lambda: f.fqt_layernorm_backward(g, x, mean[:4], rstd)):
        with pytest.raises(ValueError):
            bad()
    for bad, code in ((lambda: f.fqt_layernorm_forward(x[:0]), 1), (lambda: f.fqt_layernorm_forward(x, eps=-1.0), 1),
                      (lambda: f.fqt_layernorm_forward(x, eps=float("nan")), 1),
                      (lambda: f.fqt_layernorm_backward(g, x, mean, rstd, ws=torch.empty(16, dtype=torch.uint8, device="cuda")), 4)):
        with pytest.raises(f.FqtError) as e:
            bad()
        assert e.value.code == code
