"""Layer norm's gradient on rows of no variance and of large means.

Tolerances as in the other tests of the gradient: with u = 2^-24 and trees of at most 64 additions, 66 u rstd (|c| +
mean|c| + |xh| mean|c xh|) of grad_X and (rows + 66) u of the parameters' sums of magnitudes, and half a unit in the last
place of the output's type."""
import numpy as np
import pytest

from tests.test_gpu_layernorm import EPS, HALF, TINY, U, check_backward, host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402


def formula(g, x, mean, rstd, gamma):
    """The gradient with the given statistics, float64, and the tolerances of its three parts."""
    g, x, gamma = host(g), host(x), host(gamma)
    m, r = host(mean)[:, None], host(rstd)[:, None]
    xh, c = (x - m) * r, g * gamma
    gx = r * (c - c.mean(1, keepdims=True) - xh * (c * xh).mean(1, keepdims=True))
    a = np.abs
    tol = 66 * U * r * (a(c) + a(c).mean(1, keepdims=True) + a(xh) * a(c * xh).mean(1, keepdims=True))
    n = (g.shape[0] + 66) * U
    return (gx, tol), ((g * xh).sum(0), n * a(g * xh).sum(0)), (g.sum(0), n * a(g).sum(0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 5, 17])
@pytest.mark.parametrize("cols", [1, 3, 100, 128, 300, 1001, 1100, 2100, 5000, 9000, 20011])
def test_lanes_without_a_column_and_teams_without_a_row_add_nothing(rows, cols, dtype):
    """The first row is 2^120 throughout: its own (x - mean) rstd is 0, while (0 - mean) rstd passes float32's range."""
    gen = torch.Generator("cuda").manual_seed(rows + cols)
    x = torch.randn((rows, cols), device="cuda", generator=gen)
    g = torch.randn((rows, cols), device="cuda", generator=gen).to(dtype)
    gamma = 1.0 + 0.3 * torch.randn(cols, device="cuda", generator=gen)
    x[0] = 2.0 ** 120
    x = x.to(dtype)
    mean, rstd = x.double().mean(1).float(), torch.full((rows,), 0.75, device="cuda")
    mean[0], rstd[0] = 2.0 ** 120, 1024.0
    gx, gg, gb, _ = fqt.fqt_layernorm_backward(g, x, mean, rstd, gamma)
    name = str(dtype).split(".")[1]
    (wx, tx), (wg, tg), (wb, tb) = formula(g, x, mean, rstd, gamma)
    assert np.all(np.abs(host(gx) - wx) <= tx + HALF[name] * np.abs(wx) + TINY[name])
    assert np.all(np.abs(host(gg) - wg) <= tg) and np.all(np.abs(host(gb) - wb) <= tb)
    only, _, _, _ = fqt.fqt_layernorm_backward(g, x, mean, rstd, gamma, params=False)
    assert torch.equal(only, gx)


def test_constant_row_that_the_forward_normalizes():
    """128 columns of 2^120: the mean is exact, the variance 0, rstd = eps^-1/2."""
    x = torch.full((3, 128), 2.0 ** 120, device="cuda")
    x[1] = -(2.0 ** 120)
    x[2] = torch.linspace(-1, 1, 128, device="cuda")
    g = torch.randn((3, 128), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    gamma = torch.ones(128, device="cuda")
    Y, mean, rstd = fqt.fqt_layernorm_forward(x, gamma, eps=EPS)
    assert (Y[:2] == 0).all()
    gx, gg, gb, _ = fqt.fqt_layernorm_backward(g, x, mean, rstd, gamma)
    for got, (want, tol) in zip((gx, gg, gb), formula(g, x, mean, rstd, gamma)):
        assert np.all(np.abs(host(got) - want) <= tol + HALF["float32"] * np.abs(want))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("cols", [200, 1000, 3000, 17000])
def test_rows_of_no_variance_and_of_large_means(cols, dtype):
    dt = getattr(torch, dtype)
    gen = torch.Generator("cuda").manual_seed(cols)
    x = torch.randn((7, cols), device="cuda", generator=gen)
    x[0], x[1], x[2] = 3.25, 0.0, -500.0
    x[3] = 1e4 + x[3] * (1.0 if dtype == "float32" else 300.0)
    x[4] = -300.0 + 0.01 * x[4]
    x[5, 1:] = 0.0
    x = x.to(dt)
    g = torch.randn((7, cols), device="cuda", generator=gen).to(dt)
    gamma, beta = 1.0 + 0.3 * torch.randn(cols, device="cuda", generator=gen), torch.zeros(cols, device="cuda")
    _, mean, rstd = fqt.fqt_layernorm_forward(x, gamma, beta, eps=EPS)
    gx, gg, gb, _ = fqt.fqt_layernorm_backward(g, x, mean, rstd, gamma)
    assert all(torch.isfinite(t).all() for t in (gx, gg, gb))
    check_backward(g, x, gamma, gx, gg, gb)
