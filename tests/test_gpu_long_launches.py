"""Calls of 2^32 and more threads, which one dimension of a grid does not hold: against calls on parts, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402


@pytest.mark.parametrize("rows", [1 << 26, (1 << 26) + 4099])
def test_layer_norm_of_many_short_rows(rows):
    """Four rows a block of 256 threads."""
    x = torch.empty((rows, 3), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    Y = torch.full_like(x, 9.0)
    _, mean, rstd = fqt.fqt_layernorm_forward(x, Y=Y)
    for a, b in ((0, 5000), ((1 << 25) + 1, (1 << 25) + 7000), (rows - 9001, rows)):
        y, m, r = fqt.fqt_layernorm_forward(x[a:b])
        assert torch.equal(Y[a:b], y) and torch.equal(mean[a:b], m) and torch.equal(rstd[a:b], r)


def test_parameter_gradients_of_a_very_long_row():
    """2^27 columns and more: 64 of the two sums' columns a block of 1024 threads."""
    cols = (1 << 27) + 70
    gen = torch.Generator("cuda").manual_seed(2)
    x = torch.empty((2, cols), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    g = torch.empty((2, cols), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    mean, rstd = torch.tensor([0.25, -0.5], device="cuda"), torch.tensor([1.5, 0.75], device="cuda")
    _, gg, gb, _ = fqt.fqt_layernorm_backward(g, x, mean, rstd)
    for a, b in ((0, 20000), (cols // 2 - 9000, cols // 2 + 9000), (cols - 20000, cols)):
        gd, xh = g[:, a:b].double(), (x[:, a:b].double() - mean.double()[:, None]) * rstd.double()[:, None]
        assert ((gg[a:b].double() - (gd * xh).sum(0)).abs() <= 2.0 ** -21 * (gd * xh).abs().sum(0)).all()
        assert ((gb[a:b].double() - gd.sum(0)).abs() <= 2.0 ** -21 * gd.abs().sum(0)).all()


def test_product_of_few_rows_and_very_many_outputs():
    """2^27 outputs a row and more: 16 a block of 512 threads."""
    N, K = (1 << 27) + 40, 100
    gen = torch.Generator("cuda").manual_seed(3)
    q = torch.empty((N, 128), dtype=torch.uint8, device="cuda").random_(0, 120, generator=gen)
    q[:, K:] = 0
    W = dict(q=q.view(torch.float8_e4m3fn), exp=torch.full((1, N, 4), 127, dtype=torch.uint8, device="cuda"), K=K)
    x = torch.randn((3, K), device="cuda", generator=gen).bfloat16()
    C, _ = fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], W, dtype=torch.bfloat16)
    Y, _, _ = fqt.fqt_fp8_linear_forward(x, W, save=False)
    assert torch.equal(C, Y)
    for a, b in ((0, 3000), (N // 2 - 7, N // 2 + 3000), (N - 3001, N)):
        part = dict(q=W["q"][a:b], exp=W["exp"][:, a:b].contiguous(), K=K)
        assert torch.equal(C[:, a:b], fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], part, dtype=torch.bfloat16)[0])


def test_codes_of_a_very_long_column():
    """2^31 - 50 rows: 2^24 tiles of 256 threads."""
    rows = (1 << 31) - 50
    x = torch.empty((rows, 1), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(4))
    _, a = fqt.fqt_fp8_quantize(x, by_row=False, by_col=True)
    for first in (0, 1 << 30, (rows >> 9 << 9) - 5120):
        n = min(7000, rows - first)
        _, b = fqt.fqt_fp8_quantize(x[first:first + n], by_row=False, by_col=True)
        whole = n // 128 * 128 if first + n < rows else b["q"].shape[1]
        assert torch.equal(a["q"][:, first:first + whole].view(torch.uint8), b["q"][:, :whole].view(torch.uint8))
        blocks = whole // 128 // 4
        assert torch.equal(a["exp"][first // 512:first // 512 + blocks], b["exp"][:blocks])
