"""Workspaces that a caller hands over: anything but contiguous bytes on the current device is refused before a launch."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402

N = 1 << 22
BAD = {
    "host": lambda: torch.empty(N, dtype=torch.uint8),
    "expanded": lambda: torch.empty(1, dtype=torch.uint8, device="cuda").expand(N),
    "every second byte": lambda: torch.empty(2 * N, dtype=torch.uint8, device="cuda")[::2],
    "not bytes": lambda: torch.empty(N, dtype=torch.float32, device="cuda"),
}


def calls():
    """Every entry point that takes a workspace, as f(ws) -> outputs."""
    x = torch.linspace(-1, 1, 80 * 200, device="cuda").view(80, 200)
    w, g = torch.linspace(-1, 1, 60 * 200, device="cuda").view(60, 200), torch.ones((80, 60), device="cuda")
    W8, W8t = fqt.fqt_fp8_quantize(w, tile=True, by_row=True, by_col=True)
    _, X8t, _ = fqt.fqt_fp8_linear_forward(x, W8)
    _, mean, rstd = fqt.fqt_layernorm_forward(x)
    return {
        "layernorm": lambda ws: fqt.fqt_layernorm_backward(x, x, mean, rstd, ws=ws)[:3],
        "layernorm, grad_X only": lambda ws: fqt.fqt_layernorm_backward(x, x, mean, rstd, params=False, ws=ws)[:1],
        "gemm": lambda ws: fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], W8, ws=ws)[:1],
        "forward": lambda ws: fqt.fqt_fp8_linear_forward(x, W8, save=False, ws=ws)[:1],
        "backward": lambda ws: fqt.fqt_fp8_linear_backward(g, X8t, W8t, ws=ws)[:2],
        "clip": lambda ws: (lambda out: (fqt.fqt_grad_norm_clip([x, w], 0.5, outs=out, ws=ws)[0], *out))(
            [torch.empty_like(x), torch.empty_like(w)]),
    }


@pytest.mark.parametrize("kind", list(BAD))
@pytest.mark.parametrize("name", ["layernorm", "layernorm, grad_X only", "gemm", "forward", "backward", "clip"])
def test_refused(name, kind):
    with pytest.raises(ValueError):
        calls()[name](BAD[kind]())


@pytest.mark.parametrize("name", ["layernorm", "layernorm, grad_X only", "gemm", "forward", "backward", "clip"])
def test_a_caller_s_bytes_give_the_same_results(name):
    f = calls()[name]
    for a, b in zip(f(None), f(torch.empty(N, dtype=torch.uint8, device="cuda"))):
        assert torch.equal(a, b)
