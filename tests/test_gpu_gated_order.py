"""A row of the gated forward has the same bits wherever it stands in its batch and whatever stands beside it, in every
form of the layer."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402
from tests import test_gpu_gated as base  # noqa: E402
from tests.test_gpu_gated_forms import CASES, form_of  # noqa: E402

LIST = [(form, *cases[0]) for form, cases in CASES.items()] + [("rows", 60, 1100, 130, torch.bfloat16, "silu"),
                                                               ("rows", 16, 3000, 70, torch.float32, "gelu_tanh")]


@pytest.mark.parametrize("form,N,d_in,hidden,dtype,act", LIST)
def test_rows_in_another_order(form, N, d_in, hidden, dtype, act):
    save = form != "rows"
    X = base.matrix(N, N, d_in, dtype)
    _, W8, _ = base.weights(hidden, hidden, d_in)
    H, kept, ws = fqt.fqt_fp8_gated_forward(X, W8, act=act, save=save)
    assert form_of(N, d_in, hidden) == form if save else ws is None
    order = torch.randperm(N, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    moved, again, _ = fqt.fqt_fp8_gated_forward(X[order], W8, act=act, save=save)
    assert torch.equal(moved, H[order])
    others = torch.randn((N, d_in), generator=torch.Generator("cuda").manual_seed(2), device="cuda").to(dtype)
    others[::7] = X[::7]
    assert torch.equal(fqt.fqt_fp8_gated_forward(others, W8, act=act, save=save)[0][::7], H[::7])
    for name in ("d_gate", "d_up") if save else ():
        assert torch.equal(again[name]["q"].view(torch.uint8), kept[name]["q"].view(torch.uint8)[order])
        assert torch.equal(again[name]["exp"], kept[name]["exp"][order])
