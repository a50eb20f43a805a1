"""The gated block keeps nothing while it serves: the same output, bit for bit, wherever both ways take the same tiles."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import ffn, fqt  # noqa: E402


@pytest.mark.parametrize("act", sorted(fqt.ACTS))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,D,H", [(300, 192, 520), (129, 100, 70), (1500, 256, 640)])
def test_a_batch_without_checkpoints_has_the_batchs_bits(N, D, H, dtype, act):
    """More than 128 rows: the layer's form does not depend on what is kept, and the norms give the same rows."""
    b = ffn.GatedFeedForward(D, H, dtype=dtype, seed=4, act=act)
    X = torch.randn((N, D), generator=torch.Generator("cuda").manual_seed(5), device="cuda").to(dtype)
    kept, none = b.forward(X), b.forward(X, keep=False)
    assert none[1] is None and torch.isfinite(none[0]).all()
    assert torch.equal(kept[0], none[0])
