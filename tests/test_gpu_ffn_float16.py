"""The feed-forward block's training step with float16 activations: the loss's gradient is diff / (tokens x width), mostly
below float16's smallest step (6e-8) for a batch of any size, and has to reach the parameters all the same."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import ffn, fqt  # noqa: E402


def tokens(N, D, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn((N, D), generator=gen, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [0.3, 0.003])
def test_the_step_follows_autograd(dtype, size, monkeypatch):
    """Gradients of one step against autograd of the block without quantization, with the same units on.  Noise of 3
    mantissa bits: at most 6.4 % of a gradient (a cosine of 0.998, a norm 0.2 % too large); the cosine's bound of 0.99 and
    the norm's of 5 % leave room for the types' roundings."""
    N, D, H = 8192, 1024, 256
    b = ffn.FeedForward(D, H, dtype=dtype, seed=0)
    X = tokens(N, D, 1).to(dtype)
    Y, kept = b.forward(X)
    target = (Y.float() - size * tokens(N, D, 2))
    params = [p.clone().requires_grad_() for p in b.parameters()]
    before = [p.clone() for p in b.parameters()]
    n = torch.nn.functional.layer_norm(X.float(), (D,), params[2], params[3])
    y = X.float() + ((n @ params[0].t()) * (kept[4] > 0)) @ params[1].t()
    diff = Y.float() - target
    y.backward(diff / diff.numel())
    want = torch.stack([p.grad.double().square().sum() for p in params]).sum().sqrt()
    clip, bounds = fqt.fqt_grad_norm_clip, []

    def record(grads, max_norm, *a, **k):
        bounds.append(max_norm)
        return clip(grads, max_norm, *a, **k)
    monkeypatch.setattr(fqt, "fqt_grad_norm_clip", record)
    lr = 1e3
    loss, norm = b.step(X, target, lr, max_norm=float(want) / 4, seed=7)
    assert len(bounds) == 1
    assert abs(float(loss) - 0.5 * size ** 2) < 0.02 * size ** 2
    assert abs(float(norm) / float(want) - 1) < 0.05
    moved = [(p0.double() - p.double()) / lr for p0, p in zip(before, b.parameters())]
    total = torch.stack([m.square().sum() for m in moved]).sum().sqrt()
    assert abs(float(total) / (float(want) / 4) - 1) < 0.01  # clipped to the bound, in float32
    for m, p in zip(moved[:2], params[:2]):
        g = p.grad.double()
        assert float((m * g).sum() / (m.norm() * g.norm())) > 0.99


def test_training_in_float16_lowers_the_loss():
    teacher, block = (ffn.FeedForward(128, 384, dtype=torch.float16, seed=s) for s in (1, 2))
    losses = []
    for i in range(60):
        X = tokens(512, 128, 100 + i).half()
        losses.append(block.step(X, teacher.forward(X, keep=False)[0], 2.0, 1.0, seed=i)[0])
    losses = [float(v) for v in losses]
    assert sum(losses[-10:]) < 0.7 * sum(losses[:10])
