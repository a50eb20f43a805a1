"""The gated feed-forward block: norm, gated layer and down projection with their checkpoints, used together: against
autograd of the same block without quantization, while serving, as a command, on another stream and in a graph."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ACTS = {"silu": torch.nn.functional.silu, "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh"),
        "relu": torch.relu}


def block(D=192, H=520, dtype=torch.float32, seed=0, act="silu"):
    from paper_2010_14298_amd import ffn
    return ffn.GatedFeedForward(D, H, dtype=dtype, seed=seed, act=act)


def tokens(N, D, seed, dtype=torch.float32):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn((N, D), generator=gen, device="cuda").to(dtype)


def plain(b, X, dY):
    """Output and gradients of the block without quantization, by autograd in float32."""
    params = [p.clone().requires_grad_() for p in b.parameters()]
    x = X.float().requires_grad_()
    n = torch.nn.functional.layer_norm(x, (X.shape[1],), params[2], params[3])
    both = n @ params[0].t()
    h = both.shape[1] // 2
    y = x + (ACTS[b.act](both[:, :h]) * both[:, h:]) @ params[1].t()
    y.backward(dY.float())
    return y.detach(), [p.grad for p in params + [x]]


def cosine(p, q):
    return float((p.double() * q.double()).sum() / (p.double().norm() * q.double().norm()))


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gradients_follow_autograd(dtype, act):
    """Relative noise of 3 mantissa bits: 2.6 % nearest, 3.7 % stochastic.  grad_W1 has that of X, the checkpoint (2.6
    each) and D (3.7), of dH (4.5: its two operands), and of a and b, whose operands' noise (3.7 each) moves both
    derivatives: 9 % together, a cosine of 0.996; 0.98 leaves 20 %.  A ReLU's gate switches where a is within its noise
    of zero, for 1 % of the units, which then are wrong altogether: 10 % more."""
    b = block(dtype=dtype, act=act)
    X, dY = tokens(300, 192, 1, dtype), tokens(300, 192, 2, dtype)
    Y, kept = b.forward(X)
    grads, dX = b.backward(dY, kept, seed=5)
    y, want = plain(b, X, dY)
    assert cosine(Y, y) > 0.99
    for got, g in zip(grads + [dX], want):
        assert got.shape == g.shape and cosine(got, g) > 0.98


def test_gradients_are_unbiased_over_seeds():
    """The mean of 200 backward passes from one forward pass against the products of the same checkpoints and operands
    without stochastic rounding: each draw is off by about 3.7 % of a gradient's norm, the mean by 0.26 %."""
    from oracle import gated as G
    from paper_2010_14298_amd import fqt
    b = block(64, 96)
    X, dH = tokens(128, 64, 1), tokens(128, 96, 2)
    _, kept, _ = fqt.fqt_fp8_gated_forward(X, b.W1_8)
    d = [torch.from_numpy(G.kept_values(kept[n]["q"].view(torch.uint8).cpu().numpy(), kept[n]["exp"].cpu().numpy(), 96))
         for n in ("d_gate", "d_up")]
    D = torch.cat([dH.double().cpu() * d[0], dH.double().cpu() * d[1]], dim=1)
    codes = [kept["X8t"], b.W1_8t]
    x, w = (o["q"].float().cpu().double() * torch.exp2(o["exp"].transpose(0, 1).reshape(o["q"].shape[0], -1)[
        :, :o["q"].shape[1] // 128].double().cpu() - 127).repeat_interleave(128, 1) for o in codes)
    want = [D.t() @ x[:, :128].t(), D @ w[:, :192].t()]
    total = [0.0, 0.0]
    for s in range(200):
        gW, gX, _ = fqt.fqt_fp8_gated_backward(dH, kept, b.W1_8t, seed=s)
        total = [t + g.double().cpu() for t, g in zip(total, (gW, gX))]
    for t, g in zip(total, want):
        assert float((t / 200 - g).norm() / g.norm()) < 0.006


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_serving_one_token_matches_the_batch(dtype):
    """A row's codes do not depend on the other rows; its sums run in another order, which may move a hidden unit's code
    in the down projection by one step (6 % of one of 520 terms)."""
    b = block(dtype=dtype)
    X = tokens(300, 192, 3, dtype)
    Y = b.forward(X, keep=False)[0]
    assert torch.equal(Y, b.forward(X)[0]) or dtype != torch.float32 or cosine(Y, b.forward(X)[0]) > 0.99999
    for i in (0, 17, 299):
        one = b.forward(X[i:i + 1], keep=False)[0]
        tol = 1e-2 if dtype == torch.float32 else 2.0 ** -6
        assert float((one - Y[i:i + 1]).abs().max()) <= tol * float(Y.abs().max())


@pytest.mark.parametrize("gate", list(ACTS))
def test_the_command_runs(gate):
    from paper_2010_14298_amd import ffn
    losses = ffn.main(["--tokens", "256", "--width", "128", "--hidden", "200", "--steps", "3", "--gate", gate])
    assert len(losses) == 3 and all(v == v and v < float("inf") for v in losses)


def outputs(b, X, dY):
    Y, kept = b.forward(X)
    grads, dX = b.backward(dY, kept, seed=5)
    return [Y, kept[0]["q"].view(torch.uint8), kept[2]["d_gate"]["q"].view(torch.uint8), *grads, dX,
            b.forward(X[:5], keep=False)[0]]


@pytest.mark.parametrize("N,D,H,dtype", [(40, 100, 70, torch.float32), (300, 192, 520, torch.bfloat16),
                                         (1500, 256, 640, torch.float16)])
def test_replays_of_a_graph(N, D, H, dtype):
    """Forward, backward and a serving pass recorded: every replay on new inputs equals the eager pass, bit for bit."""
    b = block(D, H, dtype)
    X, dY = torch.zeros((N, D), dtype=dtype, device="cuda"), torch.zeros((N, D), dtype=dtype, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outputs(b, X, dY)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        recorded = outputs(b, X, dY)
    for turn in range(4):
        X.copy_(tokens(N, D, 10 + turn) * 2.0 ** turn)
        dY.copy_(tokens(N, D, 20 + turn))
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in recorded]
        torch.randn(1 << 16, device="cuda").sum().item()  # work between replays
        for i, (p, q) in enumerate(zip(kept, outputs(b, X, dY))):
            assert torch.equal(p, q), (turn, i)


def test_two_streams_at_once():
    """Two passes at a time on streams of their own give what they give one after the other."""
    b = block(192, 520, torch.bfloat16)
    data = [(tokens(700, 192, s, torch.bfloat16), tokens(700, 192, s + 50, torch.bfloat16)) for s in range(2)]
    want = [outputs(b, *d) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in data]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = outputs(b, *data[i])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(w, g))
