"""The floating-point operators recorded in a HIP graph: every replay on new inputs equals the eager calls, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2010_14298_amd import fqt  # noqa: E402

DEV = "cuda"


def replays(make, inputs, times=4):
    """make() -> list of outputs, reading the tensors `inputs` in place."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        make()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        recorded = make()
    gen = torch.Generator(device=DEV).manual_seed(3)
    for turn in range(times):
        for t in inputs:
            t.copy_(torch.randn(t.shape, generator=gen, device=DEV) * 2.0 ** turn)
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in recorded]
        torch.randn(1 << 16, device=DEV).sum().item()  # work between replays
        expected = make()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(kept, expected)):
            assert torch.equal(a, b), (turn, i)


@pytest.mark.parametrize("rows,cols,dtype", [(1, 1024, torch.bfloat16), (300, 1001, torch.float32),
                                             (5, 20000, torch.float16)])
def test_layer_norm(rows, cols, dtype):
    X, G = (torch.zeros((rows, cols), dtype=dtype, device=DEV) for _ in range(2))
    gamma, beta = (torch.zeros(cols, device=DEV) for _ in range(2))

    def make():
        Y, mean, rstd = fqt.fqt_layernorm_forward(X, gamma, beta)
        gX, gg, gb, _ = fqt.fqt_layernorm_backward(G, X, mean, rstd, gamma)
        return [Y, mean, rstd, gX, gg, gb]

    replays(make, [X, G, gamma, beta])


# one token; few rows; a product in parts along K; whole tiles of each size
@pytest.mark.parametrize("rows,d_in,d_out,dtype", [(1, 256, 512, torch.bfloat16), (40, 384, 130, torch.float16),
                                                   (130, 4096, 260, torch.float32), (1024, 512, 1024, torch.bfloat16)])
def test_fp8_layer(rows, d_in, d_out, dtype):
    X = torch.zeros((rows, d_in), dtype=dtype, device=DEV)
    G = torch.zeros((rows, d_out), dtype=dtype, device=DEV)
    W = torch.zeros((d_out, d_in), device=DEV)

    def make():
        W8, W8t = fqt.fqt_fp8_quantize(W, tile=True, by_row=True, by_col=True)
        Y, X8t, _ = fqt.fqt_fp8_linear_forward(X, W8, relu=True)
        gW, gX, _ = fqt.fqt_fp8_linear_backward(G, X8t, W8t, seed=11)
        return [W8["exp"], Y, gW, gX]

    replays(make, [X, G, W])


def test_gradient_clipping():
    grads = [torch.zeros(n, device=DEV) for n in [1, 31, 4097, 100000] + [7] * 170]

    def make():
        outs = [torch.empty_like(g) for g in grads]
        norm, _ = fqt.fqt_grad_norm_clip(grads, 3.0, outs)
        return [norm] + outs

    replays(make, grads)
