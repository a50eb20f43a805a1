"""Products whose large terms cancel: outputs of every type are summed in float32.

Each block of 128 holds pairs of codes whose products are +-2^16 and cancel, beside products of size 1.  Every partial
sum is an integer below 2^24, so float32 sums are exact, and the result is an integer of at most 8 bits, which every
output type holds: the comparison is exact.  Random operands: |error| <= K 2^-24 sum |a b| for float32 accumulation of K
terms in any order, and half a unit in the last place of the output's type."""
import numpy as np
import pytest

from oracle import feedforward as F

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def cancelling(M, N, K):
    """(A, B) of small integers: 256 against +-256 in half of each block's pairs (8 of them), else -1, 0 or 1."""
    gen = torch.Generator("cuda").manual_seed(M + N + K)

    def ones(rows):
        x = torch.randint(-1, 2, (rows, K), device="cuda", generator=gen).float()
        return x * (torch.rand((rows, K), device="cuda", generator=gen) < 0.05)
    a, b = ones(M), ones(N)
    for k in range(0, K - 1, 16):
        a[:, k:k + 2] = 256.0
        b[:, k], b[:, k + 1] = 256.0, -256.0
    return a, b


# few rows from codes; small, middle and large tiles; products in parts along K
SHAPES = [(1, 33, 640), (16, 100, 160), (17, 64, 1000), (40, 257, 512), (64, 64, 4096), (65, 129, 9008), (100, 90, 256),
          (300, 520, 1100), (2048, 2048, 640), (1000, 700, 5000), (3870, 4090, 1100), (8192, 4096, 512), (8185, 1022, 200),
          (8000, 4096, 1000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_large_products_that_cancel(M, N, K, dtype):
    a, b = cancelling(M, N, K)
    A, B = fqt.fqt_fp8_quantize(a)[0], fqt.fqt_fp8_quantize(b)[0]
    assert torch.equal(A["q"][:, :K].float(), a) and torch.equal(B["q"][:, :K].float(), b)  # E = 0: 448 >= 256 > 224
    want = a.double() @ b.double().t().contiguous()
    assert float(want.abs().max()) <= 256.0
    C, _ = fqt.fqt_fp8_gemm(A, B, dtype=dtype)
    assert torch.equal(C.double(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,d_in,d_out", [(1, 1000, 130), (16, 512, 100), (70, 640, 333), (300, 1100, 520)])
def test_a_layer_whose_products_cancel(N, d_in, d_out, dtype):
    """Through the layer's forward and grad_X: rows quantized in registers, and by the quantizer."""
    a, b = cancelling(N, d_out, d_in)
    W8 = fqt.fqt_fp8_quantize(b, tile=True)[0]
    Y, _, _ = fqt.fqt_fp8_linear_forward(a.to(dtype), W8, save=False)
    assert torch.equal(Y.double(), a.double() @ b.double().t().contiguous())
    g, w = cancelling(N, d_in, d_out)  # grad_X = g W with W [d_out, d_in] = w^T
    X8t = fqt.fqt_fp8_quantize(torch.ones((N, d_in), device="cuda"), by_row=False, by_col=True)[1]
    W8t = fqt.fqt_fp8_quantize(w, tile=True)[0]
    _, gX, _ = fqt.fqt_fp8_linear_backward(g.to(dtype), X8t, W8t, stochastic=False)
    assert torch.equal(gX.double(), g.double() @ w.double().t().contiguous())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 300, 1024), (50, 200, 4096), (129, 255, 2570), (600, 1000, 2048)])
def test_random_operands_without_a_term_for_dropped_products(M, N, K, dtype):
    rng = np.random.default_rng(M)

    def draw(rows):
        x = rng.standard_normal((rows, K))
        x[:, ::128] *= 100.0  # one large element a block
        return torch.from_numpy(x.astype(np.float32)).cuda()
    x, w = draw(M), draw(N) * K ** -0.5 / 64
    C, _ = fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], fqt.fqt_fp8_quantize(w)[0], dtype=dtype)
    a, b = F.operand(x.cpu().numpy())["value"], F.operand(w.cpu().numpy())["value"]
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    tol = K * 2.0 ** -24 * size + HALF[dtype] * np.abs(want) + TINY[dtype]
    assert np.all(np.abs(C.double().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_block_scales_far_apart(dtype):
    """Each block of a row has a scale of its own, 2^-30 .. 2^30 in one operand and its inverse in the other, so that
    every block counts: exact integers again."""
    rng = np.random.default_rng(5)
    M, N, kb = 150, 140, 9
    s = np.repeat(2.0 ** rng.integers(-30, 31, kb), 128)
    x, w = rng.integers(-3, 4, (M, kb * 128)), rng.integers(-3, 4, (N, kb * 128))
    x[:, 64:], w[:, 64:] = x[:, 64:] * (rng.random(x[:, 64:].shape) < 0.02), w[:, 64:]
    x[:, :64] *= rng.random((M, 64)) < 0.1
    A = fqt.fqt_fp8_quantize(torch.from_numpy((x * s).astype(np.float32)).cuda())[0]
    B = fqt.fqt_fp8_quantize(torch.from_numpy((w / s).astype(np.float32)).cuda())[0]
    want = (x @ w.T).astype(np.float64)
    assert np.abs(want).max() <= 256
    for rows in (M, 40, 7):
        C, _ = fqt.fqt_fp8_gemm(dict(A, q=A["q"][:rows], exp=A["exp"][:, :rows].contiguous()), B, dtype=dtype)
        np.testing.assert_array_equal(C.double().cpu().numpy(), want[:rows])


def test_codes_and_scales_are_read_exactly():
    """Every finite code under every scale against one element 2^40, 1 or 2^-40: the exact product wherever float32 holds
    it as a normal number; with scales below 2^-124 that of the nearest multiple of 2^-133."""
    codes = np.concatenate([np.arange(127), 128 + np.arange(127)]).astype(np.uint8)
    q = np.zeros((248, 254, 128), np.uint8)
    q[:, :, 5] = codes
    exp = np.full((1, 248 * 254, 4), 127, np.uint8)
    exp[0, :, 0] = np.repeat(np.arange(248), 254)
    E = np.arange(248)[:, None] - 127.0
    value = F.decode(codes)[None] * 2.0 ** E
    value = np.where(E < -124, np.round(value * 2.0 ** 133) * 2.0 ** -133, value).reshape(-1)
    b = torch.zeros((20, 128), device="cuda")
    b[:, 5] = torch.tensor([2.0 ** 40, 1.0, 2.0 ** -40, 0.0] * 5, device="cuda")
    B = fqt.fqt_fp8_quantize(b)[0]
    for r0, r1 in ((0, 248 * 254), (0, 64), (400, 440), (254 * 4 + 90, 254 * 4 + 100), (254 * 247, 254 * 248 - 200)):
        A = dict(q=torch.from_numpy(q.reshape(-1, 128)[r0:r1].copy()).cuda().view(torch.float8_e4m3fn),
                 exp=torch.from_numpy(exp[:, r0:r1].copy()).cuda(), K=128)
        C = fqt.fqt_fp8_gemm(A, B)[0].double().cpu().numpy()
        want = value[r0:r1, None] * b[:, 5].double().cpu().numpy()
        fits = (np.abs(value[r0:r1, None]) < 2.0 ** 128) & (np.abs(want) < 2.0 ** 128) & ((np.abs(want) >= 2.0 ** -126) | (want == 0))
        assert fits.sum() > 0.4 * fits.size
        np.testing.assert_array_equal(C[fits], want[fits])
