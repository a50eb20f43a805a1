"""8-bit floating point layers: the block quantizer bit for bit against the oracle, the products against float64.

Products: with s = sum |a b| of an output, float32 accumulation of K terms in any order is off by at most K 2^-24 s.
The 8-bit matrix instructions, which 16-bit outputs take, drop what lies more than 13 bits below the largest product of a
group: 2^-12 s covers a group that loses its half.  The output's type adds half a unit in its last place (and float16's
smallest step)."""
import numpy as np
import pytest

from oracle import feedforward as F

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def fqt():
    from paper_2010_14298_amd import fqt as f
    f.load()
    return f


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def heavy(seed, rows, cols, dtype=torch.float32, spread=2.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.normal(0, spread, (rows, 1)))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    return torch.from_numpy(x).to(dtype).cuda()


def same_operand(got, want, why=""):
    np.testing.assert_array_equal(got["exp"].cpu().numpy(), want["exp"], err_msg=f"exp {why}")
    np.testing.assert_array_equal(got["q"].view(torch.uint8).cpu().numpy(), want["q"], err_msg=f"codes {why}")


def check_product(C, A, B, relu=False, mask=None):
    a, b = A["value"], B["value"]
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    drop = 2.0 ** -12 if C.dtype != torch.float32 else 0.0
    tol = (a.shape[1] * 2.0 ** -24 + drop) * size + HALF[C.dtype] * np.abs(want) + TINY[C.dtype]
    if relu:
        want = np.maximum(want, 0.0)
    if mask is not None:
        want = np.where(mask > 0, want, 0.0)
    assert np.all(np.abs(host(C) - want) <= tol)


# ---------------------------------------------------------------------------
# quantizer
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 129), (3, 5), (127, 128), (128, 256), (129, 300), (200, 1030),
                                       (700, 131)])
def test_codes_bit_for_bit(rows, cols, dtype, tile, stochastic):
    f = fqt()
    x = heavy(rows * 7 + cols, rows, cols, dtype)
    a, b = f.fqt_fp8_quantize(x, tile=tile, by_row=True, by_col=True, stochastic=stochastic, seed=(7 << 32) + 5)
    xd = host(x)
    u = [F.uniforms(rows, cols, (7 << 32) + 5, s) for s in (0, 1)] if stochastic else [None, None]
    same_operand(a, F.operand(xd, tile, u[1]), "by row")
    same_operand(b, F.operand(xd.T, tile, u[0].T if stochastic else None), "by column")
    # each operand alone is the same
    one, none = f.fqt_fp8_quantize(x, tile=tile, stochastic=stochastic, seed=(7 << 32) + 5)
    two = f.fqt_fp8_quantize(x, tile=tile, by_row=False, by_col=True, stochastic=stochastic, seed=(7 << 32) + 5)[1]
    assert none is None
    for p, q in ((one, a), (two, b)):
        assert torch.equal(p["q"].view(torch.uint8), q["q"].view(torch.uint8)) and torch.equal(p["exp"], q["exp"])


def test_codes_at_the_edges_of_the_ranges():
    """Empty blocks, block maxima at, just under and just over 448 2^k, rounding ties, float32's subnormals and
    largest values, negative zeros."""
    f = fqt()
    x = np.zeros((64, 128), np.float32)
    x[1, 3], x[2, 3], x[3, 3] = 448.0, np.nextafter(np.float32(448), np.float32(0)), np.nextafter(np.float32(448), np.float32(1e9))
    x[4, 3], x[5, 3], x[6, 3], x[7, 3] = 1e-45, 1.17e-38, 3.4e38, 448.0 * 2.0 ** -127
    m = F.magnitudes()
    x[8, :126], x[8, 127] = (m[1:] + m[:-1]) / 2, 448.0
    x[9, :126], x[9, 127] = -m[:126], -448.0
    x[10] = -0.0
    x[11, :5] = [448.0, 2.0 ** -10, 2.0 ** -11, 3 * 2.0 ** -11, -(2.0 ** -10)]
    for k in range(12, 64):
        x[k] = np.random.default_rng(k).uniform(-1, 1, 128) * 2.0 ** (k * 4 - 140)
    t = torch.from_numpy(x).cuda()
    for sr in (False, True):
        a, b = f.fqt_fp8_quantize(t, by_row=True, by_col=True, stochastic=sr, seed=3)
        xd = x.astype(np.float64)
        u = [F.uniforms(64, 128, 3, s) if sr else None for s in (0, 1)]
        same_operand(a, F.operand(xd, u=u[1]))
        same_operand(b, F.operand(xd.T, u=u[0].T if sr else None))


@pytest.mark.parametrize("tile", [False, True])
def test_non_finite_blocks(tile):
    f = fqt()
    x = heavy(21, 300, 400)
    x[5, 17], x[140, 399], x[299, 130] = float("nan"), float("inf"), float("-inf")
    a, b = f.fqt_fp8_quantize(x, tile=tile, by_row=True, by_col=True)
    same_operand(a, F.operand(host(x), tile))
    same_operand(b, F.operand(host(x).T, tile))


def test_strided_input():
    f = fqt()
    x = heavy(22, 150, 260, torch.bfloat16)
    buf = torch.full((150, 271), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, 3:263] = x
    a, b = f.fqt_fp8_quantize(buf[:, 3:263], by_row=True, by_col=True, stochastic=True, seed=4)
    c, d = f.fqt_fp8_quantize(x, by_row=True, by_col=True, stochastic=True, seed=4)
    for p, q in ((a, c), (b, d)):
        assert torch.equal(p["q"].view(torch.uint8), q["q"].view(torch.uint8)) and torch.equal(p["exp"], q["exp"])
    e, _ = f.fqt_fp8_quantize(x[:1].expand(40, 260))
    same_operand(e, F.operand(np.repeat(host(x[:1]), 40, 0)))


def test_stochastic_codes_are_unbiased_over_seeds():
    """The mean of 400 draws of 64 x 128 elements: each element's error has standard deviation at most half a step,
    so the mean square of the errors in units of step / (2 sqrt(400)) is at most 1; five deviations above it is 1.08."""
    f = fqt()
    x = heavy(23, 64, 128)
    n, total = 400, 0.0
    for s in range(n):
        a, _ = f.fqt_fp8_quantize(x, stochastic=True, seed=s)
        total = total + a["q"].double()
    E = a["exp"][0, :, 0].double()[:, None] - 127
    y = x.double() * torch.exp2(-E)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    z = (total / n - y) / (step / 2 / n ** 0.5)
    assert float(z.square().mean()) < 1.08


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
SHAPES = [(1, 1, 1), (1, 17, 300), (2, 130, 128), (5, 64, 64), (16, 100, 129), (17, 33, 1000), (33, 257, 640),
          (64, 64, 4096), (100, 1001, 2048), (128, 128, 128), (129, 255, 257), (250, 300, 513), (300, 520, 4100),
          (513, 1030, 384), (1, 4096, 1024), (7, 300, 16389), (40, 40, 20000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K, dtype):
    f = fqt()
    spread = 0.3 if dtype == torch.float16 else 2.0
    x, w = heavy(M + N, M, K, spread=spread), heavy(M + N + 1, N, K, spread=spread)
    A, B = f.fqt_fp8_quantize(x)[0], f.fqt_fp8_quantize(w, tile=True)[0]
    a, b = F.operand(host(x)), F.operand(host(w), tile=True)
    C, _ = f.fqt_fp8_gemm(A, B, dtype=dtype)
    check_product(C, a, b)
    mask = torch.randn((M, N), device="cuda", generator=torch.Generator("cuda").manual_seed(M)).to(dtype)
    R, _ = f.fqt_fp8_gemm(A, B, dtype=dtype, relu=True, mask=mask)
    check_product(R, a, b, relu=True, mask=host(mask))


@pytest.mark.parametrize("M,N,K", [(1, 50, 256), (20, 70, 300), (300, 270, 1500)])
def test_product_with_block_scales_far_apart(M, N, K):
    """Every block of a row has a scale of its own, 2^-40 .. 2^40: a wrong scale for one block would show."""
    f = fqt()
    rng = np.random.default_rng(M)
    kb = -(-K // 128)

    def far(rows):
        s = np.repeat(2.0 ** rng.integers(-40, 41, (rows, kb)), 128, axis=1)[:, :K]
        return torch.from_numpy((rng.standard_normal((rows, K)) * s).astype(np.float32)).cuda()
    x, w = far(M), far(N)
    C, _ = f.fqt_fp8_gemm(f.fqt_fp8_quantize(x)[0], f.fqt_fp8_quantize(w)[0])
    check_product(C, F.operand(host(x)), F.operand(host(w)))


def test_product_is_exact_on_small_integers():
    """Integers up to 8 with K 15 bits of sum: every partial sum is exact, so the result is."""
    f = fqt()
    for M, N, K in ((3, 40, 500), (200, 300, 1200), (600, 600, 4096)):
        rng = np.random.default_rng(K)
        x, w = rng.integers(-8, 9, (M, K)), rng.integers(-8, 9, (N, K))
        A = f.fqt_fp8_quantize(torch.from_numpy(x.astype(np.float32)).cuda())[0]
        B = f.fqt_fp8_quantize(torch.from_numpy(w.astype(np.float32)).cuda())[0]
        np.testing.assert_array_equal(host(f.fqt_fp8_gemm(A, B)[0]), (x @ w.T).astype(np.float64))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(8185, 1022, 200), (8200, 1000, 1500), (3900, 4000, 130), (3870, 4090, 1100),
                                   (2048, 2048, 640), (1000, 700, 5000), (65, 129, 9000), (4000, 64, 2000)])
def test_product_of_every_tile(M, N, K, dtype):
    """Sizes that take the middle and large tiles, many stages, and products split along K: float64 on the device
    from the decoded operands; a ReLU and a mask; outputs off whole lines of memory and on them."""
    f = fqt()
    A = f.fqt_fp8_quantize(heavy(M, M, K, spread=1.0))[0]
    B = f.fqt_fp8_quantize(heavy(N + 1, N, K, spread=0.2), tile=True)[0]

    def value(a):
        e = a["exp"].transpose(0, 1).reshape(a["q"].shape[0], -1)[:, :a["q"].shape[1] // 128].double() - 127
        return (a["q"].double().view(a["q"].shape[0], -1, 128) * torch.exp2(e)[:, :, None]).flatten(1)
    a, b = value(A), value(B)
    want, size = a @ b.t().contiguous(), a.abs() @ b.abs().t().contiguous()
    drop = 2.0 ** -12 if dtype != torch.float32 else 0.0
    tol = (K * 2.0 ** -24 + drop) * size + HALF[dtype] * want.abs()
    C, _ = f.fqt_fp8_gemm(A, B, dtype=dtype)
    assert ((C.double() - want).abs() <= tol).all()
    wide = torch.empty((M, (N + 127) // 128 * 128), dtype=dtype, device="cuda")
    mask = torch.randn((M, N), device="cuda").to(dtype)
    R, _ = f.fqt_fp8_gemm(A, B, C=wide[:, :N], relu=True, mask=mask)
    assert torch.equal(R, torch.where(mask > 0, C.clamp(min=0), torch.zeros((), dtype=dtype, device="cuda")))


def test_nan_blocks_reach_their_outputs_only():
    f = fqt()
    for M, N, K in ((4, 40, 700), (150, 140, 700)):
        x, w = heavy(30, M, K), heavy(31, N, K)
        A, B = f.fqt_fp8_quantize(x)[0], f.fqt_fp8_quantize(w)[0]
        C0, _ = f.fqt_fp8_gemm(A, B)
        x[2, 300] = float("nan")
        w[7, 5] = float("inf")
        C1, _ = f.fqt_fp8_gemm(f.fqt_fp8_quantize(x)[0], f.fqt_fp8_quantize(w)[0])
        bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
        bad[2], bad[:, 7] = True, True
        assert torch.isnan(C1[bad]).all() and torch.equal(C1[~bad], C0[~bad])


def test_strided_output_keeps_its_surroundings():
    f = fqt()
    for M, N, K, dt in ((150, 200, 300, torch.bfloat16), (9, 61, 300, torch.float32)):
        x, w = heavy(32, M, K, spread=0.5), heavy(33, N, K, spread=0.5)
        A, B = f.fqt_fp8_quantize(x)[0], f.fqt_fp8_quantize(w)[0]
        buf = torch.full((M + 2, N + 9), 5.0, dtype=dt, device="cuda")
        C, _ = f.fqt_fp8_gemm(A, B, C=buf[1:M + 1, 3:N + 3])
        assert torch.equal(C, f.fqt_fp8_gemm(A, B, dtype=dt)[0])
        C.fill_(5.0)
        assert (buf == 5).all()


# ---------------------------------------------------------------------------
# the layer
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,d_in,d_out", [(1, 64, 64), (1, 1000, 130), (3, 257, 300), (16, 512, 100), (70, 200, 333),
                                          (300, 640, 257), (1030, 130, 260)])
def test_layer(N, d_in, d_out, dtype):
    f = fqt()
    spread = 0.3 if dtype == torch.float16 else 1.0
    x, g = heavy(N, N, d_in, dtype, spread), heavy(N + 1, N, d_out, dtype, spread)
    w = heavy(N + 2, d_out, d_in, spread=0.2) * d_in ** -0.5
    W8, W8t = f.fqt_fp8_quantize(w, tile=True, by_row=True, by_col=True)
    xd, wd, gd = host(x), host(w), host(g)
    for relu in (False, True):
        Y, X8t, _ = f.fqt_fp8_linear_forward(x, W8, relu=relu)
        check_product(Y, F.operand(xd), F.operand(wd, tile=True), relu=relu)
        same_operand(X8t, F.operand(xd.T))
        Y2, none, _ = f.fqt_fp8_linear_forward(x, W8, relu=relu, save=False)
        assert none is None
        check_product(Y2, F.operand(xd), F.operand(wd, tile=True), relu=relu)
    for sr in (True, False):
        u = [F.uniforms(N, d_out, 11, s) if sr else None for s in (0, 1)]
        g1, g2 = F.operand(gd.T, u=u[0].T if sr else None), F.operand(gd, u=u[1])
        gW, gX, _ = f.fqt_fp8_linear_backward(g, X8t, W8t, seed=11, stochastic=sr)
        check_product(gW, g1, F.operand(xd.T))
        check_product(gX, g2, F.operand(wd.T, tile=True))
        gW2, gX2, _ = f.fqt_fp8_linear_backward(g, X8t, W8t, seed=11, stochastic=sr, relu_input=x)
        assert torch.equal(gW, gW2)
        check_product(gX2, g2, F.operand(wd.T, tile=True), mask=xd)
        gW3, gX3, _ = f.fqt_fp8_linear_backward(g, X8t, None, seed=11, stochastic=sr, input_grad=False)
        assert gX3 is None and torch.equal(gW, gW3)


def test_gradients_estimate_the_layer_gradient():
    """Over seeds the stochastic gradients average to g^T Q(x) and g Q(w): against differences of the layer's
    forward in float64, with the spread that 64 seeds leave (the standard error of the mean, five of them, and a
    floor for the elements that hardly vary)."""
    f = fqt()
    N, d_in, d_out = 40, 130, 70
    x, g = heavy(40, N, d_in, spread=0.5), heavy(41, N, d_out, spread=1.0)
    w = heavy(42, d_out, d_in, spread=0.2)
    W8t = f.fqt_fp8_quantize(w, tile=True, by_row=False, by_col=True)[1]
    X8t = f.fqt_fp8_quantize(x, by_row=False, by_col=True)[1]
    draws = [f.fqt_fp8_linear_backward(g, X8t, W8t, seed=s)[:2] for s in range(64)]
    gd, xq, wq = host(g), F.operand(host(x).T)["value"].T, F.operand(host(w), tile=True)["value"]

    def loss(a, b):
        return ((a @ b.T) * gd).sum()
    for k, (i, j) in ((0, (0, 0)), (0, (69, 129)), (1, (0, 5)), (1, (39, 77))):
        v = np.array([float(d[k][i, j]) for d in draws])
        d = np.zeros_like(wq if k == 0 else xq)
        d[i, j] = 1.0  # the loss is bilinear: a difference of any size is the derivative
        num = (loss(xq, wq + d) - loss(xq, wq - d)) / 2 if k == 0 else (loss(xq + d, wq) - loss(xq - d, wq)) / 2
        assert abs(v.mean() - num) <= 5 * v.std(ddof=1) / 8 + 1e-4 * np.abs(gd).max()


def test_same_result_twice_and_on_another_stream():
    f = fqt()
    x, g = heavy(50, 700, 520, torch.bfloat16), heavy(51, 700, 300, torch.bfloat16)
    W8, W8t = f.fqt_fp8_quantize(heavy(52, 300, 520), tile=True, by_row=True, by_col=True)

    def step():
        Y, X8t, _ = f.fqt_fp8_linear_forward(x, W8)
        gW, gX, _ = f.fqt_fp8_linear_backward(g, X8t, W8t, seed=1)
        return Y, X8t["q"].view(torch.uint8), gW, gX
    a = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = step()
    s.synchronize()
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_output_offsets_beyond_32_bits():
    """2^31 + outputs and operand bytes: rows at the end against the same rows alone."""
    f = fqt()
    M, N, K = (1 << 20) + 130, 2050, 2100
    w = heavy(60, N, K)
    B = f.fqt_fp8_quantize(w, tile=True)[0]
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda").normal_()
    A, At = f.fqt_fp8_quantize(x, by_row=True, by_col=True, stochastic=True, seed=2)
    C, _ = f.fqt_fp8_gemm(A, B, dtype=torch.bfloat16)
    tail = dict(q=A["q"][-400:].contiguous(), exp=A["exp"][:, -400:].contiguous(), K=K)
    D, _ = f.fqt_fp8_gemm(tail, B, dtype=torch.bfloat16)
    # another number of rows may take another order of sums: two roundings apart at most
    d = (C[-400:].double() - D.double()).abs()
    assert (d <= 2.0 ** -7 * D.double().abs() + 1e-3).all()
    # the codes of the last rows: against the oracle with the elements' 64-bit indices
    from oracle import philox
    r0 = M - 40
    e = np.arange(r0 * K, M * K, dtype=np.uint64)
    u = (philox.draws(e, 2, 1) & np.uint64(0xFFFFFF)).astype(np.float64).reshape(40, K)
    want = F.operand(host(x[r0:]), u=u)
    np.testing.assert_array_equal(A["q"][r0:].view(torch.uint8).cpu().numpy(), want["q"])
    u0 = (philox.draws(e, 2, 0) & np.uint64(0xFFFFFF)).astype(np.float64).reshape(40, K)
    first = (M // 128) * 128  # the last, partial block of rows: M - first rows
    n = M - first
    wt = F.operand(host(x[first:]).T, u=u0[-n:].T)
    np.testing.assert_array_equal(At["q"][:, first:first + 128].view(torch.uint8).cpu().numpy(), wt["q"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_operands_that_lie_column_by_column(dtype):
    """q whose transpose is contiguous: the same results as row by row, through every entry point that reads one."""
    f = fqt()
    x, g = heavy(64, 150, 260, dtype, 0.5), heavy(65, 150, 70, dtype, 0.5)
    W8, W8t = f.fqt_fp8_quantize(heavy(66, 70, 260, spread=0.5), tile=True, by_row=True, by_col=True)
    A = f.fqt_fp8_quantize(x)[0]

    def turned(a):
        return dict(a, q=a["q"].view(torch.uint8).t().contiguous().t().view(torch.float8_e4m3fn))
    assert not turned(A)["q"].is_contiguous()
    assert torch.equal(f.fqt_fp8_gemm(A, W8, dtype=dtype)[0], f.fqt_fp8_gemm(turned(A), turned(W8), dtype=dtype)[0])
    Y, X8t, _ = f.fqt_fp8_linear_forward(x, W8)
    assert torch.equal(Y, f.fqt_fp8_linear_forward(x, turned(W8))[0])
    a, b = f.fqt_fp8_linear_backward(g, X8t, W8t)[:2], f.fqt_fp8_linear_backward(g, turned(X8t), turned(W8t))[:2]
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_refusals():
    f = fqt()
    x, w, g = heavy(70, 40, 200), heavy(71, 60, 200), heavy(72, 40, 60)
    W8, W8t = f.fqt_fp8_quantize(w, tile=True, by_row=True, by_col=True)
    _, X8t, _ = f.fqt_fp8_linear_forward(x, W8)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    bad_layout = dict(W8, q=W8["q"][:, :200])
    for bad in (lambda: f.fqt_fp8_quantize(x.double()), lambda: f.fqt_fp8_quantize(x.cpu()),
                lambda: f.fqt_fp8_quantize(x.t()), lambda: f.fqt_fp8_linear_forward(x[:, :100], W8),
                lambda: f.fqt_fp8_linear_forward(x, W8t), lambda: f.fqt_fp8_linear_forward(x, bad_layout),
                lambda: f.fqt_fp8_linear_forward(x, dict(W8, exp=W8["exp"].int())),
                lambda: f.fqt_fp8_gemm(W8, W8t), lambda: f.fqt_fp8_gemm(W8, W8, C=torch.empty(4, 4, device="cuda")),
                lambda: f.fqt_fp8_linear_backward(g, X8t, W8), lambda: f.fqt_fp8_linear_backward(g[:20], X8t, W8t),
                lambda: f.fqt_fp8_linear_backward(g, X8t, W8t, relu_input=x.half()),
                lambda: f.fqt_fp8_linear_backward(g, X8t, W8t, grad_W=torch.empty(60, 200, dtype=torch.half, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad, code in ((lambda: f.fqt_fp8_quantize(x[:0]), 1), (lambda: f.fqt_fp8_quantize(x, by_row=False), 1),
                      (lambda: f.fqt_fp8_linear_forward(x, W8, ws=small), 4),
                      (lambda: f.fqt_fp8_linear_backward(g, X8t, W8t, ws=small), 4),
                      (lambda: f.fqt_fp8_linear_backward(g, X8t, None), 1)):
        with pytest.raises(f.FqtError) as e:
            bad()
        assert e.value.code == code
