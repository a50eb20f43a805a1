"""The gated 8-bit layer against the float64 oracle.

Forward: with s = sum |x w| over K terms, float32 sums in any order are off by K 2^-24 s, so a and b are off by da, db.
Through H = act(a) b: |act'| <= 1.13 and |act(a)| <= |a|, so 1.13 da (|b| + db) + (|a| + da) db.  The activation itself
(exponent, reciprocal, a few roundings): with z the sigmoid's argument (a, or 2 u) s(z) is off by (4 |z| + 8) 2^-24 s(z),
of which |a s(z)| is the activation.  H's type adds half a unit in its last place (and float16's smallest step).

Checkpoints: the derivatives are off by 1.13 (the slope's own slope) da |b| + 1.13 db and 1.13 da, and 2^-19 (1 + |a|) for
the evaluation of the slope; a code adds half a step of the format at its block's scale, and the scale is the least that
holds the block's largest value within that error.  A ReLU whose input is within da of zero may be on or off.

Backward: the codes of D are defined bit for bit; the products of float32 sums are off by K 2^-24 sum |d x|."""
import numpy as np
import pytest

from oracle import feedforward as F
from oracle import gated as G

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def fqt():
    from paper_2010_14298_amd import fqt as f
    f.load()
    return f


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def matrix(seed, rows, cols, dtype=torch.float32, std=1.0, spread=0.5):
    rng = np.random.default_rng(seed)
    x = std * rng.standard_normal((rows, cols)) * np.exp(rng.normal(0, spread, (rows, 1)))
    return torch.from_numpy(x).to(dtype).cuda()


def weights(seed, hidden, d_in):
    W = matrix(seed, 2 * hidden, d_in, std=d_in ** -0.5)
    W8, W8t = fqt().fqt_fp8_quantize(W, tile=True, by_row=True, by_col=True)
    return W, W8, W8t


def bytes_of(t):
    return t.view(torch.uint8).cpu().numpy()


def check_kept(k, want, err, cols):
    """A checkpoint of values within err of want."""
    q, exp = bytes_of(k["q"]), k["exp"].cpu().numpy()
    rows, nb = exp.shape
    assert q.shape == (rows, nb * 32) and k["cols"] == cols
    assert (q[:, cols:] == 0).all()
    pad = ((0, 0), (0, nb * 32 - cols))
    top = np.pad(np.abs(want), pad).reshape(rows, nb, 32).max(2)
    slack = np.pad(err, pad).reshape(rows, nb, 32).max(2)
    E = exp.astype(int) - 127
    assert np.all(top - slack <= 448.0 * 2.0 ** E)
    assert np.all((top + slack > 448.0 * 2.0 ** (E - 1.0)) | (top <= slack) | (E == -127))
    scale = np.repeat(2.0 ** E, 32, axis=1)[:, :cols]
    y = (np.abs(want) + err) / scale
    step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3) * scale
    got = G.kept_values(q, exp, cols)
    assert np.all(np.abs(got - want) <= err + 0.5 * step)


def check_forward(X, W, act, H, kept, K):
    x, w = host(X), host(W)
    f = G.gated_forward(x, w, act)
    h = f["a"].shape[1]
    size = np.abs(F.operand(x)["value"]) @ np.abs(F.operand(w, tile=True)["value"]).T
    da, db = K * U * size[:, :h], K * U * size[:, h:]
    a, b = f["a"], f["b"]
    z = np.abs(a) if act == "silu" else 0.0 if act == "relu" else 1.6 * np.abs(a) * (1 + 0.044715 * a * a)
    value = np.abs(f["d_up"])
    ev = value * (4 * z + 8) * U
    tol = 1.13 * da * (np.abs(b) + db) + (np.abs(a) + da) * db + ev * np.abs(b)
    tol = tol + HALF[H.dtype] * (np.abs(f["H"]) + tol) + TINY[H.dtype]
    assert np.all(np.abs(host(H) - f["H"]) <= tol)
    if kept is None:
        return
    eg = 1.13 * da * np.abs(b) + 1.13 * db + 2.0 ** -19 * (1 + np.abs(a)) * np.abs(b)
    if act == "relu":
        eg = np.where(np.abs(a) <= da, np.abs(b) + db, eg)
    check_kept(kept["d_gate"], f["d_gate"], eg, h)
    check_kept(kept["d_up"], f["d_up"], 1.13 * da + ev, h)
    want = F.operand(x.T)
    np.testing.assert_array_equal(kept["X8t"]["exp"].cpu().numpy(), want["exp"])
    np.testing.assert_array_equal(bytes_of(kept["X8t"]["q"]), want["q"])


# ---------------------------------------------------------------------------
# forward
# ---------------------------------------------------------------------------
SHAPES = [(1, 64, 32), (1, 1000, 1001), (2, 129, 33), (7, 100, 1), (16, 256, 512), (17, 130, 96), (64, 384, 200),
          (65, 512, 131), (130, 4096, 68), (257, 640, 320), (300, 96, 1000), (513, 320, 257), (131, 1200, 70),
          (190, 1800, 65), (129, 900, 1)]


@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,d_in,hidden", SHAPES)
def test_forward(N, d_in, hidden, dtype, act):
    X = matrix(N + d_in, N, d_in, dtype)
    W, W8, _ = weights(hidden, hidden, d_in)
    f = fqt()
    H, kept, _ = f.fqt_fp8_gated_forward(X, W8, act=act)
    check_forward(X, W, act, H, kept, d_in)
    alone, none, _ = f.fqt_fp8_gated_forward(X, W8, act=act, save=False)
    assert none is None
    check_forward(X, W, act, alone, None, d_in)


@pytest.mark.parametrize("N,d_in,hidden,dtype", [(1024, 512, 2048, torch.bfloat16), (2304, 256, 1024, torch.float32),
                                                 (1000, 1024, 1200, torch.float16), (4100, 130, 900, torch.bfloat16),
                                                 (1030, 1100, 1100, torch.float32)])
def test_forward_of_many_tiles(N, d_in, hidden, dtype):
    X = matrix(1, N, d_in, dtype)
    W, W8, _ = weights(2, hidden, d_in)
    H, kept, _ = fqt().fqt_fp8_gated_forward(X, W8)
    check_forward(X, W, "silu", H, kept, d_in)


@pytest.mark.parametrize("N", [3, 40, 200, 600])
def test_exact_sums_give_the_oracles_bits(N):
    """Small whole numbers: every sum is exact, and with the ReLU so are H and both derivatives."""
    rng = np.random.default_rng(N)
    d_in, hidden = 160, 100
    x = rng.integers(-4, 5, (N, d_in)) * (rng.random((N, d_in)) < 0.1)
    w = rng.integers(-2, 3, (2 * hidden, d_in)) * (rng.random((2 * hidden, d_in)) < 0.2)
    x[0, ::7], w[0, 3] = 4, 2  # every block's scale takes the numbers as they are
    X = torch.from_numpy(x.astype(np.float32)).cuda()
    W8, _ = fqt().fqt_fp8_quantize(torch.from_numpy(w.astype(np.float32)).cuda(), tile=True)
    H, kept, _ = fqt().fqt_fp8_gated_forward(X, W8, act="relu")
    f = G.gated_forward(x, w, "relu")
    np.testing.assert_array_equal(host(H), f["H"])
    for name in ("d_gate", "d_up"):
        want = G.kept(f[name])
        np.testing.assert_array_equal(kept[name]["exp"].cpu().numpy(), want["exp"])
        got = bytes_of(kept[name]["q"])
        np.testing.assert_array_equal(F.decode(got), F.decode(want["q"]))


@pytest.mark.parametrize("N", [5, 50, 300])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu"])
def test_non_finite_rows_stay_in_their_rows(N, act):
    """A NaN in X: its row of H is NaN and its checkpoints' blocks are; other rows keep their bits."""
    X = matrix(3, N, 200)
    _, W8, _ = weights(4, 70, 200)
    H0, k0, _ = fqt().fqt_fp8_gated_forward(X, W8, act=act)
    Y = X.clone()
    Y[N // 2, 7] = float("nan")
    H1, k1, _ = fqt().fqt_fp8_gated_forward(Y, W8, act=act)
    rows = torch.arange(N, device="cuda") != N // 2
    assert torch.equal(H0[rows], H1[rows]) and torch.isnan(H1[N // 2]).all()
    for name in ("d_gate", "d_up"):
        assert torch.equal(k0[name]["exp"][rows], k1[name]["exp"][rows])
        assert torch.equal(k0[name]["q"][rows].view(torch.uint8), k1[name]["q"][rows].view(torch.uint8))
        assert (k1[name]["exp"][N // 2] == 255).all()
        assert torch.isnan(k1[name]["q"][N // 2].float()).all()


@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu"])
def test_saturated_activations(act):
    """Pre-activations of 2^60 and -2^60: the value is a or next to 0, the slope 1 or 0, nothing is non-finite."""
    X = torch.zeros((4, 32), device="cuda")
    X[0, 0], X[1, 0], X[:, 1] = 2.0 ** 60, -(2.0 ** 60), 1.0
    X[:2, 1] = 0.0
    W = torch.zeros((64, 32), device="cuda")
    W[:32, 0], W[32:, 0], W[32:, 1] = 1.0, 1.0, 1.0
    W8, _ = fqt().fqt_fp8_quantize(W, tile=True)
    H, kept, _ = fqt().fqt_fp8_gated_forward(X, W8, act=act)
    assert torch.isfinite(H[:1]).all() and (H[0] == 2.0 ** 120).all() and (H[1].abs() <= 2.0 ** 30).all()
    up, gate = (torch.from_numpy(G.kept_values(bytes_of(kept[n]["q"]), kept[n]["exp"].cpu().numpy(), 32))
                for n in ("d_up", "d_gate"))
    assert (up[0] == 2.0 ** 60).all() and (up[1].abs() <= 2.0 ** -60).all() and (up[2:] == 0).all()
    # b is 2^60, -2^60, 1, 1; the slope at 0 is a half, a ReLU's 0
    half = 0.0 if act == "relu" else 0.5
    assert (gate[0] == 2.0 ** 60).all() and (gate[1].abs() <= 2.0 ** -60).all() and (gate[2:] == half).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [9, 300])
def test_strides_and_rows_behind_stay(N, dtype):
    """X and H inside larger buffers: what lies around H keeps its values."""
    X = matrix(5, N, 200, dtype)
    _, W8, _ = weights(6, 70, 200)
    f = fqt()
    want, kept, _ = f.fqt_fp8_gated_forward(X, W8)
    buf = torch.full((N, 217), float("nan"), dtype=dtype, device="cuda")
    buf[:, 5:205] = X
    out = torch.full((N + 3, 79), 7.0, dtype=dtype, device="cuda")
    H, kept2, _ = f.fqt_fp8_gated_forward(buf[:, 5:205], W8, H=out[1:N + 1, 3:73])
    assert torch.equal(H, want)
    assert (out[0] == 7).all() and (out[N + 1:] == 7).all() and (out[:, :3] == 7).all() and (out[:, 73:] == 7).all()
    for name in ("d_gate", "d_up"):
        assert torch.equal(kept[name]["q"].view(torch.uint8), kept2[name]["q"].view(torch.uint8))
    repeated, _, _ = f.fqt_fp8_gated_forward(X[:1].expand(N, 200), W8)
    assert torch.equal(repeated, repeated[:1].expand(N, 70))


def test_weights_that_lie_column_by_column():
    X = matrix(7, 150, 256, torch.bfloat16)
    W, W8, _ = weights(8, 128, 256)
    turned = dict(q=W8["q"].t().contiguous().t(), exp=W8["exp"], K=W8["K"])
    f = fqt()
    a, b = f.fqt_fp8_gated_forward(X, W8)[0], f.fqt_fp8_gated_forward(X, turned)[0]
    assert torch.equal(a, b)


def test_the_same_call_gives_the_same_bits():
    X = matrix(9, 700, 512, torch.bfloat16)
    _, W8, W8t = weights(10, 300, 512)
    G_ = matrix(11, 700, 300, torch.bfloat16)
    f = fqt()

    def once():
        H, kept, _ = f.fqt_fp8_gated_forward(X, W8)
        gW, gX, _ = f.fqt_fp8_gated_backward(G_, kept, W8t, seed=3)
        return [H, kept["d_gate"]["q"].view(torch.uint8), kept["d_up"]["q"].view(torch.uint8), gW, gX]
    first = once()
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, once()))


# ---------------------------------------------------------------------------
# backward
# ---------------------------------------------------------------------------
def checkpoint(seed, rows, cols, spread=1.0):
    """A checkpoint of random values, in the oracle's bytes."""
    rng = np.random.default_rng(seed)
    v = rng.standard_normal((rows, cols)) * np.exp(rng.normal(0, spread, (rows, cols)))
    k = G.kept(v)
    return dict(q=torch.from_numpy(k["q"]).cuda().view(torch.float8_e4m3fn), exp=torch.from_numpy(k["exp"]).cuda(),
                cols=cols), k["value"]


def identity(n):
    """The operand of the n x n identity: products with it give the other operand's values exactly."""
    e, _ = fqt().fqt_fp8_quantize(torch.eye(n, device="cuda"))
    return e


def read_out(g, d_gate, d_up, **how):
    """Both quantizations of D as they stand for: (D^T's [2 hidden, N], D's [N, 2 hidden])."""
    f = fqt()
    N, cols = g.shape[0], 2 * g.shape[1]
    gW = f.fqt_fp8_gated_backward(g, dict(X8t=identity(N), d_gate=d_gate, d_up=d_up), None, input_grad=False, **how)[0]
    X8t, _ = f.fqt_fp8_quantize(torch.zeros((cols, N), device="cuda"))
    gX = f.fqt_fp8_gated_backward(g, dict(X8t=X8t, d_gate=d_gate, d_up=d_up), identity(cols), **how)[1]
    return gW, gX


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,hidden", [(1, 1), (3, 2), (5, 3), (130, 64), (128, 65), (200, 66), (77, 131), (257, 100), (130, 256),
                                      (64, 130), (200, 258), (33, 389)])
def test_gradient_codes_bit_for_bit(N, hidden, dtype, stochastic):
    """Both quantizations of D, read out through products with identities."""
    g = matrix(N, N, hidden, dtype, spread=2.0)
    d_gate, vg = checkpoint(1, N, hidden)
    d_up, vu = checkpoint(2, N, hidden)
    seed = (5 << 32) + 11
    gW, gX = read_out(g, d_gate, d_up, seed=seed, stochastic=stochastic)
    t, r = G.gradient_operands(host(g), vg, vu, seed if stochastic else None)
    np.testing.assert_array_equal(host(gW), t["value"])
    if dtype == torch.float32:
        np.testing.assert_array_equal(host(gX), r["value"])
    else:
        assert np.all(np.abs(host(gX) - r["value"]) <= HALF[dtype] * np.abs(r["value"]) + TINY[dtype])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,d_in,hidden", [(1, 64, 32), (33, 130, 70), (300, 192, 520), (700, 96, 131),
                                           (1200, 160, 600)])
def test_backward(N, d_in, hidden, dtype):
    f = fqt()
    X, g = matrix(20, N, d_in, dtype), matrix(21, N, hidden, dtype, spread=1.5)
    W, W8, W8t = weights(22, hidden, d_in)
    _, kept, _ = f.fqt_fp8_gated_forward(X, W8)
    gW, gX, ws = f.fqt_fp8_gated_backward(g, kept, W8t, seed=17)
    vg, vu = (G.kept_values(bytes_of(kept[n]["q"]), kept[n]["exp"].cpu().numpy(), hidden) for n in ("d_gate", "d_up"))
    t, r = G.gradient_operands(host(g), vg, vu, 17)
    xt, wt = F.operand(host(X).T)["value"], F.operand(host(W).T, tile=True)["value"]
    want_W, size_W = t["value"] @ xt.T, np.abs(t["value"]) @ np.abs(xt).T
    assert np.all(np.abs(host(gW) - want_W) <= N * U * size_W)
    want, size = r["value"] @ wt.T, np.abs(r["value"]) @ np.abs(wt).T
    assert np.all(np.abs(host(gX) - want) <= 2 * hidden * U * size + HALF[dtype] * (np.abs(want) + 2 * hidden * U * size)
                  + TINY[dtype])
    # alone (its sums may run in another order, which float32's bound covers), and into a caller's buffers
    only, none, _ = f.fqt_fp8_gated_backward(g, kept, None, seed=17, input_grad=False, ws=ws)
    assert none is None and np.all(np.abs(host(only) - want_W) <= N * U * size_W)
    out, buf = torch.full_like(gW, 3.0), torch.full((N, d_in + 9), 5.0, dtype=dtype, device="cuda")
    f.fqt_fp8_gated_backward(g, kept, W8t, seed=17, grad_W=out, grad_X=buf[:, 2:d_in + 2])
    assert torch.equal(out, gW) and torch.equal(buf[:, 2:d_in + 2], gX)
    assert (buf[:, :2] == 5).all() and (buf[:, d_in + 2:] == 5).all()


def test_operands_that_lie_column_by_column():
    f = fqt()
    X, g = matrix(20, 256, 128), matrix(21, 256, 64)
    _, W8, W8t = weights(22, 64, 128)
    _, kept, _ = f.fqt_fp8_gated_forward(X, W8)
    a = f.fqt_fp8_gated_backward(g, kept, W8t, seed=17)

    def turned(o):
        return dict(q=o["q"].t().contiguous().t(), exp=o["exp"], K=o["K"])
    b = f.fqt_fp8_gated_backward(g, dict(kept, X8t=turned(kept["X8t"])), turned(W8t), seed=17)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_gradient_strides_zeros_and_non_finite():
    N, hidden = 140, 90
    g = matrix(30, N, hidden, torch.bfloat16)
    g[3], g[70] = 0.0, 0.0
    d_gate, vg = checkpoint(31, N, hidden)
    d_up, vu = checkpoint(32, N, hidden)
    a = read_out(g, d_gate, d_up, seed=4)
    assert (a[1][3] == 0).all() and (a[0][:, 70] == 0).all()
    buf = torch.full((N, hidden + 13), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, 7:hidden + 7] = g
    b = read_out(buf[:, 7:hidden + 7], d_gate, d_up, seed=4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    one = read_out(g[:1].expand(N, hidden), d_gate, d_up, seed=4)
    two = read_out(g[:1].expand(N, hidden).contiguous(), d_gate, d_up, seed=4)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    g[5, 2] = float("inf")  # the blocks that hold it become NaN
    c = read_out(g, d_gate, d_up, seed=4)
    t, r = G.gradient_operands(host(g), vg, vu, 4)
    assert np.isnan(r["value"][5]).any() and not np.isnan(r["value"][6]).any()
    assert torch.isnan(c[1][5]).all() and torch.isfinite(c[1][6]).all()


def test_smallest_scales():
    """Checkpoints with the least scale 2^-127 and gradients near float32's ends."""
    N, hidden = 4, 32
    q = torch.full((N, 32), 0x78, dtype=torch.uint8, device="cuda")  # 256
    q[:, 1::2] = 0x01                                                # 2^-9
    low = dict(q=q.view(torch.float8_e4m3fn), exp=torch.zeros((N, 1), dtype=torch.uint8, device="cuda"), cols=hidden)
    one = dict(q=q.view(torch.float8_e4m3fn), exp=torch.full((N, 1), 127, dtype=torch.uint8, device="cuda"), cols=hidden)
    g = torch.full((N, hidden), 2.0 ** 100, device="cuda")
    gW, gX = read_out(g, low, one, stochastic=False)
    vg = G.kept_values(q.cpu().numpy(), np.zeros((N, 1), np.uint8), hidden)
    vu = G.kept_values(q.cpu().numpy(), np.full((N, 1), 127, np.uint8), hidden)
    t, r = G.gradient_operands(host(g), vg, vu)
    np.testing.assert_array_equal(host(gW), t["value"])
    np.testing.assert_array_equal(host(gX), r["value"])


def test_gradients_against_differences():
    """The loss sum(G H) of the layer without quantization, by differences in float64, against the kernels' gradients:
    four operands' noise of 3 mantissa bits, at most 7 % together (a cosine of 0.997); 0.99 leaves room."""
    f = fqt()
    N, d_in, hidden = 64, 48, 40
    X, g = matrix(40, N, d_in), matrix(41, N, hidden)
    W, W8, W8t = weights(42, hidden, d_in)
    _, kept, _ = f.fqt_fp8_gated_forward(X, W8)
    gW, gX, _ = f.fqt_fp8_gated_backward(g, kept, W8t, seed=1)
    x, w, gd = host(X), host(W), host(g)

    def loss(x, w):
        a, b = x @ w[:hidden].T, x @ w[hidden:].T
        return float((gd * G.activation(a, "silu")[0] * b).sum())
    rng = np.random.default_rng(0)
    for got, at, of in ((host(gW), w, lambda v: loss(x, v)), (host(gX), x, lambda v: loss(v, w))):
        num, kernel = [], []
        for _ in range(60):
            d = rng.standard_normal(at.shape)
            num.append((of(at + 1e-5 * d) - of(at - 1e-5 * d)) / 2e-5)
            kernel.append(float((got * d).sum()))
        num, kernel = np.array(num), np.array(kernel)
        assert num @ kernel / np.linalg.norm(num) / np.linalg.norm(kernel) > 0.99


@pytest.mark.parametrize("N,d_in,hidden,dtype", [(9, 200, 70, torch.float32), (140, 200, 70, torch.float16),
                                                 (1024, 512, 2048, torch.float16), (2304, 256, 1024, torch.bfloat16),
                                                 (8192, 128, 2048, torch.bfloat16)])
def test_each_output_alone(N, d_in, hidden, dtype):
    """What a caller of the library may leave out: any of what the forward keeps, either gradient."""
    f = fqt()
    lib, stream = f.load(), torch.cuda.current_stream().cuda_stream
    X, g = matrix(60, N, d_in, dtype), matrix(61, N, hidden, dtype)
    W, W8, W8t = weights(62, hidden, d_in)
    H, kept, _ = f.fqt_fp8_gated_forward(X, W8)
    t, w8 = f.TYPES[dtype], f.Fp8(W8["q"].data_ptr(), W8["exp"].data_ptr(), 0)
    ws = torch.empty(max(f.fqt_fp8_gated_forward_workspace(N, d_in, hidden), 16), dtype=torch.uint8, device="cuda")
    for name in ("X8t", "d_gate", "d_up"):
        out = {k: torch.full_like(kept[name][k].view(torch.uint8), 9) for k in ("q", "exp")}
        where = (f.Fp8(out["q"].data_ptr(), out["exp"].data_ptr(), 0) if name == "X8t"
                 else f.Kept(out["q"].data_ptr(), out["exp"].data_ptr()))
        alone = torch.empty_like(H)
        assert lib.fqt_fp8_gated_forward(X.data_ptr(), t, N, d_in, d_in, w8, hidden, 0, alone.data_ptr(), hidden,
                                         *(where if n == name else None for n in ("X8t", "d_gate", "d_up")),
                                         ws.data_ptr(), ws.numel(), stream) == 0
        assert torch.equal(out["q"], kept[name]["q"].view(torch.uint8)) and torch.equal(out["exp"], kept[name]["exp"])
        if name != "X8t":  # (without a checkpoint few rows take another form)
            assert torch.equal(alone, H)
    _, gX, ws = f.fqt_fp8_gated_backward(g, kept, W8t, seed=3)
    c = {n: f.Kept(kept[n]["q"].data_ptr(), kept[n]["exp"].data_ptr()) for n in ("d_gate", "d_up")}
    w8t, alone = f.Fp8(W8t["q"].data_ptr(), W8t["exp"].data_ptr(), 0), torch.empty_like(gX)
    assert lib.fqt_fp8_gated_backward(g.data_ptr(), t, N, hidden, hidden, c["d_gate"], c["d_up"], None, w8t, d_in, 1, 3, None,
                                      alone.data_ptr(), d_in, ws.data_ptr(), ws.numel(), stream) == 0
    vg, vu = (G.kept_values(bytes_of(kept[n]["q"]), kept[n]["exp"].cpu().numpy(), hidden) for n in ("d_gate", "d_up"))
    r = G.gradient_operands(host(g), vg, vu, 3)[1]["value"]
    wt = F.operand(host(W).T, tile=True)["value"]
    size = np.abs(r) @ np.abs(wt).T
    # both within 2 hidden U of the exact sums, and each rounded once
    bound = 4 * hidden * U * size + 2 * HALF[dtype] * (np.abs(host(gX)) + 4 * hidden * U * size) + 2 * TINY[dtype]
    assert np.all(np.abs(host(alone) - host(gX)) <= bound)


# ---------------------------------------------------------------------------
# refusals of the binding
# ---------------------------------------------------------------------------
def test_refusals():
    f = fqt()
    X, g = matrix(50, 20, 64, torch.bfloat16), matrix(51, 20, 48, torch.bfloat16)
    _, W8, W8t = weights(52, 48, 64)
    odd, _ = f.fqt_fp8_quantize(matrix(53, 33, 64), tile=True)
    _, kept, _ = f.fqt_fp8_gated_forward(X, W8)
    for call in (lambda: f.fqt_fp8_gated_forward(X, W8, act="tanh"), lambda: f.fqt_fp8_gated_forward(X, odd),
                 lambda: f.fqt_fp8_gated_forward(X[:, :60], W8), lambda: f.fqt_fp8_gated_forward(X.cpu(), W8),
                 lambda: f.fqt_fp8_gated_forward(X.double(), W8), lambda: f.fqt_fp8_gated_forward(X.t(), W8),
                 lambda: f.fqt_fp8_gated_forward(X, W8, H=torch.empty((20, 47), dtype=X.dtype, device="cuda")),
                 lambda: f.fqt_fp8_gated_forward(X, W8, H=torch.empty((20, 48), device="cuda")),
                 lambda: f.fqt_fp8_gated_backward(g[:, :47], kept, W8t), lambda: f.fqt_fp8_gated_backward(g[:19], kept, W8t),
                 lambda: f.fqt_fp8_gated_backward(g, dict(kept, d_up=dict(kept["d_up"], cols=47)), W8t),
                 lambda: f.fqt_fp8_gated_backward(g, dict(kept, d_gate=dict(kept["d_gate"], exp=kept["d_gate"]["exp"].cpu())), W8t),
                 lambda: f.fqt_fp8_gated_backward(g, dict(kept, d_gate=dict(kept["d_gate"], q=kept["d_gate"]["q"].view(torch.uint8))), W8t),
                 lambda: f.fqt_fp8_gated_backward(g, kept, W8), lambda: f.fqt_fp8_gated_backward(g, kept, W8t, grad_W=torch.empty((96, 64)))):
        with pytest.raises(ValueError):
            call()
    assert f.fqt_fp8_gated_forward(X, W8, save=False)[2] is None  # twenty rows, read as they are
    with pytest.raises(f.FqtError) as e:
        f.fqt_fp8_gated_forward(X, W8, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 4
