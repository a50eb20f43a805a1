"""The gated forward's largest tiles, at sizes that take them, against float64 on the GPU: whole blocks and ragged edges,
widths up to and beyond 1024, every type, with and without checkpoints.  Tolerances: those of test_gpu_gated.py."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def operand_values(a):
    rows, ld = a["q"].shape
    e = a["exp"].transpose(0, 1).reshape(rows, -1)[:, :ld // 128].double() - 127
    return a["q"].double() * torch.exp2(e).repeat_interleave(128, 1)


def check_kept(k, want, err):
    rows, cols = want.shape
    nb = (cols + 31) // 32
    assert (k["q"][:, cols:].float() == 0).all()
    pad = (0, nb * 32 - cols)
    top, slack = (torch.nn.functional.pad(t, pad).view(rows, nb, 32).amax(2) for t in (want.abs(), err))
    E = k["exp"].double() - 127
    assert (top - slack <= 448.0 * torch.exp2(E)).all()
    assert ((top + slack > 448.0 * torch.exp2(E - 1.0)) | (top <= slack) | (E == -127)).all()
    scale = torch.exp2(E).repeat_interleave(32, 1)[:, :cols]
    y = (want.abs() + err) / scale
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3) * scale
    assert ((k["q"][:, :cols].double() * scale - want).abs() <= err + 0.5 * step).all()


@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("N,d_in,hidden,dtype", [(8100, 128, 2040, torch.bfloat16), (8192, 256, 2048, torch.float32),
                                                 (8192, 384, 2048, torch.float16), (8100, 1100, 2040, torch.float16),
                                                 (8192, 1152, 2048, torch.bfloat16), (8100, 200, 2040, torch.float32)])
def test_largest_tiles(N, d_in, hidden, dtype, act):
    assert fqt.fqt_fp8_gemm_form(N, 2 * hidden, d_in, masked=True) == "large"
    gen = torch.Generator("cuda").manual_seed(N + d_in)
    X = torch.randn((N, d_in), generator=gen, device="cuda").to(dtype)
    W8, _ = fqt.fqt_fp8_quantize(torch.randn((2 * hidden, d_in), generator=gen, device="cuda") * d_in ** -0.5, tile=True)
    H, kept, _ = fqt.fqt_fp8_gated_forward(X, W8, act=act)
    alone, _, _ = fqt.fqt_fp8_gated_forward(X, W8, act=act, save=False)
    assert torch.equal(H, alone)
    x, w = operand_values(fqt.fqt_fp8_quantize(X)[0]), operand_values(W8)
    a, b = (x @ w.t()).split(hidden, 1)
    da, db = (x.abs() @ w.abs().t() * (d_in * U)).split(hidden, 1)
    if act == "relu":
        z, value, slope = torch.zeros_like(a), a.clamp(min=0.0), (a > 0).double()
    else:
        z = a if act == "silu" else math.sqrt(8 / math.pi) * (a + 0.044715 * a ** 3)
        dz = 1.0 if act == "silu" else math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * a ** 2)
        s = torch.sigmoid(z)
        value, slope = a * s, s + a * s * (1 - s) * dz
    ev = value.abs() * (4 * z.abs() + 8) * U
    want = value * b
    tol = 1.13 * da * (b.abs() + db) + (a.abs() + da) * db + ev * b.abs()
    assert ((H.double() - want).abs() <= tol + HALF[dtype] * (want.abs() + tol) + TINY[dtype]).all()
    eg = 1.13 * da * b.abs() + 1.13 * db + 2.0 ** -19 * (1 + a.abs()) * b.abs()
    if act == "relu":
        eg = torch.where(a.abs() <= da, b.abs() + db, eg)
    check_kept(kept["d_gate"], slope * b, eg)
    check_kept(kept["d_up"], value, 1.13 * da + ev)


def test_one_checkpoint_of_the_two_and_rows_behind():
    """Either checkpoint may be left out of the C call; what lies behind H keeps its values."""
    import ctypes
    N, d_in, hidden = 8192, 128, 2048
    gen = torch.Generator("cuda").manual_seed(5)
    X = torch.randn((N, d_in), generator=gen, device="cuda").bfloat16()
    W8, _ = fqt.fqt_fp8_quantize(torch.randn((2 * hidden, d_in), generator=gen, device="cuda") * d_in ** -0.5, tile=True)
    buf = torch.full((N + 1, hidden + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    H, kept, ws = fqt.fqt_fp8_gated_forward(X, W8, H=buf[:N, :hidden])
    assert (buf[N] == 5).all() and (buf[:, hidden:] == 5).all()
    assert torch.equal(H, fqt.fqt_fp8_gated_forward(X, W8)[0])
    for name, at in (("d_gate", 11), ("d_up", 12)):
        one = fqt.fp8_kept(N, hidden, "cuda")
        c = fqt.Kept(one["q"].data_ptr(), one["exp"].data_ptr())
        args = [X.data_ptr(), 1, N, d_in, d_in, fqt.Fp8(W8["q"].data_ptr(), W8["exp"].data_ptr(), 0), hidden, 0,
                H.data_ptr(), hidden + 8, None, None, None, ws.data_ptr(), ws.numel(),
                torch.cuda.current_stream().cuda_stream]
        args[at] = ctypes.byref(c)
        assert fqt.load().fqt_fp8_gated_forward(*args) == 0
        torch.cuda.synchronize()
        assert torch.equal(one["q"].view(torch.uint8), kept[name]["q"].view(torch.uint8))
        assert torch.equal(one["exp"], kept[name]["exp"])
