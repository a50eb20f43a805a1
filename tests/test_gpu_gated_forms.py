"""Every form of the gated forward of many rows, on sizes that take it and keep it in its loop: the same tiles as the
plain products' of [W_gate; W_up], where these are not split, and the parts where the workspace holds them.
Tolerances: those of test_gpu_gated.py."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402
from tests import test_gpu_gated as base  # noqa: E402

gpu = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16

# N, d_in, hidden, type, activation.  Stages (of 128 along K) that the tile's unrolled loop needs: 6 (256 x 128), 8
# (128 x 128 and 64 x 128), 4 (256 x 256, even and odd counts end by different ways), 3 (two blocks a unit).
CASES = {
    "parts": [(130, 9000, 1, F32, "silu"), (130, 9000, 67, BF16, "gelu_tanh"), (130, 9000, 131, F32, "relu"),
              (190, 5000, 67, F16, "silu"), (129, 4000, 1, BF16, "relu"), (1000, 4999, 350, F32, "gelu_tanh"),
              (250, 2048, 66, F16, "silu"), (130, 6000, 3, F16, "gelu_tanh")],
    "half": [(2048, 1100, 512, BF16, "silu"), (1024, 2000, 1024, F32, "gelu_tanh"), (1990, 1100, 501, F16, "relu")],
    "small": [(1500, 1500, 700, BF16, "silu"), (2048, 2048, 1000, F32, "relu")],
    "middle": [(8185, 900, 511, F32, "silu"), (8192, 1100, 512, BF16, "gelu_tanh"), (8185, 1000, 500, F16, "relu")],
    "pair": [(8100, 1000, 2040, BF16, "gelu_tanh"), (8192, 512, 2048, F32, "silu")],
    "large": [(8192, 1280, 2048, BF16, "silu"), (8100, 1200, 2040, F32, "gelu_tanh")],
}
LIST = [(form, *c) for form, cases in CASES.items() for c in cases]


def parts(N, d_in, hidden):
    """How many parts along K the workspace has room for (0: none)."""
    operand = N * ((d_in + 127) // 128 * 128) + (d_in + 511) // 512 * 4 * N
    room = fqt.fqt_fp8_gated_forward_workspace(N, d_in, hidden) - operand
    return room // (8 * N * hidden) if room >= 1024 else 0


def form_of(N, d_in, hidden):
    if parts(N, d_in, hidden) > 1:
        return "parts"
    form = fqt.fqt_fp8_gemm_form(N, 2 * hidden, d_in, masked=True)
    if form == "small":  # not split by the plain product's rule, and a pass over parts costs the gated one more
        return "half" if -(-N // 128) * -(-hidden // 64) <= 128 else "small"
    if form == "large":
        return "pair" if d_in <= 1024 else "large"
    return form


@pytest.mark.skipif(not os.path.exists(fqt.LIB_PATH), reason="libfqt.so not built")
def test_the_sizes_take_their_forms():
    for form, N, d_in, hidden, _, _ in LIST:
        assert form_of(N, d_in, hidden) == form, (form, N, d_in, hidden)


@gpu
@pytest.mark.parametrize("form,N,d_in,hidden,dtype,act", LIST)
def test_forward(form, N, d_in, hidden, dtype, act):
    assert form_of(N, d_in, hidden) == form
    X = base.matrix(N + d_in, N, d_in, dtype)
    W, W8, _ = base.weights(hidden, hidden, d_in)
    H, kept, _ = fqt.fqt_fp8_gated_forward(X, W8, act=act)
    base.check_forward(X, W, act, H, kept, d_in)
    alone, none, ws = fqt.fqt_fp8_gated_forward(X, W8, act=act, save=False)
    assert none is None and ws is not None and torch.equal(H, alone)


@gpu
@pytest.mark.parametrize("form,N,d_in,hidden,dtype,act", [c for c in LIST if c[0] == "parts"])
def test_parts_leave_the_rest_alone(form, N, d_in, hidden, dtype, act):
    """H at odd offsets inside a larger buffer, either checkpoint left out: the same bits, and nothing around them."""
    X = base.matrix(N + d_in, N, d_in, dtype)
    _, W8, _ = base.weights(hidden, hidden, d_in)
    want, kept, ws = fqt.fqt_fp8_gated_forward(X, W8, act=act)
    out = torch.full((N + 2, hidden + 5), 7.0, dtype=dtype, device="cuda")
    H, again, _ = fqt.fqt_fp8_gated_forward(X, W8, act=act, H=out[1:N + 1, 3:hidden + 3], ws=ws)
    assert torch.equal(H, want)
    assert (out[0] == 7).all() and (out[N + 1] == 7).all() and (out[:, :3] == 7).all() and (out[:, hidden + 3:] == 7).all()
    w8 = fqt.Fp8(W8["q"].data_ptr(), W8["exp"].data_ptr(), 0)
    for name in ("d_gate", "d_up"):
        assert torch.equal(again[name]["q"].view(torch.uint8), kept[name]["q"].view(torch.uint8))
        assert torch.equal(again[name]["exp"], kept[name]["exp"])
        rows, pitch = kept[name]["q"].shape
        q, e = (torch.full((rows + 1, n), 9, dtype=torch.uint8, device="cuda") for n in (pitch, pitch // 32))
        one, alone = fqt.Kept(q.data_ptr(), e.data_ptr()), torch.empty_like(want)
        assert fqt.load().fqt_fp8_gated_forward(
            X.data_ptr(), fqt.TYPES[dtype], N, d_in, d_in, w8, hidden, fqt.ACTS[act], alone.data_ptr(), hidden, None,
            *(one if n == name else None for n in ("d_gate", "d_up")), ws.data_ptr(), ws.numel(),
            torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(alone, want) and torch.equal(q[:rows], kept[name]["q"].view(torch.uint8))
        assert torch.equal(e[:rows], kept[name]["exp"]) and (q[rows] == 9).all() and (e[rows] == 9).all()
