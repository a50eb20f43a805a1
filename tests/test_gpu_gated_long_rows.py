"""Few rows of long widths, nothing kept: read as they are while that is faster, in parts along K beyond.  A call that takes
no workspace reads them as they are."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402
from tests import test_gpu_gated as base  # noqa: E402

# N, d_in, hidden: on both sides of each bound
RAW = [(16, 12800, 64), (1, 16384, 512), (1, 1 << 16, 3057), (16, 1 << 20, 4096), (17, 8192, 512), (128, 8192, 512),
       (48, 4096, 2048), (17, 4096, 4096), (17, 12288, 16)]
TILES = [(16, 12801, 64), (1, 16385, 512), (1, 1 << 16, 3056), (17, 12289, 512), (128, 32768, 16), (48, 6145, 2048),
         (48, 8192, 1365), (1, 1 << 23, 1), (33, 1 << 20, 1)]


@pytest.mark.skipif(not os.path.exists(fqt.LIB_PATH), reason="libfqt.so not built")
def test_which_rows_are_read_as_they_are():
    for case in RAW:
        assert fqt.fqt_fp8_gated_forward_workspace(*case, save=False) == 0, case
    for case in TILES:
        assert fqt.fqt_fp8_gated_forward_workspace(*case, save=False) > 0, case


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", base.TYPES)
@pytest.mark.parametrize("N,d_in,hidden,act,raw", [
    (1, 16384, 64, "silu", False), (16, 12801, 33, "gelu_tanh", False), (17, 12289, 40, "relu", False),
    (48, 8192, 1365, "silu", False), (16, 12800, 64, "silu", True), (17, 12288, 16, "relu", True)])
def test_long_rows(N, d_in, hidden, act, raw, dtype):
    X = base.matrix(N + d_in, N, d_in, dtype)
    W, W8, _ = base.weights(hidden, hidden, d_in)
    H, none, ws = fqt.fqt_fp8_gated_forward(X, W8, act=act, save=False)
    assert none is None and (ws is None) == raw
    base.check_forward(X, W, act, H, None, d_in)
    kept = fqt.fqt_fp8_gated_forward(X, W8, act=act)[0]
    base.check_forward(X, W, act, kept, None, d_in)
    if ws is not None:  # the same tiles and parts, whether anything is kept or not
        assert torch.equal(H, kept)
