"""Every tensor argument of the floating-point operators' binding has to be on the current device: each in turn says that
it is on another one, and the call is refused before anything of it reaches the library.

Runs without a GPU: host tensors stand for the current device's (their device number is -1, and so the current one's)."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402

pytestmark = pytest.mark.skipif(not os.path.exists(fqt.LIB_PATH), reason="libfqt.so not built")

N, D, H = 12, 40, 24


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


def elsewhere(t):
    return t.as_subclass(Elsewhere)


def moved(args, path):
    """args with the tensor at path (keys, outermost first) on another device."""
    if not path:
        return elsewhere(args)
    return {**args, path[0]: moved(args[path[0]], path[1:])}


def operand(rows, K):
    return fqt.fp8_operand(rows, K, "cpu")


def calls():
    """name -> (function, its arguments, where their tensors are)."""
    x, g, h = torch.zeros((N, D)), torch.zeros((N, D)), torch.zeros((N, H))
    vec, rows, ws = torch.zeros(D), torch.zeros(N), torch.zeros(1 << 20, dtype=torch.uint8)
    kept = dict(X8t=operand(D, N), d_gate=fqt.fp8_kept(N, H, "cpu"), d_up=fqt.fp8_kept(N, H, "cpu"))
    of = [("q",), ("exp",)]
    return {
        "layernorm_forward8": (fqt.fqt_layernorm_forward8, dict(X=x, gamma=vec, beta=vec, Y=g),
                               [("X",), ("gamma",), ("beta",), ("Y",)]),
        "layernorm_backward8": (fqt.fqt_layernorm_backward8,
                                dict(G=g, xh8=fqt.fp8_kept(N, D, "cpu"), rstd=rows, gamma=vec, grad_X=x, ws=ws),
                                [("G",), ("rstd",), ("gamma",), ("grad_X",), ("ws",), *(("xh8",) + o for o in of)]),
        "gated_forward": (fqt.fqt_fp8_gated_forward, dict(X=x, W8=operand(2 * H, D), H=h, ws=ws),
                          [("X",), ("H",), ("ws",), *(("W8",) + o for o in of)]),
        "gated_backward": (fqt.fqt_fp8_gated_backward,
                           dict(G=h, kept=kept, W8t=operand(D, 2 * H), grad_W=torch.zeros((2 * H, D)), grad_X=x, ws=ws),
                           [("G",), ("grad_W",), ("grad_X",), ("ws",), *(("W8t",) + o for o in of),
                            *(("kept", n) + o for n in kept for o in of)]),
    }


CASES = [(name, path) for name, (_, _, paths) in calls().items() for path in paths]


@pytest.fixture
def library(monkeypatch):
    """Host tensors count as the current device's; what would reach the library is collected instead."""
    reached = []

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_workspace"):
                return lambda *a: 1 << 10
            return lambda *a: reached.append(name) or 0
    lib = Lib()
    monkeypatch.setattr(fqt, "_device", lambda: -1)
    monkeypatch.setattr(fqt, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(fqt, "load", lambda *a: lib)
    return reached


@pytest.mark.parametrize("name", list(calls()))
def test_all_on_the_current_device(name, library):
    f, args, _ = calls()[name]
    f(**args)
    assert library == [f.__name__]


@pytest.mark.parametrize("name,path", CASES)
def test_one_elsewhere_is_refused(name, path, library):
    f, args, _ = calls()[name]
    with pytest.raises(ValueError):
        f(**moved(args, path))
    assert library == []
