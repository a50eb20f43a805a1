"""Pins of the float64 oracle of the operators around the layers: the 8-bit format against torch's type, the block
exponent's defining inequality, stochastic rounding's mean, the layer norm gradient against autograd and against
differences, clipping's invariants."""
import numpy as np
import pytest

from oracle import feedforward as F

torch = pytest.importorskip("torch")


def test_format_matches_torch_for_every_code():
    q = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(q.copy()).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(F.decode(q), want)


def test_nearest_rounding_matches_torch():
    rng = np.random.default_rng(0)
    m = F.magnitudes()
    y = np.concatenate([m, -m, (m[1:] + m[:-1]) / 2, rng.uniform(-448, 448, 4000), rng.normal(0, 2.0 ** -7, 4000)])
    y = y.astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(F.encode(y), want)


def test_block_exponent_is_the_least():
    rng = np.random.default_rng(1)
    top = np.concatenate([np.exp(rng.uniform(-87, 88, 500)), 448.0 * 2.0 ** np.arange(-20, 20), [0.0, 1e-45, 3.4e38]])
    E = F.block_exponent(top)
    assert np.all(top <= 448.0 * 2.0 ** E)
    assert np.all((E == -127) | (top == 0) | (top > 448.0 * 2.0 ** (E - 1.0)))


def test_stochastic_codes_are_unbiased():
    y = np.array([0.3, 1.03, -5.7, 400.1, 2.0 ** -9 * 0.25, 448.0, -0.0])
    rng = np.random.default_rng(2)
    n = 40000
    d = np.stack([F.decode(F.encode(y, rng.integers(0, 1 << 24, y.size))) for _ in range(n)])
    step = np.array([2.0 ** -5, 2.0 ** -3, 0.5, 32.0, 2.0 ** -9, 32.0, 2.0 ** -9])
    assert np.all(np.abs(d.mean(0) - y) < 5 * step / 2 / np.sqrt(n) + 1e-12)


def test_operand_layout():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 700)) * np.exp(rng.normal(0, 3, (5, 1)))
    a = F.operand(x)
    assert a["q"].shape == (5, 768) and a["exp"].shape == (2, 5, 4)
    assert (a["q"][:, 700:] == 0).all() and (a["exp"][1, :, 2:] == 127).all()
    E = a["exp"].transpose(1, 0, 2).reshape(5, 8)[:, :6].astype(int) - 127
    back = F.decode(a["q"]) * np.repeat(2.0 ** E, 128, axis=1)
    np.testing.assert_array_equal(back[:, :700], a["value"])
    assert np.abs(a["value"] - x).max() <= np.abs(x).max() * 2.0 ** -4


def test_layernorm_gradient_against_autograd_and_differences():
    rng = np.random.default_rng(4)
    x, g = rng.standard_normal((4, 37)) * 3 + 1, rng.standard_normal((4, 37))
    gamma, beta = rng.standard_normal(37), rng.standard_normal(37)
    t = [torch.from_numpy(v.copy()).requires_grad_() for v in (x, gamma, beta)]
    y = torch.nn.functional.layer_norm(t[0], (37,), t[1], t[2], 1e-5)
    np.testing.assert_allclose(F.layernorm(x, gamma, beta)[0], y.detach().numpy(), rtol=1e-12, atol=1e-12)
    y.backward(torch.from_numpy(g))
    gx, gg, gb = F.layernorm_backward(g, x, gamma)
    for got, v in ((gx, t[0]), (gg, t[1]), (gb, t[2])):
        np.testing.assert_allclose(got, v.grad.numpy(), rtol=1e-10, atol=1e-11)
    h = 1e-5
    for i, j in ((0, 0), (2, 36), (3, 17)):
        d = np.zeros_like(x)
        d[i, j] = h
        num = ((F.layernorm(x + d, gamma, beta)[0] - F.layernorm(x - d, gamma, beta)[0]) * g).sum() / (2 * h)
        assert abs(num - gx[i, j]) < 1e-7


def test_clip_invariants():
    rng = np.random.default_rng(5)
    g = [rng.standard_normal(n) for n in (1, 50, 700)]
    n, out = F.clip(g, 2.5)
    assert abs(n - np.linalg.norm(np.concatenate(g))) < 1e-12
    assert abs(np.linalg.norm(np.concatenate(out)) - 2.5) < 1e-12
    assert all((a == b).all() for a, b in zip(F.clip(g, 1e9)[1], g))
    g[1][3] = np.inf
    assert all((a == b).all() for a, b in zip(F.clip(g, 1.0)[1], g))
