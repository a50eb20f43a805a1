"""Pins of the float64 oracle of the gated layer and the 8-bit checkpoints: the activations against torch's and their
derivatives against differences, the backward's formula against autograd, checkpoints against the operands' quantizer,
half-word stochastic rounding's mean and independence, the norm's gradient from an exact checkpoint."""
import numpy as np
import pytest

from oracle import feedforward as F
from oracle import gated as G

torch = pytest.importorskip("torch")

ACTS = {"silu": torch.nn.functional.silu, "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh"),
        "relu": torch.relu}


@pytest.mark.parametrize("act", list(ACTS))
def test_activations(act):
    a = np.concatenate([np.linspace(-12, 12, 241), [0.0, -0.0, 1e-8, -30.0, 40.0]])
    value, slope = G.activation(a, act)
    t = torch.from_numpy(a).requires_grad_()
    y = ACTS[act](t)
    y.sum().backward()
    np.testing.assert_allclose(value, y.detach().numpy(), rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(slope, t.grad.numpy(), rtol=1e-11, atol=1e-13)
    h = 1e-6
    away = np.abs(a) > 1e-3
    num = (G.activation(a + h, act)[0] - G.activation(a - h, act)[0]) / (2 * h)
    assert np.abs(num - slope)[away].max() < 1e-8


@pytest.mark.parametrize("act", list(ACTS))
def test_the_backward_is_the_gradient(act):
    """Without rounding: D from the derivatives, and both products, against autograd."""
    rng = np.random.default_rng(1)
    x, w, g = rng.standard_normal((7, 11)), rng.standard_normal((10, 11)), rng.standard_normal((7, 5))
    a, b = x @ w[:5].T, x @ w[5:].T
    value, slope = G.activation(a, act)
    D = np.concatenate([g * b * slope, g * value], axis=1)
    tx, tw = (torch.from_numpy(v.copy()).requires_grad_() for v in (x, w))
    both = tx @ tw.t()
    (ACTS[act](both[:, :5]) * both[:, 5:]).backward(torch.from_numpy(g))
    np.testing.assert_allclose(D.T @ x, tw.grad.numpy(), rtol=1e-10, atol=1e-11)
    np.testing.assert_allclose(D @ w, tx.grad.numpy(), rtol=1e-10, atol=1e-11)


def test_checkpoints_are_blocks_of_32():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((6, 70)) * np.exp(rng.normal(0, 3, (6, 70)))
    x[2, 40], x[3] = np.inf, 0.0
    k = G.kept(x)
    assert k["q"].shape == (6, 96) and k["exp"].shape == (6, 3) and (k["q"][:, 70:][k["exp"][:, 2] != 255] == 0).all()
    for b in range(3):
        part = np.where(np.isfinite(x[:, 32 * b:32 * b + 32]), x[:, 32 * b:32 * b + 32], np.inf)
        o = F.operand(part)  # the same block alone in a block of 128
        np.testing.assert_array_equal(k["exp"][:, b], o["exp"][0, :, 0])
        np.testing.assert_array_equal(k["value"][:, 32 * b:32 * b + 32], o["value"])
    np.testing.assert_array_equal(G.kept_values(k["q"], k["exp"], 70), k["value"])
    assert k["exp"][2, 1] == 255 and (k["exp"][3] == 127).all() and np.isnan(k["value"][2, 32:64]).all()


def test_half_word_rounding_is_unbiased_and_independent():
    """4000 seeds of four elements: means within five deviations (half a step at most, and 2^-16 of a step for a
    16-bit uniform); the two roundings of an element are uncorrelated."""
    g, one = np.array([[0.3, 1.03, -5.7, 400.1]]), np.ones((1, 4))
    n = 4000
    ups, downs = [], []
    for seed in range(n):
        t, r = G.gradient_operands(g, one, one, seed)
        ups.append(t["value"][:4, 0])
        downs.append(r["value"][0, :4])
    ups, downs = np.stack(ups), np.stack(downs)
    D = g[0].astype(np.float32).astype(np.float64)
    # by column: each element alone in its block, largest 256 .. 448 times a power of two: steps of 1/16 to 1/8
    for v in (ups, downs):
        step = np.array([np.diff(np.unique(v[:, j])).max(initial=0.0) for j in range(4)])
        assert np.all(np.abs(v.mean(0) - D) < (5 / 2 / np.sqrt(n) + 2.0 ** -16) * step + 1e-12)
    c = np.corrcoef(ups[:, 0], downs[:, 0])[0, 1]
    assert abs(c) < 5 / np.sqrt(n)


def test_half_word_rounding_rule():
    """Around the border, and where frac has more than 20 bits (results below the format's normal numbers)."""
    top = 448.0
    for frac, u, up in ((0.5, 32767, True), (0.5, 32768, False), (0.0, 0, False), (2.0 ** -20, 0, True),
                        (2.0 ** -21, 0, False), (2.0 ** -16, 1, False), (2.0 ** -16 + 2.0 ** -20, 1, True),
                        (1 - 2.0 ** -20, 65535, True), (1 - 2.0 ** -16, 65535, False)):
        for base, step in ((16.0, 2.0), (0.0, 2.0 ** -9), (3 * 2.0 ** -9, 2.0 ** -9)):
            x = np.zeros((1, 128))
            x[0, 0], x[0, 1] = top, base + frac * step
            got = G.stochastic_operand(x, np.full((1, 128), float(u)))["value"][0, 1]
            assert got == base + (step if up else 0.0), (frac, u, base)


def test_norm_gradient_from_an_exact_checkpoint():
    rng = np.random.default_rng(3)
    x, g, gamma = rng.standard_normal((5, 40)), rng.standard_normal((5, 40)), rng.standard_normal(40)
    xh, _, rstd = F.layernorm(x)
    for got, want in zip(G.layernorm_backward8(g, xh, rstd, gamma), F.layernorm_backward(g, x, gamma)):
        np.testing.assert_allclose(got, want, rtol=1e-12, atol=1e-13)


def test_quantization_noise_of_the_gradients():
    """Gradients through the codes against those without: relative noise of the operands (3 mantissa bits: 2.6 %
    nearest, 3.7 % stochastic), of the checkpoints (2.6 %) and of a and b themselves, within 10 %."""
    rng = np.random.default_rng(4)
    x, w, g = rng.standard_normal((256, 96)), rng.standard_normal((128, 96)) / 96 ** 0.5, rng.standard_normal((256, 64))
    f = G.gated_forward(x, w, "silu")
    gw, gx = G.gated_backward(g, G.kept(f["d_gate"])["value"], G.kept(f["d_up"])["value"], x, w, seed=9)
    a, b = x @ w[:64].T, x @ w[64:].T
    value, slope = G.activation(a, "silu")
    D = np.concatenate([g * b * slope, g * value], axis=1)
    for got, want in ((gw, D.T @ x), (gx, D @ w)):
        assert np.linalg.norm(got - want) < 0.1 * np.linalg.norm(want)
