"""The gated layer and the 8-bit checkpoints in float64 (oracle; test infrastructure only), each from its definition
in include/fqt.h.  Formats, operands and random words are those of oracle/feedforward.py."""
import numpy as np

from . import feedforward as F
from . import philox

KEPT = 32


def kept(x):
    """Checkpoint of x [rows, cols]: dict(q=code bytes [rows, padded cols], exp=scale bytes [rows, blocks],
    value=float64 [rows, cols])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // KEPT)
    wide = np.zeros((rows, nb * KEPT))
    wide[:, :cols] = x
    bad = ~np.isfinite(wide).reshape(rows, nb, KEPT).all(2)
    top = np.where(np.isfinite(wide), np.abs(wide), 0.0).reshape(rows, nb, KEPT).max(2)
    E = F.block_exponent(top)
    scale, wb = np.repeat(2.0 ** E, KEPT, axis=1), np.repeat(bad, KEPT, axis=1)
    q = np.where(wb, 0x7F, F.encode(np.where(wb, 0.0, wide) / scale)).astype(np.uint8)
    exp = np.where(bad, 255, E + 127).astype(np.uint8)
    return dict(q=q, exp=exp, value=np.where(wb, np.nan, F.decode(q) * scale)[:, :cols])


def kept_values(q, exp, cols):
    """float64 values of a checkpoint's bytes."""
    scale = np.where(exp == 255, np.nan, 2.0 ** (exp.astype(np.float64) - 127))
    return (F.decode(q) * np.repeat(scale, KEPT, axis=1))[:, :cols]


def sigmoid(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z))


def activation(a, act):
    """(value, derivative) at a."""
    a = np.asarray(a, np.float64)
    if act == "relu":
        return np.maximum(a, 0.0), (a > 0).astype(np.float64)
    if act == "silu":
        s = sigmoid(a)
        return a * s, s + a * s * (1.0 - s)
    u = np.sqrt(2.0 / np.pi) * (a + 0.044715 * a ** 3)
    du = np.sqrt(2.0 / np.pi) * (1.0 + 3.0 * 0.044715 * a ** 2)
    s = sigmoid(2.0 * u)
    return a * s, s + a * s * (1.0 - s) * 2.0 * du


def gated_forward(x, w, act):
    """dict(a, b, H, d_gate, d_up) in float64 from Q(x) and the codes of w = [W_gate; W_up] in 128 x 128 tiles."""
    both = F.operand(x)["value"] @ F.operand(w, tile=True)["value"].T
    h = both.shape[1] // 2
    a, b = both[:, :h], both[:, h:]
    value, slope = activation(a, act)
    return dict(a=a, b=b, H=value * b, d_gate=b * slope, d_up=value)


def gradient_operands(g, d_gate, d_up, seed=None):
    """(operand of D^T, operand of D), D = [g d_gate | g d_up] rounded to float32; seed None: to nearest."""
    with np.errstate(invalid="ignore", over="ignore"):
        D = np.concatenate([g * d_gate, g * d_up], axis=1).astype(np.float32).astype(np.float64)
    if seed is None:
        return F.operand(D.T), F.operand(D)
    w = philox.draws(np.arange(D.size, dtype=np.uint64), seed, 2).reshape(D.shape)
    low, high = (v.astype(np.float64) for v in (w & np.uint64(0xFFFF), w >> np.uint64(16)))
    return stochastic_operand(D.T, low.T), stochastic_operand(D, high)


def stochastic_operand(x, u):
    """F.operand with 16-bit uniforms: up iff 2^4 u < floor(frac 2^20), which is frac 2^24 >= 2^8 u + 16; F.encode's rule is
    a strict inequality, so its uniform is the number below that bound."""
    return F.operand(x, u=np.nextafter(256.0 * u + 16.0, 0.0))


def gated_backward(g, d_gate, d_up, x, w, seed=None):
    """(grad_w, grad_x) in float64; d_gate and d_up as kept, x and w quantized as the layer does."""
    g1, g2 = gradient_operands(g, d_gate, d_up, seed)
    return g1["value"] @ F.operand(x.T)["value"].T, g2["value"] @ F.operand(w.T, tile=True)["value"].T


def layernorm_backward8(g, xh, rstd, gamma=None):
    """(grad_x, grad_gamma, grad_beta) in float64 from xh as kept."""
    g, xh = np.asarray(g, np.float64), np.asarray(xh, np.float64)
    c = g if gamma is None else g * np.asarray(gamma, np.float64)
    gx = np.asarray(rstd, np.float64)[:, None] * (c - c.mean(1, keepdims=True) - xh * (c * xh).mean(1, keepdims=True))
    return gx, (g * xh).sum(0), g.sum(0)
