"""The floating-point operators around the layers, in float64 (oracle; test infrastructure only).

Layer norm and its gradient, the 8-bit floating point block quantizer, the products of its operands, and the
global gradient norm with clipping, each from its definition in include/fqt.h.

The 8-bit format (4 exponent bits with bias 7, 3 mantissa bits, no infinity, one NaN) is taken as the sorted list
of its 127 magnitudes; rounding is a search in that list.
"""
import numpy as np

from . import philox

BLOCK = 128


# ---------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------
def layernorm(x, gamma=None, beta=None, eps=1e-5):
    """(y, mean, rstd) over the columns of x, float64."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return y, mean, rstd


def layernorm_backward(g, x, gamma=None, eps=1e-5):
    """(grad_x, grad_gamma, grad_beta), float64."""
    g = np.asarray(g, np.float64)
    xh, _, rstd = layernorm(x, eps=eps)
    c = g if gamma is None else g * np.asarray(gamma, np.float64)
    gx = rstd[:, None] * (c - c.mean(1, keepdims=True) - xh * (c * xh).mean(1, keepdims=True))
    return gx, (g * xh).sum(0), g.sum(0)


# ---------------------------------------------------------------------------
# 8-bit floating point
# ---------------------------------------------------------------------------
def magnitudes():
    """The 127 finite magnitudes of the format, code order: 0, 2^-9 .. 448."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * 2.0 ** (e.astype(np.float64) - 7.0))


def decode(q):
    """Values of code bytes (0x7F and 0xFF are NaN)."""
    q = np.asarray(q, np.uint8)
    mag = np.append(magnitudes(), np.nan)[q & 0x7F]
    return np.where(q & 0x80, -mag, mag)


def encode(y, u=None):
    """Code bytes of y, |y| <= 448: nearest (ties to the even code), or with 24-bit uniforms u up iff
    u < frac 2^24, frac the position of |y| between its two neighbours."""
    y = np.asarray(y, np.float64)
    mag, a = magnitudes(), np.abs(y)
    assert np.all(a <= 448.0)
    lo = np.searchsorted(mag, a, side="right") - 1
    hi = np.minimum(lo + 1, 126)
    gap = np.where(hi > lo, mag[hi] - mag[lo], 1.0)
    frac = (a - mag[lo]) / gap
    if u is None:
        up = (frac > 0.5) | ((frac == 0.5) & (lo % 2 == 1))
    else:
        up = u < frac * 2.0 ** 24
    code = np.where(up, hi, lo).astype(np.uint8)
    return code | (np.signbit(y).astype(np.uint8) << 7)


def block_exponent(top):
    """The least integer E >= -127 with top <= 448 2^E (0 for an empty block), by trying every one."""
    top = np.asarray(top, np.float64)
    e = np.full(top.shape, 128)
    for k in range(127, -128, -1):
        e = np.where(top <= 448.0 * 2.0 ** k, k, e)
    return np.where(top > 0, e, 0)


def uniforms(rows, cols, seed, stream):
    """The 24-bit uniform of every element of a [rows, cols] matrix."""
    e = np.arange(rows * cols, dtype=np.uint64)
    return (philox.draws(e, seed, stream) & np.uint64(0xFFFFFF)).astype(np.float64).reshape(rows, cols)


def operand(x, tile=False, u=None):
    """Operand of x [rows, K]: dict(q=code bytes [rows, padded K], exp=scale bytes [blocks / 4, rows, 4],
    value=float64 [rows, K])."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    kb = -(-K // BLOCK)
    wide = np.zeros((rows, kb * BLOCK))
    wide[:, :K] = x
    bad = ~np.isfinite(wide).reshape(rows, kb, BLOCK).all(2)
    top = np.where(np.isfinite(wide), np.abs(wide), 0.0).reshape(rows, kb, BLOCK).max(2)
    if tile:
        for r in range(0, rows, BLOCK):
            top[r:r + BLOCK] = top[r:r + BLOCK].max(0)
            bad[r:r + BLOCK] = bad[r:r + BLOCK].any(0)
    E = block_exponent(top)
    scale = np.repeat(2.0 ** E, BLOCK, axis=1)
    wb = np.repeat(bad, BLOCK, axis=1)
    uu = None
    if u is not None:
        uu = np.zeros_like(wide)
        uu[:, :K] = u
    q = encode(np.where(wb, 0.0, wide) / scale, uu)
    q = np.where(wb, 0x7F, q).astype(np.uint8)
    exp = np.full((rows, -(-kb // 4) * 4), 127, np.uint8)
    exp[:, :kb] = np.where(bad, 255, E + 127)
    value = np.where(wb, np.nan, decode(q) * scale)[:, :K]
    return dict(q=q, exp=exp.reshape(rows, -1, 4).transpose(1, 0, 2).copy(), value=value)


def linear_forward(x, w, relu=False):
    """Q(x) Q(w)^T with the weights in 128 x 128 tiles, float64."""
    y = operand(x)["value"] @ operand(w, tile=True)["value"].T
    return np.maximum(y, 0.0) if relu else y


def linear_backward(g, x, w, seed, stochastic=True, relu_input=None):
    """(grad_w, grad_x): Q_b1(g)^T Q(x) and Q_b2(g) Q(w), float64."""
    rows, cols = g.shape
    u1, u2 = (uniforms(rows, cols, seed, s) if stochastic else None for s in (0, 1))
    g1 = operand(g.T, u=None if u1 is None else u1.T)["value"]
    g2 = operand(g, u=u2)["value"]
    gx = g2 @ operand(w.T, tile=True)["value"].T
    if relu_input is not None:
        gx = np.where(np.asarray(relu_input) > 0, gx, 0.0)
    return g1 @ operand(x.T)["value"].T, gx


# ---------------------------------------------------------------------------
# gradient norm and clipping
# ---------------------------------------------------------------------------
def clip(grads, max_norm):
    """(norm, scaled gradients), float64; a norm that is not finite scales nothing."""
    g = [np.asarray(t, np.float64) for t in grads]
    n = float(np.sqrt(sum(float((t * t).sum()) for t in g)))
    scale = max_norm / n if np.isfinite(n) and n > max_norm else 1.0
    return n, [t * scale for t in g]
