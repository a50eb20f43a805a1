"""The gated backward's quantizations of D = [G d_gate | G d_up] where there are 1536 tiles of 128 x 128 and more, in one
call for both gradients, bit for bit against the oracle.

A product of whole sums reads them out: operands of one-hot rows pick 256 tokens of D^T and 256 columns of D, whole
blocks of 128, among them the last ones and the one that lies across both halves.  A sum of one term is exact; grad_X
rounds it to its type once."""
import numpy as np
import pytest

from oracle import feedforward as F
from oracle import gated as G
from oracle import philox
from tests import test_gpu_gated as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HALF, TINY = base.HALF, base.TINY
SIZES = [(8192, 1600), (8190, 1541), (8100, 1540)]  # whole tiles; rows and hidden units off every tile, and off 4


def random_checkpoint(seed, rows, cols):
    """Codes of every kind, NaN's aside, and scales that leave products with a gradient inside float16; zero codes past
    cols."""
    rng = np.random.default_rng(seed)
    nb = -(-cols // 32)
    q = rng.integers(0, 256, (rows, nb * 32), dtype=np.uint8)
    q[(q & 0x7F) == 0x7F] = 0x3A
    q[:, cols:] = 0
    exp = rng.integers(105, 119, (rows, nb), dtype=np.uint8)
    kept = dict(q=torch.from_numpy(q).cuda().view(torch.float8_e4m3fn), exp=torch.from_numpy(exp).cuda(), cols=cols)
    return kept, lambda r: G.kept_values(q[r], exp[r], cols)


def picks(at, K):
    """The operand of 256 one-hot rows, row j at K's element at[j]."""
    one = torch.zeros((256, K), device="cuda")
    one[torch.arange(len(at)), torch.from_numpy(at)] = 1.0
    return base.fqt().fqt_fp8_quantize(one)[0]


def blocks(n, *first):
    return np.concatenate([np.arange(b * 128, min(b * 128 + 128, n)) for b in first])


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", base.TYPES)
@pytest.mark.parametrize("N,hidden", SIZES)
def test_codes_of_many_tiles(N, hidden, dtype, stochastic):
    f = base.fqt()
    cols, seed = 2 * hidden, (7 << 32) + 5
    assert -(-N // 128) * -(-cols // 128) >= 1536
    g = base.matrix(N, N, hidden, dtype, spread=2.0)
    g[N - 3], g[5] = 0.0, 0.0
    d_gate, gate = random_checkpoint(1, N, hidden)
    d_up, up = random_checkpoint(2, N, hidden)
    tokens = blocks(N, 37, (N - 1) // 128)
    columns = blocks(cols, hidden // 128, (cols - 1) // 128)
    X8t, W8t = picks(tokens, N), picks(columns, cols)
    how = dict(seed=seed, stochastic=stochastic)
    kept = dict(X8t=X8t, d_gate=d_gate, d_up=d_up)
    gW, gX, _ = f.fqt_fp8_gated_backward(g, kept, W8t, **how)

    gh = base.host(g)

    def D(rows):
        return np.concatenate([gh[rows] * gate(rows), gh[rows] * up(rows)], axis=1).astype(np.float32).astype(np.float64)

    def operand(x, rows, cs, transposed):
        if not stochastic:
            return F.operand(x.T if transposed else x)["value"]
        w = philox.draws((rows[:, None] * cols + cs[None, :]).astype(np.uint64), seed, 2).reshape(x.shape)
        u = (w & np.uint64(0xFFFF) if transposed else w >> np.uint64(16)).astype(np.float64)
        return G.stochastic_operand(x.T, u.T)["value"] if transposed else G.stochastic_operand(x, u)["value"]

    every = np.arange(cols)
    for first in range(0, len(tokens), 128):  # a block of K at a time: its elements share a scale
        rows = tokens[first:first + 128]
        want = operand(D(rows), rows, every, True)
        np.testing.assert_array_equal(base.host(gW)[:, first:first + len(rows)], want)
    rows = np.arange(N)
    whole = D(rows)
    for first in range(0, len(columns), 128):
        cs = columns[first:first + 128]
        want, got = operand(whole[:, cs], rows, cs, False), base.host(gX)[:, first:first + len(cs)]
        if dtype == torch.float32:
            np.testing.assert_array_equal(got, want)
        else:
            assert np.all(np.abs(got - want) <= HALF[dtype] * np.abs(want) + TINY[dtype])

    # kept operands that lie column by column are laid out in the quantizer's launch: the same bits
    def turned(o):
        return dict(q=o["q"].t().contiguous().t(), exp=o["exp"], K=o["K"])
    for x, w in ((turned(X8t), turned(W8t)), (X8t, turned(W8t)), (turned(X8t), W8t)):
        a, b, _ = f.fqt_fp8_gated_backward(g, dict(kept, X8t=x), w, **how)
        assert torch.equal(a, gW) and torch.equal(b, gX)
