"""Global gradient norm and clipping against the float64 oracle.

The norm: squares and sums in float64 (a relative error far below 2^-30), rounded once to float32.  A scaled element:
the factor rounded to float32, one product, the type's rounding."""
import numpy as np
import pytest

from oracle import feedforward as F

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def fqt():
    from paper_2010_14298_amd import fqt as f
    f.load()
    return f


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def draw(sizes, types, seed=0, size=1.0):
    rng = np.random.default_rng(seed)
    return [torch.from_numpy(rng.standard_normal(n) * size * np.exp(rng.normal(-2, 1))).to(t).cuda()
            for n, t in zip(sizes, types)]


def check(grads, outs, norm, max_norm):
    n, want = F.clip([host(t) for t in grads], max_norm)
    assert abs(float(norm) - n) <= 2.0 ** -23 * n
    for o, w in zip(outs, want):
        assert np.all(np.abs(host(o) - w) <= (2.0 ** -23 + HALF[o.dtype]) * np.abs(w) + TINY[o.dtype])


SETS = [[1], [0, 1, 0], [5, 3, 0, 16384, 16385, 16383], [100003], [7] * 96, [13] * 97, [1, 1000, 0, 31] * 75,
        [3000000, 17, 1 << 20], [7] * 168, [13] * 169, [1, 1000, 0, 31] * 175, [0, 0]]


@pytest.mark.parametrize("max_norm", [0.125, 1e9])
@pytest.mark.parametrize("k", range(len(SETS)))
def test_norm_and_scaling(k, max_norm):
    f = fqt()
    sizes = SETS[k]
    types = [TYPES[(i + k) % 3] for i in range(len(sizes))]
    grads = draw(sizes, types, seed=k)
    keep = [t.clone() for t in grads]
    outs = [torch.full_like(t, 9.0) for t in grads]
    norm, _ = f.fqt_grad_norm_clip(grads, max_norm, outs=outs)
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    check(keep, outs, norm, max_norm)
    norm2, _ = f.fqt_grad_norm_clip(grads, max_norm)  # in place
    assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(grads, outs))


def test_views_at_odd_offsets_keep_their_surroundings():
    f = fqt()
    flat = torch.randn(50000, device="cuda").bfloat16()
    out = torch.full_like(flat, 3.0)
    cuts = [(1, 8), (9, 20001), (20004, 20005), (20011, 49999)]
    g, o = [flat[a:b] for a, b in cuts], [out[a + 0:b] for a, b in cuts]
    norm, _ = f.fqt_grad_norm_clip(g, 1.0, outs=o)
    check(g, o, norm, 1.0)
    inside = torch.zeros(50000, dtype=torch.bool, device="cuda")
    for a, b in cuts:
        inside[a:b] = True
    assert (out[~inside] == 3).all()
    # outputs at another alignment than their gradients
    shifted = torch.full((50001,), 3.0, dtype=torch.bfloat16, device="cuda")
    f.fqt_grad_norm_clip(g, 1.0, outs=[shifted[a + 1:b + 1] for a, b in cuts])
    assert torch.equal(shifted[1:], out)


def test_squares_beyond_float32():
    """Elements whose squares pass float32's largest value, and ones whose squares vanish in it."""
    f = fqt()
    for size in (1e30, 1e-30):
        g = draw([1000, 77], [torch.float32, torch.bfloat16], seed=3, size=size)
        outs = [torch.empty_like(t) for t in g]
        norm, _ = f.fqt_grad_norm_clip(g, size / 8, outs=outs)
        check(g, outs, norm, size / 8)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_norm_scales_nothing(bad):
    f = fqt()
    g = draw([500, 600], [torch.float32, torch.float16], seed=4)
    g[1][33] = bad
    outs = [torch.empty_like(t) for t in g]
    norm, _ = f.fqt_grad_norm_clip(g, 1.0, outs=outs)
    assert not np.isfinite(float(norm))
    for a, b in zip(g, outs):
        assert torch.equal(a.nan_to_num(1e4, 1e4), b.nan_to_num(1e4, 1e4))


def test_norm_at_the_bound_and_norm_only():
    f = fqt()
    g = [torch.tensor([3.0, 4.0], device="cuda")]
    norm, _ = f.fqt_grad_norm_clip(g, 5.0)
    assert float(norm) == 5.0 and g[0].tolist() == [3.0, 4.0]
    norm, _ = f.fqt_grad_norm_clip(g, float("inf"))
    assert float(norm) == 5.0 and g[0].tolist() == [3.0, 4.0]
    norm, _ = f.fqt_grad_norm_clip([torch.zeros(100, device="cuda")], 1.0)
    assert float(norm) == 0.0


def test_same_result_twice_and_under_a_graph():
    f = fqt()
    g = draw([100000, 3, 77777], [torch.float32] * 3, seed=5)
    outs = [torch.empty_like(t) for t in g]
    ws = torch.empty(f.fqt_grad_norm_clip_workspace(3), dtype=torch.uint8, device="cuda")
    norm, _ = f.fqt_grad_norm_clip(g, 1.0, outs=outs, ws=ws)
    first = [norm.clone()] + [t.clone() for t in outs]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        n2, _ = f.fqt_grad_norm_clip(g, 1.0, outs=outs, ws=ws)
    for k in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, [n2] + outs))


def test_refusals():
    f = fqt()
    t = torch.ones(10, device="cuda")
    for bad in (lambda: f.fqt_grad_norm_clip([t.cpu()], 1.0), lambda: f.fqt_grad_norm_clip([t.double()], 1.0),
                lambda: f.fqt_grad_norm_clip([t[::2]], 1.0), lambda: f.fqt_grad_norm_clip([t], 1.0, outs=[t[:5]]),
                lambda: f.fqt_grad_norm_clip([t], 1.0, outs=[t.half()])):
        with pytest.raises(ValueError):
            bad()
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    for bad, code in ((lambda: f.fqt_grad_norm_clip([], 1.0), 1), (lambda: f.fqt_grad_norm_clip([t], 0.0), 1),
                      (lambda: f.fqt_grad_norm_clip([t], float("nan")), 1),
                      (lambda: f.fqt_grad_norm_clip([t], 1.0, ws=small), 4)):
        with pytest.raises(f.FqtError) as e:
            bad()
        assert e.value.code == code
