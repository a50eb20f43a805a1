"""Every form of the 8-bit floating point products on sizes that take it, as the library says for each (so that another
rule of choice cannot empty these tests).

Exact: integers up to 8 have partial sums below 2^24, so a float32 sum in any order is the integer, and the output is it
rounded once, whatever the type.  Random operands: |error| <= K 2^-24 sum |a b| and half a unit in the last place."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402

gpu = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}

FORMS = {
    "rows": [(1, 4096, 1024), (16, 33, 16389), (17, 300, 500), (33, 70, 2000), (64, 129, 4097)],
    "small": [(100, 300, 500), (129, 255, 257), (2048, 2048, 640), (512, 4096, 999)],
    "parts": [(65, 129, 9000), (250, 1001, 2048), (1000, 700, 4999)],
    "middle": [(4352, 4096, 512), (8185, 1022, 200), (8192, 1024, 2049), (8448, 4096, 1000)],
    "large": [(3840, 4096, 512), (3870, 4090, 1100), (8000, 8192, 600), (16896, 4096, 513), (4096, 4096, 127)],
    # 512 tiles (two a block) and the fewest stages; 400 (one or two); 1056 (four or five); rows that end inside a tile
    "several": [(8192, 4096, 512), (5120, 5120, 1024), (16896, 4096, 512), (16896, 4096, 1000), (8000, 4096, 1000),
                (12033, 4096, 999)],
}
CASES = [(form, *s) for form, shapes in FORMS.items() for s in shapes]
SEVERAL = FORMS["several"]


def lines(N, dtype):
    return N * dtype.itemsize % 128 == 0


@pytest.mark.skipif(not os.path.exists(fqt.LIB_PATH), reason="libfqt.so not built")
def test_the_sizes_take_their_forms():
    for form, M, N, K in CASES:
        assert fqt.fqt_fp8_gemm_form(M, N, K) == form, (form, M, N, K)
    for M, N, K in SEVERAL:
        assert fqt.fqt_fp8_gemm_form(M, N, K, masked=True) == "large"
        assert fqt.fqt_fp8_gemm_form(M, N, K, lines=False) == "large"
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, (1 << 23) + 1), (1 << 31, 1, 1)):
        with pytest.raises(ValueError):
            fqt.fqt_fp8_gemm_form(*bad)


def integers(seed, rows, K):
    gen = torch.Generator("cuda").manual_seed(seed)
    return torch.randint(-8, 9, (rows, K), device="cuda", generator=gen).float()


def random(seed, rows, K, tile=False):
    gen = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((rows, K), device="cuda", generator=gen)
    x *= torch.exp2(torch.randint(-3, 4, (rows, 1), device="cuda", generator=gen).float())
    return fqt.fqt_fp8_quantize(x, tile=tile)[0]


def value(a):
    e = a["exp"].transpose(0, 1).reshape(a["q"].shape[0], -1)[:, :a["q"].shape[1] // 128].double() - 127
    return (a["q"].double().view(a["q"].shape[0], -1, 128) * torch.exp2(e)[:, :, None]).flatten(1)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form,M,N,K", CASES)
def test_exact_on_small_integers(form, M, N, K, dtype):
    assert fqt.fqt_fp8_gemm_form(M, N, K) == form
    x, w = integers(M, M, K), integers(N + 1, N, K)
    w[:, -1] = torch.where(w[:, -1] == 0, 1.0, w[:, -1])  # the last code counts in every output
    x[:, -1] = torch.where(x[:, -1] == 0, 1.0, x[:, -1])
    C, _ = fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], fqt.fqt_fp8_quantize(w)[0], dtype=dtype)
    wt = w.double().t().contiguous()
    for r in range(0, M, 4096):
        want = x[r:r + 4096].double() @ wt
        assert torch.equal(C[r:r + 4096], want.float().to(dtype)), r


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SEVERAL)
def test_several_tiles_a_block(M, N, K, dtype):
    """Against float64; a ReLU; the same bits with a block for each tile (a mask that is positive throughout); an output
    with a pitch and rows behind it that stay as they were."""
    assert fqt.fqt_fp8_gemm_form(M, N, K) == "several" and lines(N, dtype) and lines(N + 128, dtype)
    A, B = random(M, M, K), random(N + 1, N, K, tile=True)
    C, _ = fqt.fqt_fp8_gemm(A, B, dtype=dtype)
    R, _ = fqt.fqt_fp8_gemm(A, B, dtype=dtype, relu=True)
    assert torch.equal(R, C.clamp(min=0))
    one, _ = fqt.fqt_fp8_gemm(A, B, dtype=dtype, mask=torch.ones((M, N), dtype=dtype, device="cuda"))
    assert torch.equal(one, C)
    wide = torch.full((M + 260, N + 128), 7.0, dtype=dtype, device="cuda")
    fqt.fqt_fp8_gemm(A, B, C=wide[:M, 64:N + 64])
    assert torch.equal(wide[:M, 64:N + 64], C)
    wide[:M, 64:N + 64] = 7.0
    assert (wide == 7.0).all()
    b = value(B)
    bt, bat = b.t().contiguous(), b.abs().t().contiguous()
    for r in range(0, M, 2048):
        a = value(dict(q=A["q"][r:r + 2048], exp=A["exp"][:, r:r + 2048]))
        want, size = a @ bt, a.abs() @ bat
        tol = K * 2.0 ** -24 * size + HALF[dtype] * want.abs()
        assert ((C[r:r + 2048].double() - want).abs() <= tol).all(), r


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_nan_rows_reach_their_outputs_only(dtype):
    M, N, K = 16896, 4096, 512
    assert fqt.fqt_fp8_gemm_form(M, N, K) == "several"
    x = torch.randn((M, K), device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    B = random(6, N, K, tile=True)
    C0, _ = fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], B, dtype=dtype)
    bad = torch.tensor([0, 255, 256, 4095, 8191, 16895], device="cuda")
    x[bad, 77] = float("nan")
    C1, _ = fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], B, dtype=dtype, relu=True)
    assert torch.isnan(C1[bad]).all()
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert torch.equal(C1[keep], C0[keep].clamp(min=0))


@gpu
@pytest.mark.parametrize("form,M,N,K,dtype", [("rows", 40, 130, 384, torch.float16), ("small", 1024, 1024, 512, torch.bfloat16),
                                              ("parts", 130, 260, 4096, torch.float32), ("middle", 4352, 4096, 512, torch.bfloat16),
                                              ("large", 3840, 4096, 512, torch.float16),
                                              ("several", 8192, 4096, 512, torch.bfloat16),
                                              ("several", 5120, 5120, 1024, torch.float32)])
def test_replays_of_a_graph(form, M, N, K, dtype):
    from tests.test_gpu_train_graphs import replays
    assert fqt.fqt_fp8_gemm_form(M, N, K) == form
    x, w = torch.zeros((M, K), device="cuda"), torch.zeros((N, K), device="cuda")

    def make():
        return [fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], fqt.fqt_fp8_quantize(w, tile=True)[0], dtype=dtype)[0]]

    replays(make, [x, w])
