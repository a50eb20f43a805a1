"""Products of more whole 256 x 256 tiles than compute units, whose blocks form several tiles each.  Tolerances as for the
other products: K 2^-24 of the sum of |a b| for the accumulation, 2^-12 for what the 8-bit instructions drop, and half a
unit in the last place of the output."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2010_14298_amd import fqt  # noqa: E402

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def operand(seed, rows, K, tile=False):
    gen = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((rows, K), device="cuda", generator=gen)
    x *= torch.exp2(torch.randint(-3, 4, (rows, 1), device="cuda", generator=gen).float())
    return fqt.fqt_fp8_quantize(x, tile=tile)[0]


def value(a):
    e = a["exp"].transpose(0, 1).reshape(a["q"].shape[0], -1)[:, :a["q"].shape[1] // 128].double() - 127
    return (a["q"].double().view(a["q"].shape[0], -1, 128) * torch.exp2(e)[:, :, None]).flatten(1)


def rows_of(a, r0, r1):
    return dict(q=a["q"][r0:r1], exp=a["exp"][:, r0:r1].contiguous(), K=a["K"])


# four stages (the fewest) and more; an end inside a block; 272 tiles (some blocks with one) to 1056 (four or five)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K", [(4352, 4096, 512), (8448, 4096, 1000), (16640, 1024, 1250), (16896, 4096, 513)])
def test_against_float64(M, N, K, dtype):
    A, B = operand(M, M, K), operand(N, N, K, tile=True)
    C, _ = fqt.fqt_fp8_gemm(A, B, dtype=dtype)
    R, _ = fqt.fqt_fp8_gemm(A, B, dtype=dtype, relu=True)
    assert torch.equal(R, C.clamp(min=0))
    b = value(B)
    bt, bat = b.t().contiguous(), b.abs().t().contiguous()
    for r in range(0, M, 2048):
        a = value(rows_of(A, r, min(r + 2048, M)))
        want, size = a @ bt, a.abs() @ bat
        tol = (K * 2.0 ** -24 + 2.0 ** -12) * size + HALF[dtype] * want.abs()
        assert ((C[r:r + 2048].double() - want).abs() <= tol).all(), r


@pytest.mark.parametrize("M,N,K", [(4352, 4096, 512), (8448, 4096, 1000)])
def test_same_bits_as_products_of_fewer_rows(M, N, K):
    """Runs of rows with fewer tiles than units take a block for each tile."""
    A, B = operand(1, M, K), operand(2, N, K, tile=True)
    C, _ = fqt.fqt_fp8_gemm(A, B, dtype=torch.bfloat16)
    for r in range(0, M, 3840):
        P, _ = fqt.fqt_fp8_gemm(rows_of(A, r, min(r + 3840, M)), B, dtype=torch.bfloat16)
        assert torch.equal(C[r:r + 3840], P), r


def test_output_with_a_pitch_keeps_its_surroundings():
    M, N, K = 4352, 4096, 640 + 384
    A, B = operand(3, M, K), operand(4, N, K, tile=True)
    C, _ = fqt.fqt_fp8_gemm(A, B, dtype=torch.bfloat16)
    wide = torch.full((M + 2, N + 128), 7.0, dtype=torch.bfloat16, device="cuda")
    fqt.fqt_fp8_gemm(A, B, C=wide[1:M + 1, 64:N + 64])
    assert torch.equal(wide[1:M + 1, 64:N + 64], C)
    wide[1:M + 1, 64:N + 64] = 7.0
    assert (wide == 7.0).all()


def test_nan_rows_reach_their_outputs_only():
    M, N, K = 8192, 4096, 512
    gen = torch.Generator("cuda").manual_seed(5)
    x = torch.randn((M, K), device="cuda", generator=gen)
    B = operand(6, N, K, tile=True)
    C0, _ = fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], B, dtype=torch.bfloat16)
    bad = torch.tensor([0, 255, 256, 4095, 8191], device="cuda")
    x[bad, 77] = float("nan")
    C1, _ = fqt.fqt_fp8_gemm(fqt.fqt_fp8_quantize(x)[0], B, dtype=torch.bfloat16, relu=False)
    assert torch.isnan(C1[bad]).all()
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert torch.equal(C1[keep], C0[keep])


@pytest.mark.parametrize("M", [4097, 8000, 8447])
def test_rows_that_end_inside_a_tile(M):
    """The same bits as the product of whole tiles, and nothing stored past the last row."""
    N, K = 4096, 768
    A, B = operand(7, 8448, K), operand(8, N, K, tile=True)
    C, _ = fqt.fqt_fp8_gemm(A, B, dtype=torch.bfloat16)
    wide = torch.full((M + 260, N), 7.0, dtype=torch.bfloat16, device="cuda")
    fqt.fqt_fp8_gemm(rows_of(A, 0, M), B, C=wide[:M])
    assert torch.equal(wide[:M], C[:M])
    assert (wide[M:] == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(4352, 4096, 512), (8000, 4096, 1000), (16640, 1024, 1250)])
def test_float32_against_float64(M, N, K):
    """float32 outputs: codes converted exactly, float32 accumulation in any order, no dropped terms."""
    A, B = operand(M + 1, M, K), operand(N + 1, N, K, tile=True)
    wide = torch.full((M + 260, N), 7.0, device="cuda")
    fqt.fqt_fp8_gemm(A, B, C=wide[:M])
    C = wide[:M]
    R, _ = fqt.fqt_fp8_gemm(A, B, relu=True)
    assert torch.equal(R, C.clamp(min=0)) and (wide[M:] == 7.0).all()
    b = value(B)
    bt, bat = b.t().contiguous(), b.abs().t().contiguous()
    for r in range(0, M, 2048):
        a = value(rows_of(A, r, min(r + 2048, M)))
        want, size = a @ bt, a.abs() @ bat
        tol = (K * 2.0 ** -24) * size + 2.0 ** -24 * want.abs()
        assert ((C[r:r + 2048].double() - want).abs() <= tol).all(), r
