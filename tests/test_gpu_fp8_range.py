"""Products of 8-bit matrices whose scale bytes lie at the ends of their range, 1 to 254, against float64.

A float32 result is a float32 sum of exact products whatever the scales; a bfloat16 result is one of the 8-bit matrix
unit's.  The bounds are those of the products with ordinary scales; values below float32's least step cannot be held
and are kept out of the sums by the choice of the other operand's scales."""
import numpy as np
import pytest

from oracle import operators_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2410_05985_amd import layup as LU  # noqa: E402
from tests.test_gpu_operators import BF16, DEV, EPS, F32, FP8, TILES, U, f64, near, product_bound, quantised, tile_call, values  # noqa: E402


def operand(rng, rows, K, fmt, first, last):
    """Values over the format's whole range, its least and largest among them, and a scale byte of first .. last for
    each row and block."""
    kp, nb = -(-K // 128) * 128, -(-K // 128)
    top = R.TOPS[fmt][0]
    v = rng.normal(size=(rows, kp)) * np.exp2(rng.integers(-6, top - 2, size=(rows, kp)))
    v = np.clip(v, -1.75 * 2.0 ** top, 1.75 * 2.0 ** top)
    v[:, ::7] = 2.0 ** (-9 if fmt == "e4m3" else -16)
    v[:, 3::11] = -1.75 * 2.0 ** top
    v[:, K:] = 0
    q = torch.from_numpy(v).float().to(FP8[fmt]).to(DEV)
    e = np.full((rows, -(-nb // 4) * 4), 0x55, np.uint8)
    e[:, :nb] = rng.integers(first, last + 1, size=(rows, nb))
    return q, torch.from_numpy(e).to(DEV)


def check(M, N, K, fa, fb, a_bytes, b_bytes, out, cfg=-1, splits=1, bias=False):
    rng = np.random.default_rng(M + N + K + a_bytes[0])
    (qa, ea), (qb, eb) = operand(rng, M, K, fa, *a_bytes), operand(rng, N, K, fb, *b_bytes)
    c = torch.full((M + 1, N), 7.0, dtype=out, device=DEV)
    b = torch.from_numpy(rng.normal(size=N)).float().to(DEV) if bias else None
    ws = torch.empty(splits * M * N * 4, dtype=torch.uint8, device=DEV) if splits > 1 else None
    desc = LU.gemm_fp8_desc(qa, ea, 1, qb, eb, 1, c[:M], K, bias=b, workspace=ws)
    if cfg < 0:
        LU.layup_gemm_fp8(desc, torch.cuda.current_stream())
    else:
        tile_call(desc, cfg, splits)
    torch.cuda.synchronize()
    va, vb = values(qa, ea, K, 1), values(qb, eb, K, 1)
    ref = va @ vb.T + (f64(b) if bias else 0.0)
    tol = product_bound(va, vb, out) + U * (np.abs(ref) + (np.abs(f64(b)) if bias else 0.0))
    near(f64(c[:M]), ref, tol + EPS[out] * (np.abs(ref) + tol), "product")
    assert bool((c[M] == 7.0).all())


# bytes of A at an end, of B so that the products are ordinary float32 numbers
ENDS = [("e4m3", (1, 12), (200, 210)), ("e5m2", (1, 20), (200, 210)), ("e4m3", (240, 254), (20, 30)), ("e5m2", (236, 254), (20, 30)),
        ("e5m2", (9, 9), (190, 190)), ("e4m3", (2, 2), (190, 190))]


@pytest.mark.parametrize("fmt,a_bytes,b_bytes", ENDS)
@pytest.mark.parametrize("M,N,K", [(1, 40, 128), (5, 33, 700), (32, 20, 2304), (70, 40, 256), (260, 300, 1100)])
@pytest.mark.parametrize("out", [F32, BF16])
def test_product_with_scales_at_the_ends(fmt, a_bytes, b_bytes, M, N, K, out):
    check(M, N, K, fmt, "e4m3", a_bytes, b_bytes, out, bias=out == F32)
    check(M, N, K, "e4m3", fmt, b_bytes, a_bytes, out)


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("K,splits", [(128, 1), (1100, 1), (4500, 1), (2048, 3)])
def test_every_tile_with_scales_at_the_ends(tile, K, splits):
    for fmt, a_bytes, b_bytes in ENDS[:4]:
        check(270, 300, K, fmt, "e5m2", a_bytes, b_bytes, F32, cfg=TILES[tile], splits=splits, bias=True)


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("where", [0, 8, 33])
def test_one_such_block_among_ordinary_ones(tile, where):
    """A scale byte at the end in one row and one block of 128, early, late and in a second round of scales."""
    M, N, K = 300, 290, 34 * 128
    rng = np.random.default_rng(where)
    (qa, ea), (qb, eb) = operand(rng, M, K, "e5m2", 120, 130), operand(rng, N, K, "e4m3", 120, 130)
    for byte in (1, 245):
        e = ea.clone()
        e[211, where] = byte
        if byte == 245:  # B's part that meets it is small, so that nothing overflows
            eb[:, where] = 20
        c = torch.empty(M, N, device=DEV)
        tile_call(LU.gemm_fp8_desc(qa, e, 1, qb, eb, 1, c, K), TILES[tile], 1)
        torch.cuda.synchronize()
        va, vb = values(qa, e, K, 1), values(qb, eb, K, 1)
        near(f64(c), va @ vb.T, product_bound(va, vb, F32) + U * np.abs(va @ vb.T), byte)


@pytest.mark.parametrize("M", [5, 70])
@pytest.mark.parametrize("size", [2.0 ** -112, 2.0 ** -125, 2.0 ** 126])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantiser_then_product_of_tiny_and_huge_blocks(M, size, fmt):
    """What the quantiser makes of tiny and of huge blocks is a product's operand like any other."""
    rng = np.random.default_rng(M)
    K, N = 300, 40
    a = torch.from_numpy(rng.uniform(-1, 1, size=(M, K)) * size).float().to(DEV)
    b = torch.from_numpy(rng.normal(size=(N, K)) / size).float().to(DEV)
    pairs = []
    for x in (a, b):
        q = torch.zeros(x.shape[0], 384, dtype=torch.uint8, device=DEV).view(FP8[fmt])
        e = torch.zeros(x.shape[0], 4, dtype=torch.uint8, device=DEV)
        LU.layup_quant_fp8(LU.quant_desc(x, 1, q=q, scale=e), torch.cuda.current_stream())
        pairs.append((q, e))
    (qa, ea), (qb, eb) = pairs
    c = torch.empty(M, N, device=DEV)
    LU.layup_gemm_fp8(LU.gemm_fp8_desc(qa, ea, 1, qb, eb, 1, c, K), torch.cuda.current_stream())
    torch.cuda.synchronize()
    va, vb = values(qa, ea, K, 1), values(qb, eb, K, 1)
    near(f64(c), va @ vb.T, product_bound(va, vb, F32) + U * np.abs(va @ vb.T), "product")


@pytest.mark.parametrize("M", [3, 70, 300])
@pytest.mark.parametrize("K", [384, 4500])
@pytest.mark.parametrize("signs", [True, False])
@pytest.mark.parametrize("out", [F32, BF16])
def test_sums_that_cancel(M, K, signs, out):
    """The bias takes the product away, so that the result is the sum's error alone: within the bound of the matrix
    unit's sums for a bfloat16 C, of float32 sums for a float32 C."""
    rng = np.random.default_rng(K)
    N = 130
    row, b = rng.normal(size=(1, K)), rng.normal(size=(N, K))
    if not signs:
        row, b = np.abs(row), np.abs(b)
    (qa, ea), (qb, eb) = (quantised(torch.from_numpy(x).float().to(DEV), 1, "e4m3") for x in (np.repeat(row, M, 0), b))
    va, vb = values(qa, ea, K, 1), values(qb, eb, K, 1)
    bias = torch.from_numpy(-(vb @ va[0])).float().to(DEV)
    c = torch.empty(M, N, dtype=out, device=DEV)
    LU.layup_gemm_fp8(LU.gemm_fp8_desc(qa, ea, 1, qb, eb, 1, c, K, bias=bias), torch.cuda.current_stream())
    torch.cuda.synchronize()
    ref = va @ vb.T + f64(bias)
    tol = product_bound(va, vb, out) + U * (np.abs(ref) + np.abs(f64(bias)))
    near(f64(c), ref, tol + EPS[out] * (np.abs(ref) + tol), "product")
