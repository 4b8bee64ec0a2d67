"""Calls of the documented sizes that need more threads than one launch may have (2^32 along a dimension)."""
import numpy as np
import pytest

from oracle import operators_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2410_05985_amd import layup as LU  # noqa: E402
from tests.test_gpu_operators import BF16, DEV, F32, TILES, U, f64, near, quantised, tile_call  # noqa: E402


def test_norm_forward_of_more_rows_than_a_launch_takes():
    """32 threads a row: 2^27 rows are 2^32 threads.  The rows on both sides of that and the last ones."""
    rows, d, seed = (1 << 27) + 11, 2, 9
    x = torch.zeros(rows + 1, d, dtype=BF16, device=DEV)
    x[-1] = 7.0
    x[:rows].normal_()
    y, mean, rstd = (torch.full(s, float("nan"), dtype=t, device=DEV) for s, t in (((rows + 1, d), BF16), ((rows,), torch.float32), ((rows,), torch.float32)))
    LU.layup_layernorm_forward(LU.layernorm_desc(x[:rows], y[:rows], mean=mean, rstd=rstd, p=0.5, seed=seed), torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert bool(torch.isnan(y[rows]).all()) and not bool(torch.isnan(mean).any()) and not bool(torch.isnan(y[:rows]).any())
    for at in (0, (1 << 27) - 16, rows - 16):
        sl = slice(at, at + 16)
        s = f64(x[sl]) * R.keep_mask(16, d, 0.5, seed, 0, row0=at) * R.drop_scale(0.5)
        ref, m, q = R.norm_fwd(s, 1.0, 0.0, 1e-5)
        # the mean of two terms and a deviation from it are off by at most 2.5 U of the terms' magnitudes, which the
        # variance takes once more: 5 U times rstd, and a few roundings of y itself
        total = np.abs(s).sum(1)
        near(f64(mean[sl]), m, 2 * U * total, "mean")
        tol = (6 * U * total * q)[:, None] + 8 * U * np.abs(ref)
        near(f64(y[sl]), ref, tol + 2.0 ** -8 * (np.abs(ref) + tol), f"y at row {at}")
    del x, y, mean, rstd
    torch.cuda.empty_cache()


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantiser_of_more_columns_than_a_launch_takes(block_rows):
    """256 threads for 128 columns: 2^31 - 128 columns are as many as a launch takes.  One row of 100 more, its last
    blocks and some of the first."""
    cols = (1 << 31) - 28
    x = torch.empty(1, cols, dtype=BF16, device=DEV).normal_()
    q = torch.full((1, 1 << 31), 0x55, dtype=torch.uint8, device=DEV)
    e = torch.full((1, 1 << 24), 0x55, dtype=torch.uint8, device=DEV)
    LU.layup_quant_fp8(LU.quant_desc(x, block_rows, q=q.view(torch.float8_e4m3fn), scale=e), torch.cuda.current_stream())
    torch.cuda.synchronize()
    for at in (0, (1 << 31) - 512):
        n = min(512, cols - at)
        ref, eref = R.quantise(f64(x[:, at:at + n]), "e4m3", block_rows)
        assert np.array_equal(q[:, at:at + n].contiguous().view(torch.float8_e4m3fn).double().cpu().numpy(), ref), at
        assert np.array_equal(e[:, at // 128:at // 128 + 4].cpu().numpy(), eref), at
    assert not bool(q[:, cols:].any())
    del x, q, e
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cfg,M,N,splits", [(c, m, n, s) for c, m, n in ((0, 2600, 300), (1, 2600, 1100), (2, 300, 2200),
                                                                         (3, 1200, 1150), (3, 70, 1200)) for s in (1, 2)]
                         + [(4, 17, 300, 1)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_product_in_slices(cfg, M, N, splits, out):
    """A product whose tiles are too many for a launch: with room for the threads of sixteen tiles (a real launch's
    2^32 would take matrices of hundreds of gigabytes) the same bits as in one launch."""
    import ctypes
    K, rng = 1100, np.random.default_rng(M)
    a, b = (torch.from_numpy(rng.normal(size=(n, K))).float().to(DEV) for n in (M, N))
    (qa, ea), (qb, eb) = quantised(a, 128, "e4m3"), quantised(b, 128, "e5m2")
    bias = torch.from_numpy(rng.normal(size=N)).float().to(DEV)
    ws = torch.empty(splits * M * N * 4, dtype=torch.uint8, device=DEV)
    got = []
    for slices in (False, True):
        c = torch.full((M + 1, N + 3), 7.0, dtype=out, device=DEV)
        desc = LU.gemm_fp8_desc(qa, ea, 128, qb, eb, 128, c[:M, :N], K, bias=bias, workspace=ws)
        if slices:
            f = LU.lib().layup_test_gemm_fp8_slices
            f.argtypes, f.restype = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p], ctypes.c_int
            LU._check(f(ctypes.byref(desc), cfg, splits, 23 * (512 if cfg < 2 else 256 if cfg < 4 else 1024),
                        LU._stream(torch.cuda.current_stream())))
        else:
            tile_call(desc, cfg, splits)
        torch.cuda.synchronize()
        got.append(c)
    assert torch.equal(got[0], got[1])
    assert bool((got[0][M] == 7.0).all()) and bool((got[0][:, N:] == 7.0).all()) and not bool((got[0][:M, :N] == 7.0).all())


def test_product_of_one_row_with_more_columns_than_a_launch_takes():
    """64 threads for 16 columns: 2^30 columns are 2^32 threads.  B is 137 GB of zeros but for its last rows."""
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("less than 160 GiB free")
    cols, K = (1 << 30) + 45, 100
    q = torch.zeros(cols, 128, dtype=torch.uint8, device=DEV)
    e = torch.full((-(-cols // 128), 4), 127, dtype=torch.uint8, device=DEV)
    q[-45:, :K] = 0x38  # 1.0
    q[0, :K] = 0x40  # 2.0
    a = torch.zeros(1, 128, dtype=torch.uint8, device=DEV)
    a[:, :K] = 0x38
    ea = torch.full((1, 4), 127, dtype=torch.uint8, device=DEV)
    c = torch.full((1, cols), 7.0, dtype=BF16, device=DEV)
    f8 = torch.float8_e4m3fn
    LU.layup_gemm_fp8(LU.gemm_fp8_desc(a.view(f8), ea, 1, q.view(f8), e, 128, c, K), torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert c[0, 0] == 2 * K and bool((c[0, -45:] == K).all()) and not bool(c[0, 1:-45].any())
    del q, c
    torch.cuda.empty_cache()
