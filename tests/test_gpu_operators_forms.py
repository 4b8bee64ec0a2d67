"""Every kernel form that the calls can choose by rows, width and tiles, against the float64 reference: the LayerNorm's
teams of threads and groups a thread on both sides of each threshold, the quantiser's form for many tiles.  The list of
cases is held against the choice itself (no GPU needed for that)."""
import numpy as np
import pytest

from oracle import operators_ref as R

torch = pytest.importorskip("torch")
from paper_2410_05985_amd import layup as LU  # noqa: E402
from tests.test_gpu_operators import BF16, DEV, F32, FP8, backward, f64, forward, matrix, room8, scale_room, whole  # noqa: E402

WIDE = [256, 300, 504, 505, 601, 640, 768, 1000, 1021, 1024]  # 32 threads a row above 768 rows
WIDER = [2056, 3001, 4096, 6000, 6001, 8192, 8191]  # 256 threads a row above 128 rows
FEW = [1, 129, 200, 500, 503, 1024, 1021, 1500, 1237, 2048, 2047, 2056, 3001, 8192, 8191, 8200, 8193, 16384, 16383]
CASES = [(771, d) for d in WIDE] + [(131, d) for d in WIDER] + [(7, d) for d in FEW]


def form(rows, d):
    """Threads of a team, groups of eight columns a thread as compiled, whole groups: the rule of the launch."""
    team = (256 if d > 256 and rows <= 768 else 32) if d <= 1024 else 256 if d <= 2048 else \
        (1024 if rows <= 128 else 256) if d <= 8192 else 1024
    groups = -(-(-(-d // 8)) // team)
    if team == 1024:
        return team, 1 if groups <= 1 else 2, d % 8 == 0
    return team, groups if d % 8 == 0 or groups <= 2 else 4, d % 8 == 0


def test_the_cases_reach_every_form():
    every = {form(rows, d) for rows in (1, 128, 129, 768, 769, 8192) for d in range(1, 16385)}
    assert {form(rows, d) for rows, d in CASES} == every


def test_quantise_all_is_quantise():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(140, 300)) * np.exp2(rng.integers(-140, 120, size=(140, 1)))
    x[0], x[1, 3], x[2, 4], x[3, 5], x[4, 0] = 0, np.inf, np.nan, 1.75 * 2.0 ** 8, np.nextafter(1.75 * 2.0 ** 8, 500)
    for fmt in R.TOPS:
        for block_rows in (1, 128):
            for a, b in zip(R.quantise(x, fmt, block_rows), R.quantise_all(x, fmt, block_rows)):
                assert np.array_equal(a, b, equal_nan=a.dtype != np.uint8)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", CASES)
@pytest.mark.parametrize("tx,ts,ty", [(BF16, F32, BF16), (F32, BF16, F32), (F32, F32, BF16), (BF16, BF16, F32)])
def test_norm_forward_forms(rows, d, tx, ts, ty):
    forward(np.random.default_rng(d), rows, d, tx, ts, ty, p=0.2, pad=d % 3)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", CASES)
@pytest.mark.parametrize("ty,ts,tx", [(F32, F32, BF16), (BF16, BF16, F32), (F32, BF16, BF16), (BF16, F32, F32)])
def test_norm_backward_forms(rows, d, ty, ts, tx):
    backward(np.random.default_rng(d), rows, d, ty, ts, tx, p=0.2, pad=d % 3)


def check8(q, e, x, fmt, block_rows, what):
    """Every byte of a room8 and of its scale table."""
    ref, eref = R.quantise_all(x, fmt, block_rows)
    rows, k = x.shape
    kp = -(-k // 128) * 128
    raw = whole(q).view(torch.uint8).cpu().reshape(rows + 1, kp + 16)
    assert np.array_equal(raw[:rows, :k].contiguous().view(FP8[fmt]).double().numpy(), ref, equal_nan=True), what + ": values"
    assert not bool(raw[:rows, k:kp].any()) and bool((raw[:rows, kp:] == 0x55).all()) and bool((raw[rows:] == 0x55).all()), what
    es = whole(e).cpu()
    assert np.array_equal(es[:eref.shape[0], :eref.shape[1]].numpy(), eref), what + ": scales"
    assert bool((es[:, eref.shape[1]:] == 0x55).all()) and bool((es[eref.shape[0]:] == 0x55).all()), what + ": scale bytes outside"


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d", CASES)
@pytest.mark.parametrize("fmt,tx,ts", [("e4m3", BF16, F32), ("e5m2", F32, BF16)])
def test_norm_in_8_bits_forms(rows, d, fmt, tx, ts):
    """The 8-bit y is the quantisation of the float32 y that the same call gives, byte for byte."""
    rng = np.random.default_rng(d)
    x, r = matrix(rng, rows, d, tx), matrix(rng, rows, d, ts)
    g, b = (torch.from_numpy(rng.normal(size=d)).float().to(DEV) for _ in range(2))
    y, q, e = torch.empty(rows, d, device=DEV), room8(rows, d, fmt), scale_room(rows, d)
    kw = dict(residual=r, p=0.1, seed=3)
    LU.layup_layernorm_forward(LU.layernorm_desc(x, y, g, b, **kw), torch.cuda.current_stream())
    LU.layup_layernorm_forward(LU.layernorm_desc(x, q, g, b, y_scale=e, **kw), torch.cuda.current_stream())
    torch.cuda.synchronize()
    check8(q, e, f64(y), fmt, 1, "y")


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(2100, 2185), (129, 33000), (33000, 129), (4097, 1024)])  # above 256 tiles of 128 x 128
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantise_many_tiles(rows, cols, block_rows, fmt, dtype):
    """q and qt together and each alone, scales far apart, a row of zeros, what is not finite, subnormals."""
    x = matrix(np.random.default_rng(rows), rows, cols, dtype, 3)
    x *= torch.exp(5 * torch.randn(rows, 1, device=DEV)).to(dtype)
    x[1] = 0
    x[2, :3] = torch.tensor([float("inf"), float("-inf"), float("nan")], dtype=dtype)
    x[3] = 1e-40
    x[rows - 1, cols - 1] = 1.75 * 2.0 ** 100
    s = torch.cuda.current_stream()
    for want in (("q", "qt"), ("q",), ("qt",)):
        room = {}
        for k in want:
            r, c = (rows, cols) if k == "q" else (cols, rows)
            room[k], room["scale" if k == "q" else "scale_t"] = room8(r, c, fmt), scale_room(-(-r // block_rows), c)
        LU.layup_quant_fp8(LU.quant_desc(x, block_rows, **room), s)
        torch.cuda.synchronize()
        if "q" in want:
            check8(room["q"], room["scale"], f64(x), fmt, block_rows, "q")
        if "qt" in want:
            check8(room["qt"], room["scale_t"], f64(x).T, fmt, block_rows, "qt")
