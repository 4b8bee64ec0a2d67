"""Refusals of the dropout, LayerNorm and 8-bit calls: every argument error is found on the host before anything is
enqueued, and what there is nothing to do for returns at once.  No call here launches a kernel; no GPU needed."""
import pytest

from paper_2410_05985_amd import layup as LU

INVALID, SHAPE, ALIGN, DTYPE = (LU.LAYUP_ERR_INVALID_ARG, LU.LAYUP_ERR_SHAPE, LU.LAYUP_ERR_ALIGN, LU.LAYUP_ERR_DTYPE)


def mask(p=0.0, **k):
    return LU.layup_dropout_mask(p=p, **k)


def dropout(**k):
    d = dict(rows=4, cols=8, x=0x1000, ldx=8, y=0x2000, ldy=8, dtype=LU.LAYUP_F32, drop=mask(0.5))
    d.update(k)
    return LU.layup_dropout, LU.layup_dropout_desc(**d)


def norm(**k):
    d = dict(rows=4, d=8, eps=1e-5, x=0x1000, ldx=8, residual=0x2000, ldr=8, sum=0x3000, lds=8, y=0x4000, ldy=8,
             gamma=0x5000, beta=0x6000, x_dtype=LU.LAYUP_BF16, s_dtype=LU.LAYUP_F32, y_dtype=LU.LAYUP_BF16, drop=mask())
    d.update(k)
    return LU.layup_layernorm_forward, LU.layup_layernorm_desc(**d)


def norm8(**k):
    return norm(**{**dict(y_dtype=LU.LAYUP_E4M3, ldy=128, y_scale=0x7000, ld_scale=4), **k})


def grad(**k):
    d = dict(rows=4, d=8, dy=0x1000, lddy=8, s=0x2000, lds=8, dsum=0x3000, lddsum=8, mean=0x4000, rstd=0x5000, gamma=0x6000,
             dres=0x7000, lddres=8, dx=0x8000, lddx=8, dgamma=0x9000, dbeta=0xa000, workspace=0xb000,
             workspace_bytes=1 << 20, dy_dtype=LU.LAYUP_F32, s_dtype=LU.LAYUP_F32, dx_dtype=LU.LAYUP_BF16, drop=mask())
    d.update(k)
    return LU.layup_layernorm_backward, LU.layup_layernorm_grad_desc(**d)


def quant(**k):
    d = dict(rows=4, cols=8, x=0x1000, ldx=8, x_dtype=LU.LAYUP_BF16, q_dtype=LU.LAYUP_E4M3, block_rows=1, q=0x2000, ldq=128,
             scale=0x3000, ld_scale=4, qt=0x4000, ldqt=128, scale_t=0x5000, ld_scale_t=4)
    d.update(k)
    return LU.layup_quant_fp8, LU.layup_quant_desc(**d)


def gemm(**k):
    d = dict(M=4, N=8, K=16, A=0x1000, lda=128, a_scale=0x2000, ld_a_scale=4, B=0x3000, ldb=128, b_scale=0x4000,
             ld_b_scale=4, C=0x5000, ldc=8, a_dtype=LU.LAYUP_E4M3, b_dtype=LU.LAYUP_E4M3, a_block=1, b_block=128)
    d.update(k)
    return LU.layup_gemm_fp8, LU.layup_gemm_fp8_desc(**d)


CASES = [
    (dropout, dict(rows=-1), SHAPE), (dropout, dict(cols=-1), SHAPE), (dropout, dict(rows=1 << 31), SHAPE),
    (dropout, dict(cols=1 << 33), SHAPE), (dropout, dict(dtype=LU.LAYUP_E4M3), DTYPE), (dropout, dict(dtype=9), DTYPE),
    (dropout, dict(drop=mask(1.0)), INVALID), (dropout, dict(drop=mask(-0.1)), INVALID),
    (dropout, dict(drop=mask(float("nan"))), INVALID), (dropout, dict(drop=mask(0.5, offset_dev=0x1004)), ALIGN),
    (dropout, dict(x=None), INVALID), (dropout, dict(y=None), INVALID), (dropout, dict(ldx=7), SHAPE),
    (dropout, dict(ldy=0), SHAPE), (dropout, dict(x=0x1002), ALIGN), (dropout, dict(dtype=LU.LAYUP_BF16, y=0x2001), ALIGN),
    (dropout, dict(y=0x1000, ldy=16), INVALID),
    (norm, dict(rows=-1), SHAPE), (norm, dict(rows=1 << 31), SHAPE), (norm, dict(d=0), SHAPE), (norm, dict(d=16385), SHAPE),
    (norm, dict(x_dtype=LU.LAYUP_E4M3), DTYPE), (norm, dict(s_dtype=7), DTYPE), (norm, dict(y_dtype=-1), DTYPE),
    (norm, dict(eps=-1.0), INVALID), (norm, dict(eps=float("nan")), INVALID), (norm, dict(eps=float("inf")), INVALID),
    (norm, dict(drop=mask(1.0)), INVALID), (norm, dict(x=None), INVALID), (norm, dict(y=None), INVALID),
    (norm, dict(ldr=4), SHAPE), (norm, dict(lds=7), SHAPE), (norm, dict(ldy=7), SHAPE), (norm, dict(sum=0x2000, lds=16), INVALID),
    (norm, dict(x=0x1001), ALIGN), (norm, dict(residual=0x2002), ALIGN), (norm, dict(gamma=0x5002), ALIGN),
    (norm, dict(mean=0x5001), ALIGN),
    (norm8, dict(ldy=120), ALIGN), (norm8, dict(ldy=112), SHAPE), (norm8, dict(y=0x4008), ALIGN),
    (norm8, dict(y_scale=None), INVALID), (norm8, dict(ld_scale=2), ALIGN), (norm8, dict(ld_scale=0), SHAPE),
    (norm8, dict(d=520, ldx=520, ldr=520, lds=520, ldy=640), SHAPE),
    (grad, dict(rows=-1), SHAPE), (grad, dict(d=16385), SHAPE), (grad, dict(dy_dtype=LU.LAYUP_E5M2), DTYPE),
    (grad, dict(dx_dtype=5), DTYPE), (grad, dict(dy=None), INVALID), (grad, dict(s=None), INVALID),
    (grad, dict(mean=None), INVALID), (grad, dict(rstd=None), INVALID), (grad, dict(lddy=7), SHAPE),
    (grad, dict(lddsum=7), SHAPE), (grad, dict(lddres=7), SHAPE), (grad, dict(lddx=7), SHAPE),
    (grad, dict(dres=0x3000, lddres=16), INVALID), (grad, dict(workspace=None), INVALID),
    (grad, dict(workspace_bytes=60), INVALID), (grad, dict(workspace=0xb004), ALIGN), (grad, dict(dgamma=0x9002), ALIGN),
    (grad, dict(rstd=0x5002), ALIGN), (grad, dict(drop=mask(2.0)), INVALID),
    (quant, dict(rows=-1), SHAPE), (quant, dict(cols=1 << 31), SHAPE), (quant, dict(x_dtype=LU.LAYUP_E4M3), DTYPE),
    (quant, dict(q_dtype=LU.LAYUP_BF16), DTYPE), (quant, dict(block_rows=64), INVALID), (quant, dict(q=None, qt=None), INVALID),
    (quant, dict(x=None), INVALID), (quant, dict(ldx=4), SHAPE), (quant, dict(x=0x1001), ALIGN), (quant, dict(ldq=64), SHAPE),
    (quant, dict(ldq=136), ALIGN), (quant, dict(q=0x2008), ALIGN), (quant, dict(scale=None), INVALID),
    (quant, dict(scale=0x3002), ALIGN), (quant, dict(ld_scale=5), ALIGN), (quant, dict(ldqt=64), SHAPE),
    (quant, dict(qt=0x4004), ALIGN), (quant, dict(scale_t=None), INVALID), (quant, dict(rows=520, ldqt=640), SHAPE),
    (gemm, dict(M=-1), SHAPE), (gemm, dict(N=1 << 31), SHAPE), (gemm, dict(K=-1), SHAPE), (gemm, dict(a_dtype=LU.LAYUP_BF16), DTYPE),
    (gemm, dict(b_dtype=4), DTYPE), (gemm, dict(a_block=2), INVALID), (gemm, dict(b_block=0), INVALID), (gemm, dict(C=None), INVALID),
    (gemm, dict(ldc=7), SHAPE), (gemm, dict(C=0x5001), ALIGN), (gemm, dict(c_f32=1, C=0x5002), ALIGN), (gemm, dict(bias=0x6002), ALIGN),
    (gemm, dict(A=None), INVALID), (gemm, dict(B=None), INVALID), (gemm, dict(lda=16), SHAPE), (gemm, dict(ldb=130), ALIGN),
    (gemm, dict(A=0x1008), ALIGN), (gemm, dict(a_scale=None), INVALID), (gemm, dict(b_scale=0x4001), ALIGN),
    (gemm, dict(ld_a_scale=6), ALIGN), (gemm, dict(K=513, lda=640, ldb=640), SHAPE), (gemm, dict(lda=(1 << 24) + 16), SHAPE),
    (gemm, dict(ld_b_scale=(1 << 24) + 4), SHAPE), (gemm, dict(workspace=0x6004), ALIGN),
]


@pytest.mark.parametrize("make,args,status", CASES, ids=lambda v: v.__name__ if callable(v) else None)
def test_refused_on_the_host(make, args, status):
    call, desc = make(**args)
    with pytest.raises(LU.LayupError) as e:
        call(desc)
    assert e.value.status == status and str(e.value).split(": ", 1)[1], e.value


@pytest.mark.parametrize("make,args", [
    (dropout, dict(rows=0, x=None, y=None)), (dropout, dict(cols=0, x=None, y=None)), (norm, dict(rows=0, x=None, y=None)),
    (grad, dict(rows=0, dy=None, s=None, mean=None, rstd=None, dgamma=None, dbeta=None, workspace=None)),
    (quant, dict(rows=0, x=None)), (quant, dict(cols=0, x=None)), (gemm, dict(M=0, C=None)), (gemm, dict(N=0, B=None, C=None)),
])
def test_nothing_to_do_returns(make, args):
    call, desc = make(**args)
    call(desc)


def test_null_descriptors():
    L = LU.lib()
    for f in (L.layup_dropout, L.layup_layernorm_forward, L.layup_layernorm_backward, L.layup_quant_fp8, L.layup_gemm_fp8):
        assert f(None, None) == INVALID and L.layup_global_error()


def test_layernorm_workspace():
    L = LU.lib()
    assert L.layup_layernorm_workspace_size(4, 8, None) == INVALID
    for rows, d in ((-1, 8), (1 << 31, 8), (4, 0), (4, 16385)):
        with pytest.raises(LU.LayupError) as e:
            LU.layup_layernorm_workspace_size(rows, d)
        assert e.value.status == SHAPE
    assert LU.layup_layernorm_workspace_size(0, 8) == 0
    for d in (8, 300, 768, 1000, 2048, 5000, 16384):  # sized for the largest batch, it serves the smaller ones
        sizes = [LU.layup_layernorm_workspace_size(r, d) for r in (1, 7, 96, 128, 129, 511, 513, 768, 769, 4000, 8192)]
        assert sizes == sorted(sizes)
    assert LU.layup_layernorm_workspace_size(8192, 768) >= 2 * 768 * 4


def test_descriptors_from_tensors():
    """The binding reads sizes, row distances and types from tensors and refuses what they cannot be."""
    torch = pytest.importorskip("torch")
    x = torch.zeros(5, 20, dtype=torch.bfloat16)[:, :12]
    d = LU.dropout_desc(x, x, p=0.5, seed=(1 << 64) - 1, offset=3)
    assert (d.rows, d.cols, d.ldx, d.ldy, d.dtype, d.drop.seed) == (5, 12, 20, 20, LU.LAYUP_BF16, (1 << 64) - 1)
    one = torch.zeros(1, 12)
    assert LU.dropout_desc(one.as_strided((1, 12), (1, 1)), one, p=0.0).ldx == 12
    for bad in (x.t(), x[0]):
        with pytest.raises(ValueError):
            LU.dropout_desc(bad, bad, p=0.5)
    with pytest.raises(ValueError):
        LU.dropout_desc(x, x[:4], p=0.5)
    with pytest.raises(TypeError):
        LU.dropout_desc(x, x.float(), p=0.5)
    with pytest.raises(TypeError):
        LU.dropout_desc(x.half(), x.half(), p=0.5)
    with pytest.raises(ValueError):
        LU.dropout_desc(x, x, p=0.5, seed=-1)
    g = torch.ones(12)
    n = LU.layernorm_desc(x, x.float(), g, None, residual=x.float())
    assert (n.rows, n.d, n.x_dtype, n.s_dtype, n.y_dtype, n.beta) == (5, 12, LU.LAYUP_BF16, LU.LAYUP_F32, LU.LAYUP_F32, None)
    with pytest.raises(ValueError):
        LU.layernorm_desc(x, x, g[:11])
    with pytest.raises(ValueError):
        LU.layernorm_desc(x, x, g.double())
    q = torch.zeros(5, 128, dtype=torch.uint8).view(torch.float8_e4m3fn)
    e = torch.zeros(5, 4, dtype=torch.uint8)
    with pytest.raises(ValueError):
        LU.layernorm_desc(x, q, g)  # an 8-bit y without its scales
    with pytest.raises(ValueError):
        LU.quant_desc(x, 1, q=q[:, :64], scale=e)
    with pytest.raises(ValueError):
        LU.quant_desc(x, 1, q=q, scale=e[:4])
    with pytest.raises(ValueError):
        LU.gemm_fp8_desc(q, e, 1, q, e, 1, torch.zeros(5, 6), 12)  # B has five rows, C six columns
    assert LU.gemm_fp8_desc(q, e, 1, q, e, 1, torch.zeros(5, 5), 12).c_f32 == 1
    with pytest.raises(ValueError):
        LU.dropout_desc(x, x.to("meta"), p=0.5)  # two devices
    with pytest.raises(ValueError):
        LU.layup_dropout(LU.dropout_desc(x, x, p=0.5))  # host memory
