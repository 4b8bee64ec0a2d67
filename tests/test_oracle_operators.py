"""Pins of the float64 reference of dropout, LayerNorm and 8-bit floats (oracle/operators_ref.py): published answers,
finite differences, torch's own 8-bit casts, and the definitions' invariants.  No GPU needed."""
import numpy as np
import pytest

from oracle import operators_ref as R

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("ctr,key,out", [
    # the published known answers of the generator
    ([0] * 4, [0] * 2, [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
     [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]),
])
def test_philox_known_answers(ctr, key, out):
    assert [int(x) for x in R.philox4x32_10([np.array(c) for c in ctr], key)] == out


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_mask_keeps_its_share(p):
    """512 x 1024 draws of a keep probability q = 1 - T/65536: the count is within six standard deviations."""
    m = R.keep_mask(512, 1024, p, 0x123456789ABCDEF, 1 << 40)
    q = 1 - R.drop_threshold(p) / 65536
    assert abs(m.sum() - m.size * q) < 6 * np.sqrt(m.size * q * (1 - q))
    other = R.keep_mask(512, 1024, p, 0x123456789ABCDEF, (1 << 40) + 1)
    both = (m & other).sum()  # another offset is another, independent mask
    assert abs(both - m.size * q * q) < 6 * np.sqrt(m.size * q * q * (1 - q * q))


def test_mask_goes_by_row_and_column():
    m = R.keep_mask(20, 50, 0.5, 7, 9)
    assert np.array_equal(R.keep_mask(12, 33, 0.5, 7, 9), m[:12, :33])
    assert np.array_equal(R.keep_mask(5, 50, 0.5, 7, 9, row0=15), m[15:])


def test_dropout_keeps_the_mean():
    assert R.drop_scale(0.0) == 1.0 and R.drop_threshold(1e-7) == 0
    assert R.drop_threshold(np.nextafter(np.float32(1), np.float32(0))) == 65535
    for p in (0.1, 1 / 3, 0.9):
        assert R.drop_scale(p) * (1 - R.drop_threshold(p) / 65536) == pytest.approx(1.0, rel=1e-15)


def test_norm_backward_by_differences():
    rng = np.random.default_rng(3)
    s, w = rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    g, b = rng.normal(size=7), rng.normal(size=7)
    _, mean, rstd = R.norm_fwd(s, g, b, 1e-5)
    ds, dg, db = R.norm_bwd(w, s, mean, rstd, g, 0.0)
    f = lambda s, g, b: (R.norm_fwd(s, g, b, 1e-5)[0] * w).sum()  # noqa: E731
    h = 1e-6
    for i in np.ndindex(*s.shape):
        e = np.zeros_like(s)
        e[i] = h
        assert (f(s + e, g, b) - f(s - e, g, b)) / (2 * h) == pytest.approx(ds[i], rel=1e-6, abs=1e-7)
    for i in range(7):
        e = np.zeros(7)
        e[i] = h
        assert (f(s, g + e, b) - f(s, g - e, b)) / (2 * h) == pytest.approx(dg[i], rel=1e-6, abs=1e-8)
        assert (f(s, g, b + e) - f(s, g, b - e)) / (2 * h) == pytest.approx(db[i], rel=1e-6, abs=1e-8)


@pytest.mark.parametrize("fmt,t", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_fp8_rounding_is_the_formats(fmt, t):
    top = 1.75 * 2.0 ** R.TOPS[fmt][0]
    every = torch.arange(256, dtype=torch.uint8).view(t).double().numpy()
    every = np.unique(every[np.isfinite(every)])
    assert every.max() == top and np.array_equal(R.round_fp8(every, fmt), every)
    mid = (every[:-1] + every[1:]) / 2  # ties, and their neighbours
    v = np.concatenate([mid, np.nextafter(mid, np.inf, dtype=np.float32), np.nextafter(mid, -np.inf, dtype=np.float32),
                        np.random.default_rng(0).uniform(-top, top, 10000), np.random.default_rng(1).normal(size=10000) * 2.0 ** -8])
    v = v.astype(np.float32)
    assert np.array_equal(R.round_fp8(v, fmt), torch.from_numpy(v).to(t).double().numpy())


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantise_scales(fmt, block_rows):
    rng = np.random.default_rng(5)
    x = rng.normal(size=(130, 300)) * np.exp(4 * rng.normal(size=(130, 1)))
    x[0] = 0
    x[128:] = 0  # a whole block of zeros
    x[3, 7], x[4, 8] = np.inf, np.nan
    q, e = R.quantise(x, fmt, block_rows)
    top, bits, _ = R.TOPS[fmt]
    fin = np.isfinite(x)
    assert np.isnan(q[3, 7]) and np.isnan(q[4, 8]) and np.isfinite(q[fin]).all()
    assert np.abs(q[fin]).max() <= 1.75 * 2.0 ** top
    assert e[-1, 0] == 127
    v = R.value(q, e, block_rows)
    amax = np.where(fin, np.abs(x), 0)
    for i in range(e.shape[0]):
        for j in range(e.shape[1]):
            at = (slice(i * block_rows, (i + 1) * block_rows), slice(128 * j, 128 * j + 128))
            big = amax[at].max()
            if big:  # the scale is the least power of two that fits
                assert big <= 1.75 * 2.0 ** (top + int(e[i, j]) - 127) and big > 1.75 * 2.0 ** (top + int(e[i, j]) - 128)
            err = np.abs(v[at] - x[at])[fin[at]]
            assert (err <= np.maximum(np.abs(x[at])[fin[at]] * 2.0 ** -(bits + 1), big * 2.0 ** -(bits + 1) * 2.0 ** -13)).all()


def test_gpt_step_with_dropout_by_differences():
    """Every gradient of a tiny two-block GPT with dropout at its sites, against central differences of its loss."""
    import oracle as O
    from paper_2410_05985_amd import synthetic as S
    cfg = S.GPTConfig(n_layer=2, d_model=8, n_head=2, d_ff=16, seq=4, batch=2, vocab=11)
    rng = np.random.default_rng(6)
    params = {n: rng.standard_normal(s) * (0.3 if len(s) >= 2 else 0.1) + (1.0 if n.endswith(".g") else 0.0)
              for n, s, _ in S.gpt_param_specs(cfg)}
    tokens = rng.integers(0, cfg.vocab, (cfg.batch, cfg.seq + 1))
    keep = [R.keep_mask(8, 8, 0.4, 3, site) * R.drop_scale(0.4) for site in range(5)]
    hp = dict(optim="adamw", lr=0.0, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0)
    _, grads, _, _ = O.gpt_step({k: v.copy() for k, v in params.items()}, None, None, None, tokens, cfg.n_head, hp, 0.0,
                                rnd=O.ident, update=False, store=O.ident, keep=keep)
    loss = lambda: O.gpt_forward(params, tokens, cfg.n_head, rnd=O.ident, keep=keep)[0]  # noqa: E731
    h = 1e-5
    for n, a in params.items():
        for i in list(np.ndindex(*a.shape))[::5]:
            old = a[i]
            a[i] = old + h
            up = loss()
            a[i] = old - h
            down = loss()
            a[i] = old
            assert (up - down) / (2 * h) == pytest.approx(grads[n][i], rel=1e-5, abs=1e-9), (n, i)
