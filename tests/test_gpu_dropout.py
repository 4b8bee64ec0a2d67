"""The GPT step with dropout (layup_set_dropout): embedding and residual dropout from the counter-based generator, in
the forward and in every unit's backward, against the oracle with the same masks."""
import numpy as np
import pytest

import oracle as O
from oracle import operators_ref as R
from paper_2410_05985_amd import synthetic as S
from tests.gpt_cases import block_cache_from_gpu, gpt_hp, gpt_setup
from tests.parity import compare, compare_chained

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from paper_2410_05985_amd import layup as LU  # noqa: E402

DEV = "cuda"
GRAD_RTOL = 2e-2  # bfloat16 operands, as the step without dropout


def keeps(cfg, p, seed, step=0):
    n = 2 * cfg.n_layer + 1
    return [R.keep_mask(cfg.batch * cfg.seq, cfg.d_model, p, seed, step * n + site) * R.drop_scale(p) for site in range(n)]


@pytest.mark.parametrize("cfg", [S.GPT_TEST, S.GPT_TEST_RAGGED, S.GPT_TEST_DH48, S.GPT_TEST_W832, S.GPT_TEST4, S.GPT_TEST_W2048],
                         ids=lambda c: c.name)
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_units_teacher_forced(cfg, p):
    """The stored activations follow from one another with the masks, and every unit's backward, from what the GPU
    handed it, matches the oracle's."""
    params, tokens, peers, m = gpt_setup(cfg)
    hp, _ = gpt_hp(cfg)
    pf = {k: v.astype(np.float64) for k, v in params.items()}
    N, d, V, L = cfg.batch * cfg.seq, cfg.d_model, cfg.vocab, cfg.n_layer
    seed = 0x1234567890ABCDEF
    keep = keeps(cfg, p, seed)
    td = torch.from_numpy(tokens).to(DEV)
    torch.cuda.synchronize()
    LU.layup_set_dropout(m.ctx, p, seed)
    LU.layup_forward(m.ctx, td, None, None)
    LU.layup_set_dropout(m.ctx, 0.7, seed + 1)  # for the next forward: this one's backward keeps its masks
    m.synchronize()
    idx = tokens[:, :cfg.seq].reshape(-1)
    emb = pf["wte"][idx] + pf["wpe"][np.tile(np.arange(cfg.seq), cfg.batch)]
    x0 = m.activation(0, 0).astype(np.float64).reshape(N, d)
    # one float32 sum and one float32 product
    assert np.all(np.abs(x0 - emb * keep[0]) <= 3 * 2.0 ** -24 * (np.abs(pf["wte"][idx]) + np.abs(emb)) * np.maximum(keep[0], 0))
    caches = [block_cache_from_gpu(m, cfg, l) for l in range(L)]
    xs = [c["x"] for c in caches] + [m.activation(11).astype(np.float64).reshape(N, d)]
    for l, c in enumerate(caches):
        q = f"h{l}."
        compare(c["a"], O.bf16(O.layernorm_fwd(c["x"], pf[q + "ln1.g"], pf[q + "ln1.b"])), 1e-2, f"ln1 {l}")
        branch = c["o"] @ O.bf16(pf[q + "proj.w"]).T + pf[q + "proj.b"]
        compare(c["h"] - c["x"], branch * keep[1 + 2 * l], 1e-4, f"attention branch {l}")
        compare(c["a2"], O.bf16(O.layernorm_fwd(c["h"], pf[q + "ln2.g"], pf[q + "ln2.b"])), 1e-2, f"ln2 {l}")
        branch = c["gl"] @ O.bf16(pf[q + "mproj.w"]).T + pf[q + "mproj.b"]
        compare(xs[l + 1] - c["h"], branch * keep[2 + 2 * l], 1e-4, f"mlp branch {l}")
        # a dropped element leaves the residual as it is
        assert np.array_equal((c["h"])[keep[1 + 2 * l] == 0], c["x"][keep[1 + 2 * l] == 0])
    Vp = (V + 63) // 64 * 64
    dlog = m.activation(10).astype(np.float64).reshape(N, Vp)[:, :V]
    xf = m.activation(9).astype(np.float64).reshape(N, d)
    LU.layup_layer_backward(m.ctx, L + 1)
    LU.layup_unit_update_mix(m.ctx, L + 1, hp, cfg.alpha, 0)
    g_ref, dx_ref, wte_head = O.gpt_head_bwd(pf, dlog, xf, xs[L])
    g = m.read("grads")
    for k, ref in g_ref.items():
        compare(g[k], ref, GRAD_RTOL, f"grad {k}")
    dx = m.activation(13).astype(np.float64).reshape(N, d)
    compare(dx, dx_ref, GRAD_RTOL, "top unit input gradient")
    for l in range(L - 1, -1, -1):
        LU.layup_layer_backward(m.ctx, l + 1)
        LU.layup_unit_update_mix(m.ctx, l + 1, hp, cfg.alpha, 0)
        g_ref, dx_ref = O.gpt_block_bwd(pf, caches[l], dx, l, cfg.batch, cfg.seq, cfg.n_head, keep=keep)
        g = m.read("grads")
        for k, ref in g_ref.items():
            compare(g[k], ref.reshape(g[k].shape), GRAD_RTOL, f"grad {k}")
        dx = m.activation(13).astype(np.float64).reshape(N, d)
        compare(dx, dx_ref, GRAD_RTOL, f"unit {l + 1} input gradient")
    LU.layup_layer_backward(m.ctx, 0)
    LU.layup_unit_update_mix(m.ctx, 0, hp, cfg.alpha, 0)
    g_ref = O.gpt_embed_bwd(dx, idx, wte_head, cfg.batch, cfg.seq, keep)
    g = m.read("grads")
    for k, ref in g_ref.items():
        compare(g[k], ref, GRAD_RTOL, f"grad {k}")
    m.close()


def test_two_steps_draw_two_masks_and_match_the_oracle():
    """Whole steps: loss and chained gradients of each against the oracle with that step's masks."""
    cfg = S.GPT_TEST
    params, tokens, peers, m = gpt_setup(cfg)
    td = torch.from_numpy(tokens).to(DEV)
    loss = torch.zeros(1, dtype=torch.float32, device=DEV)
    LU.layup_set_dropout(m.ctx, 0.2, 99)
    for step in range(2):
        hp, ohp = gpt_hp(cfg, step + 1)
        now = {k: v.astype(np.float64) for k, v in m.read("params").items()}
        torch.cuda.synchronize()
        LU.layup_step(m.ctx, td, None, hp, cfg.alpha, 0, loss)
        m.synchronize()
        runs = [O.gpt_step({k: v.copy() for k, v in now.items()}, None, None, None, tokens, cfg.n_head, ohp, cfg.alpha, rnd=r,
                           update=False, keep=keeps(cfg, 0.2, 99, step)) for r in (O.bf16, O.ident)]
        assert abs(loss.item() - runs[0][0]) <= 2e-3 * abs(runs[0][0])
        other = O.gpt_forward(now, tokens, cfg.n_head, keep=keeps(cfg, 0.2, 99, 1 - step))[0]
        assert abs(loss.item() - runs[0][0]) < abs(loss.item() - other)
        g = m.read("grads")
        for k in g:
            compare_chained(g[k], runs[0][1][k].reshape(g[k].shape), GRAD_RTOL, f"step {step} grad {k}", exact=runs[1][1][k].reshape(g[k].shape))
    m.close()


def run_steps(cfg, p, seed, n=2, two_streams=True, schedule=LU.LAYUP_SCHEDULE_LAYERWISE, first=None):
    params, tokens, peers, m = gpt_setup(cfg, two_streams)
    td = torch.from_numpy(tokens).to(DEV)
    if first is not None:
        LU.layup_set_dropout(m.ctx, *first)
    if p is not None:
        LU.layup_set_dropout(m.ctx, p, seed)
    torch.cuda.synchronize()
    for s in range(n):
        hp, _ = gpt_hp(cfg, s + 1)
        LU.layup_step_ex(m.ctx, td, None, hp, cfg.alpha, schedule)
    m.synchronize()
    out = m.params.cpu().numpy().copy()
    m.close()
    return out


def test_off_is_the_step_without():
    """p = 0, p that rounds to 0, and dropout set and taken back give the bits of a context that never had it."""
    want = run_steps(S.GPT_TEST, None, 0)
    assert np.array_equal(want, run_steps(S.GPT_TEST, 0.0, 5))
    assert np.array_equal(want, run_steps(S.GPT_TEST, 1e-6, 5))
    assert np.array_equal(want, run_steps(S.GPT_TEST, 0.0, 5, first=(0.5, 7)))
    assert not np.array_equal(want, run_steps(S.GPT_TEST, 0.1, 5))


def test_evaluation_between_steps():
    """Dropout off for a forward that has no backward, and on again: the next step is as if it had not been."""
    cfg = S.GPT_TEST
    outs, losses = [], []
    for evaluate in (False, True):
        params, tokens, peers, m = gpt_setup(cfg)
        td = torch.from_numpy(tokens).to(DEV)
        loss = torch.zeros(1, dtype=torch.float32, device=DEV)
        for s in range(2):
            hp, _ = gpt_hp(cfg, s + 1)
            if evaluate:
                LU.layup_set_dropout(m.ctx, 0.0, 0)
                torch.cuda.synchronize()
                LU.layup_forward(m.ctx, td, None, loss)
                m.synchronize()
                losses.append(loss.item())
            LU.layup_set_dropout(m.ctx, 0.3, 8)
            torch.cuda.synchronize()
            LU.layup_step(m.ctx, td, None, hp, cfg.alpha, 0)
        m.synchronize()
        outs.append(m.params.cpu().numpy().copy())
        if evaluate:
            ref = O.gpt_forward({k: v.astype(np.float64) for k, v in params.items()}, tokens, cfg.n_head)[0]
            assert abs(losses[0] - ref) <= 2e-3 * abs(ref)
        m.close()
    assert np.array_equal(outs[0], outs[1])


@pytest.mark.parametrize("cfg", [S.GPT_TEST, S.GPT_TEST4], ids=lambda c: c.name)
def test_the_same_bits_on_one_stream_and_every_time(cfg):
    want = run_steps(cfg, 0.1, 5)
    assert np.array_equal(want, run_steps(cfg, 0.1, 5))
    assert np.array_equal(want, run_steps(cfg, 0.1, 5, two_streams=False))
    assert np.array_equal(want, run_steps(cfg, 0.1, 5, schedule=LU.LAYUP_SCHEDULE_AFTER_BACKWARD))
    assert not np.array_equal(want, run_steps(cfg, 0.1, 6))


def test_fused_schedule_takes_the_same_masks():
    """The schedule that updates the weights in their dW products: the layer-wise step's parameters up to the order of
    the dW sums (its own test's bar)."""
    a = run_steps(S.GPT_TEST, 0.1, 5, n=1)
    b = run_steps(S.GPT_TEST, 0.1, 5, n=1, schedule=LU.LAYUP_SCHEDULE_FUSED_DW)
    plain = run_steps(S.GPT_TEST, None, 5, n=1)
    assert np.linalg.norm(a - b) <= 1e-2 * np.linalg.norm(a - plain)


def test_refusals():
    params, tokens, peers, m = gpt_setup(S.GPT_TEST)
    for p in (1.0, -0.1, float("nan")):
        with pytest.raises(LU.LayupError) as e:
            LU.layup_set_dropout(m.ctx, p, 0)
        assert e.value.status == LU.LAYUP_ERR_INVALID_ARG
    m.close()
    mlp = LU.Model(LU.mlp_config((8, 8), 4), "sgd")
    with pytest.raises(LU.LayupError) as e:
        LU.layup_set_dropout(mlp.ctx, 0.1, 0)
    assert e.value.status == LU.LAYUP_ERR_DTYPE
    mlp.close()
    assert LU.lib().layup_set_dropout(None, 0.1, 0) == LU.LAYUP_ERR_INVALID_ARG
