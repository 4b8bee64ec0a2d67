"""Performance cases of the operators on the way into a linear layer: dropout, LayerNorm with its residual add, and
the linear layer in 8-bit floats.

A case is a dict of plain values.  ``op`` says which call it stands for:

* ``dropout`` dropout of a matrix from a counter-based generator (its backward is the same call on the gradient);
* ``norm``    s = residual + dropout(x), y = LayerNorm(s): a forward pass, or forward and backward;
* ``quant``   a weight matrix in 8 bits, a power-of-two scale for each 128 x 128 block, as it is and transposed;
* ``linear``  y = x W^T + b with both operands in 8 bits: ``mode`` ``serve`` (weights held in 8 bits, x quantised in
  blocks of 128), ``norm`` (x is the LayerNorm of a residual stream) or ``train`` (forward, dX and dW, every operand
  quantised in the pass).

``listed`` holds the fixed cases, ``draw`` gives more of the same ranges, ``prepare`` makes what a program holds before
the call, ``run`` is one pass, ``exact`` the same in 64 bits, ``work`` what a pass cannot do without.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 8, "e5m2": 15}  # the largest value is 1.75 * 2^TOP
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one new token of a GPT-2-small-wide stack: latency alone
        dict(name="norm_token", op="norm", mode="fwd", rows=1, d=768, pad=0, x="bf16", s="f32", y="bf16", dx="bf16", p=0.0),
        # a GPT-2-small sublayer in training: 8 x 1024 tokens, float32 residual stream, bfloat16 branch
        dict(name="norm_train_gpt2", op="norm", mode="train", rows=8192, d=768, pad=0, x="bf16", s="f32", y="bf16", dx="bf16",
             p=0.1),
        # odd width, rows further apart than they are long, bfloat16 stream, float32 gradients
        dict(name="norm_train_odd", op="norm", mode="train", rows=1003, d=1237, pad=3, x="f32", s="bf16", y="f32", dx="f32",
             p=0.25),
        # wide rows, bfloat16 throughout, no dropout: four reads and writes of 134 MB each way
        dict(name="norm_train_wide", op="norm", mode="train", rows=8192, d=8192, pad=0, x="bf16", s="bf16", y="bf16", dx="bf16",
             p=0.0),
        # a few rows of a narrow layer
        dict(name="dropout_small", op="dropout", rows=33, d=516, pad=4, x="f32", p=0.5),
        # an MLP's activations, 8192 tokens of 8192 features
        dict(name="dropout_large", op="dropout", rows=8192, d=8192, pad=0, x="bf16", p=0.1),
        # the 1.3B stack's MLP weight, in the forms its forward and its dX product read
        dict(name="quant_weight", op="quant", rows=8192, d=2048, x="bf16", f="e4m3"),
        # one token through the 1.3B stack's MLP input projection: the weight stream bounds it
        dict(name="linear_token", op="linear", mode="serve", rows=1, d=2048, n=8192, f="e4m3", g="e4m3"),
        # GPT-2-small's qkv projection behind its LayerNorm
        dict(name="linear_norm_gpt2", op="linear", mode="norm", rows=8192, d=768, n=2304, f="e4m3", g="e4m3"),
        # off every tile size, gradients in the format with the wider range
        dict(name="linear_train_ragged", op="linear", mode="train", rows=1101, d=1000, n=523, f="e4m3", g="e5m2"),
        # GPT-2-medium's MLP input projection, forward and backward
        dict(name="linear_train_medium", op="linear", mode="train", rows=8192, d=1024, n=4096, f="e4m3", g="e5m2"),
        # the 1.3B stack's, forward and backward
        dict(name="linear_train_1p3b", op="linear", mode="train", rows=8192, d=2048, n=8192, f="e4m3", g="e4m3"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "dropout", "quant", "linear", "linear", "linear"])
    p = rng.choice([0.0, 0.1, 0.1, 0.3, 0.5])
    t = lambda: rng.choice(["f32", "bf16", "bf16"])  # noqa: E731
    while True:
        rows, d = _log(rng, 1, 8192), _log(rng, 8, 8192)
        if rng.random() < 0.6:
            d = max(8, d // 8 * 8)
        if op == "norm":
            c = dict(op=op, mode=rng.choice(["fwd", "train", "train"]), rows=rows, d=d, pad=rng.choice([0, 0, 1, 8]), x=t(),
                     s=t(), y=t(), dx=t(), p=p)
            if c["mode"] == "train" and rows < 16:
                continue
        elif op == "dropout":
            c = dict(op=op, rows=rows, d=d, pad=rng.choice([0, 0, 1, 8]), x=t(), p=rng.choice([0.05, 0.1, 0.3, 0.5, 0.9]))
        elif op == "quant":
            c = dict(op=op, rows=rows, d=d, x=t(), f=rng.choice(["e4m3", "e5m2"]))
        else:
            c = dict(op=op, mode=rng.choice(["serve", "norm", "train", "train"]), rows=rows, d=max(d, 64),
                     n=_log(rng, 64, 8192), f="e4m3", g=rng.choice(["e4m3", "e5m2"]))
            if c["mode"] == "serve":
                c["rows"] = _log(rng, 1, 256)
        w, top = work(c), work(listed()[3] if op != "linear" else listed()[-1])
        if w["bytes"] <= top["bytes"] and w["flops"] <= max(top["flops"], 1.0):
            return c


# ------------------------------------------------------------------- inputs


def _up(n, q):
    return (n + q - 1) // q * q


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, pad=0, std=1.0, mean=0.0):
    """A matrix of normal values whose rows lie shape[1] + pad apart."""
    m = torch.randn((shape[0], shape[1] + pad), device=DEV, generator=g, dtype=torch.float32)
    return m.mul_(std).add_(mean).to(dtype)[:, : shape[1]]


def _room(rows, d, dtype, pad=0):
    return torch.empty((rows, d + pad), device=DEV, dtype=dtype)[:, :d]


def _scales(rows, k):
    """A table of scale bytes: a row of it is a multiple of four bytes."""
    return torch.zeros((rows, _up(-(-k // 128), 4)), device=DEV, dtype=torch.uint8)


def _room8(rows, k, fmt):
    """8-bit values whose rows are filled up to a multiple of 128."""
    return torch.zeros((rows, _up(k, 128)), device=DEV, dtype=torch.uint8).view(FP8[fmt])


def _activations(g, rows, d, dtype=torch.bfloat16):
    """What a block's activations look like: a few channels are much larger than the rest."""
    loud = torch.where(torch.rand(d, device=DEV, generator=g) < 0.01, 8.0, 1.0)
    return (torch.randn((rows, d), device=DEV, generator=g) * loud).to(dtype)


def prepare(c, seed):
    g = _gen(seed)
    s = dict(case=c, seed=(0x9E3779B97F4A7C15 * (seed + 1)) & ((1 << 63) - 1), offset=3 * seed + 7)
    rows, d = c["rows"], c["d"]
    if c["op"] == "dropout":
        t = TYPES[c["x"]]
        s.update(x=_normal(g, (rows, d), t, c["pad"]), out=_room(rows, d, t, c["pad"]))
    elif c["op"] == "quant":
        s.update(x=_normal(g, (rows, d), TYPES[c["x"]], 0, 0.02), q=_room8(rows, d, c["f"]), qt=_room8(d, rows, c["f"]),
                 scale=_scales(-(-rows // 128), d), scale_t=_scales(-(-d // 128), rows))
    elif c["op"] == "norm" or c["mode"] == "norm":
        tx, ts, ty, tdx = (TYPES[c.get(k, v)] for k, v in (("x", "bf16"), ("s", "f32"), ("y", "bf16"), ("dx", "bf16")))
        pad = c.get("pad", 0)
        s.update(x=_normal(g, (rows, d), tx, pad), residual=_normal(g, (rows, d), ts, pad, 2.0, 0.3),
                 gamma=1.0 + 0.1 * torch.randn(d, device=DEV, generator=g), beta=0.1 * torch.randn(d, device=DEV, generator=g),
                 sum=_room(rows, d, ts, pad))
        if c["op"] == "norm":
            s.update(y=_room(rows, d, ty, pad))
        if c.get("mode") == "train":
            f32 = dict(device=DEV, dtype=torch.float32)
            s.update(mean=torch.empty(rows, **f32), rstd=torch.empty(rows, **f32), dgamma=torch.empty(d, **f32),
                     dbeta=torch.empty(d, **f32), dy=_normal(g, (rows, d), ty, pad, 0.01), dsum=_normal(g, (rows, d), ts, pad, 0.01),
                     dres=_room(rows, d, ts, pad), dx=_room(rows, d, tdx, pad))
    if c["op"] == "linear":
        n = c["n"]
        w = _normal(g, (n, d), torch.bfloat16, 0, 0.02)
        s.update(bias=0.1 * torch.randn(n, device=DEV, generator=g), out=_room(rows, n, torch.bfloat16),
                 q=_room8(rows, d, c["f"]), scale=_scales(rows, d), room=torch.empty(64 << 20, device=DEV, dtype=torch.uint8))
        if c["mode"] == "train":
            # gradients of tokens whose losses differ by orders of magnitude
            size = torch.exp(2.0 * torch.randn((rows, 1), device=DEV, generator=g))
            s.update(x=_activations(g, rows, d), w=w, dy=(1e-4 * size * torch.randn((rows, n), device=DEV, generator=g)).to(torch.bfloat16),
                     dx=_room(rows, d, torch.bfloat16), dw=_room(n, d, torch.float32),
                     xt=_room8(d, rows, c["f"]), xt_scale=_scales(d, rows), wq=_room8(n, d, c["f"]), wq_scale=_scales(-(-n // 128), d),
                     wt=_room8(d, n, c["f"]), wt_scale=_scales(-(-d // 128), n), gq=_room8(rows, n, c["g"]), gq_scale=_scales(rows, n),
                     gt=_room8(n, rows, c["g"]), gt_scale=_scales(n, rows))
        else:
            # the weight as a checkpoint in 8 bits holds it
            wq, e = _quant_plain(w.float(), 128, c["f"])
            s.update(wq=_room8(n, d, c["f"]), wq_scale=_scales(-(-n // 128), d))
            s["wq"].view(torch.uint8)[:, :d] = wq.view(torch.uint8)
            s["wq_scale"][:, : e.shape[1]] = e
            if c["mode"] == "serve":
                s.update(x=_activations(g, rows, d))
    return s


# ------------------------------------------------------- the framework's calls


def _plan(s):
    """The call descriptors that a program builds once and keeps beside its buffers."""
    from paper_2410_05985_amd import layup as LU
    c, calls = s["case"], []
    if c["op"] == "dropout":
        calls.append((LU.layup_dropout, LU.dropout_desc(s["x"], s["out"], p=c["p"], seed=s["seed"], offset=s["offset"])))
    elif c["op"] == "quant":
        calls.append((LU.layup_quant_fp8, LU.quant_desc(s["x"], 128, q=s["q"], scale=s["scale"], qt=s["qt"], scale_t=s["scale_t"])))
    elif c["op"] == "norm":
        drop = dict(p=c["p"], seed=s["seed"], offset=s["offset"])
        calls.append((LU.layup_layernorm_forward,
                      LU.layernorm_desc(s["x"], s["y"], s["gamma"], s["beta"], residual=s["residual"], sum_out=s["sum"],
                                        mean=s.get("mean"), rstd=s.get("rstd"), eps=EPS, **drop)))
        if c["mode"] == "train":
            s["room"] = torch.empty(max(1, LU.layup_layernorm_workspace_size(c["rows"], c["d"])), device=DEV, dtype=torch.uint8)
            calls.append((LU.layup_layernorm_backward,
                          LU.layernorm_grad_desc(s["dy"], s["sum"], s["mean"], s["rstd"], s["gamma"], dsum=s["dsum"], dres=s["dres"],
                                                 dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"], workspace=s["room"], **drop)))
    else:
        gemm = lambda a, sa, ra, b, sb, rb, out, k, bias=None: (  # noqa: E731
            LU.layup_gemm_fp8, LU.gemm_fp8_desc(a, sa, ra, b, sb, rb, out, k, bias=bias, workspace=s["room"]))
        rows, d, n = c["rows"], c["d"], c["n"]
        if c["mode"] == "norm":
            calls.append((LU.layup_layernorm_forward,
                          LU.layernorm_desc(s["x"], s["q"], s["gamma"], s["beta"], residual=s["residual"], sum_out=s["sum"], eps=EPS,
                                            y_scale=s["scale"])))
        elif c["mode"] == "serve":
            calls.append((LU.layup_quant_fp8, LU.quant_desc(s["x"], 1, q=s["q"], scale=s["scale"])))
        else:
            calls.append((LU.layup_quant_fp8, LU.quant_desc(s["x"], 1, q=s["q"], scale=s["scale"], qt=s["xt"], scale_t=s["xt_scale"])))
            calls.append((LU.layup_quant_fp8, LU.quant_desc(s["w"], 128, q=s["wq"], scale=s["wq_scale"], qt=s["wt"], scale_t=s["wt_scale"])))
        calls.append(gemm(s["q"], s["scale"], 1, s["wq"], s["wq_scale"], 128, s["out"], d, s["bias"]))
        if c["mode"] == "train":
            calls.append((LU.layup_quant_fp8, LU.quant_desc(s["dy"], 1, q=s["gq"], scale=s["gq_scale"], qt=s["gt"], scale_t=s["gt_scale"])))
            calls.append(gemm(s["gq"], s["gq_scale"], 1, s["wt"], s["wt_scale"], 128, s["dx"], n))
            calls.append(gemm(s["gt"], s["gt_scale"], 1, s["xt"], s["xt_scale"], 1, s["dw"], rows))
    return calls


def _results(s):
    c = s["case"]
    if c["op"] == "dropout":
        return s["out"]
    if c["op"] == "quant":
        return [s["q"], s["scale"], s["qt"], s["scale_t"]]
    if c["op"] == "norm":
        out = [s["sum"], s["y"]]
        return out + [s[k] for k in ("mean", "rstd", "dres", "dx", "dgamma", "dbeta")] if c["mode"] == "train" else out
    return {"serve": [s["out"]], "norm": [s.get("sum"), s["out"]], "train": [s["out"], s.get("dx"), s.get("dw")]}[c["mode"]]


def run(s):
    if own:
        if "plan" not in s:
            s["plan"] = _plan(s)
        stream = torch.cuda.current_stream()
        for call, desc in s["plan"]:
            call(desc, stream)
        return _results(s)
    return _plain(s)


# ------------------------------------------------------------ the plain forms


def _philox_plain(rows, groups, seed, offset):
    """Philox4x32-10 of the counters (group, row, offset): four words for each group of eight columns."""
    low = 0xFFFFFFFF
    z = torch.zeros((rows, groups), device=DEV, dtype=torch.int64)
    a, b = z + torch.arange(groups, device=DEV), z + torch.arange(rows, device=DEV)[:, None]
    c, e = z + (offset & low), z + (offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        u, v = a * 0xD2511F53, c * 0xCD9E8D57  # wrapping products: the low 64 bits are the unsigned ones
        a, b, c, e = ((v >> 32) & low) ^ b ^ k0, v & low, ((u >> 32) & low) ^ e ^ k1, u & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return a, b, c, e


def _dropped_plain(x, p, seed, offset):
    """dropout(x) in 32 bits: a column keeps its value where its 16 bits are not below p."""
    if p == 0.0:
        return x
    rows, d = x.shape
    thr = min(65535, int(p * 65536 + 0.5))
    words = torch.stack(_philox_plain(rows, -(-d // 8), seed, offset), -1)
    bits = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(rows, -1)[:, :d]
    return torch.where(bits >= thr, x * (65536.0 / (65536 - thr)), 0.0)


def _norm_plain(s, p=0.0):
    c = s["case"]
    t = (s["residual"].float() + _dropped_plain(s["x"].float(), p, s["seed"], s["offset"])).to(s["residual"].dtype)
    z = t.float()
    mean = z.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((z - mean) ** 2).mean(1, keepdim=True) + EPS)
    y = (z - mean) * rstd * s["gamma"] + s["beta"]
    out = [t, y.to(TYPES[c.get("y", "f32")])]
    if c["mode"] != "train":
        return out
    xh = (z - mean) * rstd
    dy = s["dy"].float()
    a = dy * s["gamma"]
    ds = s["dsum"].float() + rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    dx = _dropped_plain(ds, p, s["seed"], s["offset"])
    return out + [mean[:, 0], rstd[:, 0], ds.to(TYPES[c["s"]]), dx.to(TYPES[c["dx"]]), (dy * xh).sum(0), dy.sum(0)]


def _quant_plain(x, block, fmt):
    """x in 8 bits, and the scale byte of each block of `block` rows by 128 columns."""
    rows, d = x.shape
    nr, nc = -(-rows // block), -(-d // 128)
    t = torch.nn.functional.pad(x, (0, nc * 128 - d, 0, nr * block - rows)).reshape(nr, block, nc, 128)
    amax = torch.where(torch.isfinite(t), t.abs(), 0.0).amax((1, 3))
    m, e = torch.frexp(amax)
    e = (e - 1 - TOP[fmt] + (m > 0.875).to(e.dtype)).clamp(-126, 127)
    e = torch.where(amax == 0, 0, e).to(torch.int32)
    inv = ((127 - e) << 23).view(torch.float32)  # 2^-e
    q = (t * inv[:, None, :, None]).reshape(nr * block, nc * 128)[:rows, :d].to(FP8[fmt])
    return q, (e + 127).to(torch.uint8)


def _value_plain(q, e, block):
    """The float32 values that 8-bit values and their scale bytes stand for."""
    scale = (e.to(torch.int32) << 23).view(torch.float32)
    scale = scale.repeat_interleave(block, 0)[: q.shape[0]].repeat_interleave(128, 1)[:, : q.shape[1]]
    return q.float() * scale


def _both_plain(x, block, fmt):
    """Values of x and of its transpose in 8 bits."""
    return [_value_plain(*_quant_plain(t, block, fmt), block) for t in (x.float(), x.float().t().contiguous())]


def _plain(s):
    c = s["case"]
    if c["op"] == "dropout":
        return _dropped_plain(s["x"].float(), c["p"], s["seed"], s["offset"]).to(s["x"].dtype)
    if c["op"] == "quant":
        (q, e), (qt, et) = (_quant_plain(x, 128, c["f"]) for x in (s["x"].float(), s["x"].float().t().contiguous()))
        out = []
        for v, k in ((q, "q"), (e, "scale"), (qt, "qt"), (et, "scale_t")):  # as wide as the buffers, zeros behind
            out.append(torch.nn.functional.pad(v.view(torch.uint8), (0, s[k].shape[1] - v.shape[1])).view(v.dtype))
        return out
    if c["op"] == "norm":
        return _norm_plain(s, c["p"])
    d, n = c["d"], c["n"]
    if c["mode"] == "train":
        x, xt = _both_plain(s["x"], 1, c["f"])
        w, wt = _both_plain(s["w"], 128, c["f"])
        g, gt = _both_plain(s["dy"], 1, c["g"])
        y = x @ w.t() + s["bias"]
        return [y.bfloat16(), (g @ wt.t()).bfloat16(), gt @ xt.t()]
    first = []
    x = s["x"].float()
    if c["mode"] == "norm":
        first, x = (lambda r: (r[:1], r[1]))(_norm_plain(s))
    x = _value_plain(*_quant_plain(x, 1, c["f"]), 1)
    w = _value_plain(s["wq"][:, :d], s["wq_scale"], 128)
    return first + [(x @ w.t() + s["bias"]).bfloat16()]


# ------------------------------------------------------------- in 64 bits


def _philox_numpy(rows, d, seed, offset):
    """The 16 bits of every column, in numpy."""
    groups = -(-d // 8)
    u = np.uint64
    low = u(0xFFFFFFFF)
    ctr = [np.broadcast_to(np.arange(groups, dtype=u), (rows, groups)),
           np.broadcast_to(np.arange(rows, dtype=u)[:, None], (rows, groups)),
           np.full((rows, groups), offset & 0xFFFFFFFF, u), np.full((rows, groups), offset >> 32, u)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for r in range(10):
        p0, p1 = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        k = [u((key[0] + r * 0x9E3779B9) & 0xFFFFFFFF), u((key[1] + r * 0xBB67AE85) & 0xFFFFFFFF)]
        ctr = [(p1 >> u(32)) ^ ctr[1] ^ k[0], p1 & low, (p0 >> u(32)) ^ ctr[3] ^ k[1], p0 & low]
    out = np.empty((rows, groups, 8), np.uint16)
    for j in range(4):
        out[:, :, 2 * j] = ctr[j] & u(0xFFFF)
        out[:, :, 2 * j + 1] = ctr[j] >> u(16)
    return out.reshape(rows, -1)[:, :d]


def _keep_exact(s, p):
    """What each element is multiplied by, as float64."""
    c = s["case"]
    if p == 0.0:
        return 1.0
    thr = min(65535, int(math.floor(p * 65536 + 0.5)))
    kept = _philox_numpy(c["rows"], c["d"], s["seed"], s["offset"]) >= thr
    return torch.from_numpy(kept).to(DEV).double() * (65536.0 / (65536.0 - thr))


def _norm_exact(s, p):
    c = s["case"]
    keep = _keep_exact(s, p)
    t = s["residual"].double() + s["x"].double() * keep
    z = t.to(s["residual"].dtype).double()  # the stream's type is what the next layer reads
    var, mean = torch.var_mean(z, 1, correction=0, keepdim=True)
    rstd = torch.rsqrt(var + EPS)
    xh = (z - mean) * rstd
    out = [t, xh * s["gamma"].double() + s["beta"].double()]
    if c["mode"] != "train":
        return out
    dy = s["dy"].double()
    a = dy * s["gamma"].double()
    ds = s["dsum"].double() + rstd / c["d"] * (c["d"] * a - a.sum(1, keepdim=True) - xh * (a * xh).sum(1, keepdim=True))
    ones = torch.ones(1, c["rows"], device=DEV, dtype=torch.float64)
    return out + [mean[:, 0], rstd[:, 0], ds, ds * keep, (ones @ (dy * xh))[0], (ones @ dy)[0]]


def _quant_exact(x, block, fmt):
    """(8-bit values as float64, exponents) of blocks of `block` rows by 128 columns: the smallest power of two that
    brings the block's largest value under the format's."""
    rows, d = x.shape
    big = 1.75 * 2.0 ** TOP[fmt]
    top = x.double().abs()
    top = torch.nn.functional.max_pool2d(top[None, None], (block, 128), ceil_mode=True)[0, 0]
    e = torch.ceil(torch.log2(top / big))
    e = torch.where(top > big * torch.exp2(e), e + 1, torch.where(top <= big * torch.exp2(e - 1), e - 1, e))
    e = torch.where(top == 0, 0.0, e.clamp(-126, 127))
    each = e.repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :d]
    v = x.double() * torch.exp2(-each)
    bits, least = (3, -6) if fmt == "e4m3" else (2, -14)
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** least))) - bits)
    return torch.round(v / step) * step, e, each  # torch.round goes to even


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "dropout":
        return s["x"].double() * _keep_exact(s, c["p"])
    if c["op"] == "quant":
        out = []
        for x, q, sc in ((s["x"], "q", "scale"), (s["x"].t().contiguous(), "qt", "scale_t")):
            v, _, _ = _quant_exact(x, 128, c["f"])
            out += [torch.nn.functional.pad(v, (0, s[q].shape[1] - v.shape[1])), None]
        return out
    if c["op"] == "norm":
        return _norm_exact(s, c["p"])
    value = lambda x, block, f: (lambda v, e, each: v * torch.exp2(each))(*_quant_exact(x, block, f))  # noqa: E731
    if c["mode"] == "train":
        x, w, g = s["x"], s["w"], s["dy"]
        t = lambda m: m.t().contiguous()  # noqa: E731
        y = value(x, 1, c["f"]) @ t(value(w, 128, c["f"])) + s["bias"].double()
        dx = value(g, 1, c["g"]) @ value(w, 128, c["f"])
        dw = value(t(g), 1, c["g"]) @ t(value(t(x), 1, c["f"]))
        return [y, dx, dw]
    first, x = [], s["x"]
    if c["mode"] == "norm":
        first, x = (lambda r: (r[:1], r[1]))(_norm_exact(s, 0.0))
    e = s["wq_scale"].double().repeat_interleave(128, 0)[: c["n"]].repeat_interleave(128, 1)[:, : c["d"]]
    w = s["wq"][:, : c["d"]].double() * torch.exp2(e - 127.0)
    return first + [value(x, 1, c["f"]) @ w.t().contiguous() + s["bias"].double()]


# ------------------------------------------------------------------- work


def work(c):
    rows, d = c["rows"], c["d"]
    e = rows * d
    if c["op"] == "dropout":
        return dict(bytes=2 * e * SIZE[c["x"]], flops=0)
    if c["op"] == "quant":
        return dict(bytes=e * (SIZE[c["x"]] + 2), flops=0)
    norm = e * (SIZE[c.get("x", "bf16")] + 2 * SIZE[c.get("s", "f32")]) + 8 * d  # x, residual, sum, gain and bias
    if c["op"] == "norm":
        b = norm + e * SIZE[c["y"]]
        if c["mode"] == "train":  # dy, the sum, its gradient in and out, dx; gain, its gradients, statistics
            b += e * (SIZE[c["y"]] + 3 * SIZE[c["s"]] + SIZE[c["dx"]]) + 12 * d + 16 * rows
        return dict(bytes=b, flops=0)
    n = c["n"]
    if c["mode"] == "train":  # x, w, dy in; y, dx, dw out
        return dict(bytes=2 * e + 2 * n * d + 2 * rows * n + 4 * n + 2 * rows * n + 2 * e + 4 * n * d, flops=6 * rows * d * n)
    b = (norm if c["mode"] == "norm" else 2 * e) + n * d + 4 * n + 2 * rows * n
    return dict(bytes=b, flops=2 * rows * d * n)
