"""The work that the layer operators are measured on: norms, linear layers and merge-coefficient gradients.

A case is one pass through one operator:

* "norm_fwd", "norm_bwd", "norm_step"  layer norm or RMS norm of a matrix of rows, its backward pass from
                      saved statistics, and both in turn;
* "linear_fwd", "linear_bwd"  act(x w^T + bias) * mul + residual, with the pre-activation kept where a backward
                      pass follows, and the gradients of the inputs, weights, bias and factor;
* "coef"              the gradient of the merge coefficients, per expert and tensor, from the gradient of
                      the merged weights, over the blocks that the merge read.

With `own` false the passes are plain torch operations in 32 bits, rounded once at the end; with `own` true they
are the package's calls.  Matrices are random with the scales of a trained model: a residual stream with a few
strong channels, weights of 0.02, experts that differ from the base on an active share of the blocks.
"""
import math
import random  # noqa: F401  (the type that draw() takes)

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

# weight matrices and vectors of one transformer layer: hidden, intermediate, key/value width, biases on q, k, v
LAYERS = {"qwen2.5-0.5b": (896, 4864, 128, True), "qwen2.5-1.5b": (1536, 8960, 256, True),
          "llama-3-8b": (4096, 14336, 1024, False)}


def _norm(name, op, rows, cols, kind="rms", dtype="bf16", bias=False, add=False, pad=0):
    c = dict(op=op, rows=rows, cols=cols, kind=kind, dtype=dtype, bias=bias, add=add, pad=pad)
    return dict(c, name=name) if name else c


def _linear(name, op, rows, k, n, dtype="bf16", act="none", bias=False, mul=False, residual=False, pad=0,
            keep=False):
    c = dict(op=op, rows=rows, k=k, n=n, dtype=dtype, act=act, bias=bias, mul=mul, residual=residual, pad=pad,
             keep=keep)
    return dict(c, name=name) if name else c


def _coef(name, shape, layers, K, active, dtype="bf16", block=65536, params=0, tensors=0):
    c = dict(op="coef", shape=shape, layers=layers, K=K, active=active, dtype=dtype, block=block, params=params,
             tensors=tensors)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through a small model's norm: a launch and its latency
        _norm("rms-fwd-1x896", "norm_fwd", 1, 896),
        # calibration tokens of a large model, forward pass and backward pass in turn
        _norm("rms-step-4096x4096", "norm_step", 4096, 4096, add=True),
        # a layer norm with bias in 32 bits: odd rows and an odd width, the backward pass alone
        _norm("layer-bwd-fp32-2047x1537", "norm_bwd", 2047, 1537, kind="layer", dtype="fp32", bias=True),
        # a single token through the gated projection of a large model: the weights' bytes are the work
        _linear("gate-1x4096x14336", "linear_fwd", 1, 4096, 14336, act="silu", mul=True),
        # a handful of tokens through its down projection, added to the residual stream
        _linear("down-24x14336x4096", "linear_fwd", 24, 14336, 4096, residual=True),
        # calibration tokens through the gated projection, the pre-activation kept for the backward pass
        _linear("gate-8192x4096x14336", "linear_fwd", 8192, 4096, 14336, act="silu", mul=True, keep=True),
        # the gradients of the same projection
        _linear("gate-bwd-4096x4096x14336", "linear_bwd", 4096, 4096, 14336, act="silu", mul=True),
        # a small model's biased projection, a ragged batch of tokens, forward and backward
        _linear("qkv-fwd-777x896x1152", "linear_fwd", 777, 896, 1152, bias=True),
        _linear("fc-bwd-odd-333x901x1151", "linear_bwd", 333, 901, 1151, act="gelu", bias=True),
        # a toy layer in 32 bits
        _linear("fc-fp32-512x512x512", "linear_fwd", 512, 512, 512, dtype="fp32", act="gelu_tanh", bias=True,
                residual=True),
        # coefficients of eight experts over a few layers of a small model, each expert active on its own blocks
        _coef("coef-qwen05b-4l-k8", "qwen2.5-0.5b", 4, 8, 0.4),
        # four experts over three layers of a large model, full reads
        _coef("coef-llama8b-3l-k4", "llama-3-8b", 3, 4, 1.0),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = min(max(v, lo), hi)
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "norm_step", "linear_fwd", "linear_fwd", "linear_bwd", "linear_bwd", "coef"])
    even = rng.random() < 0.7
    fit = lambda v: max(8, v // 8 * 8) if even else v  # noqa: E731
    fit2 = lambda v: v + 8 if v == 3072 else v  # noqa: E731
    if op.startswith("norm"):
        cols = fit2(fit(_log(rng, 32, 16384)))
        rows = _log(rng, 1, max(1, min(32768, (1 << 25) // cols)))
        kind = rng.choice(["rms", "layer"])
        return _norm(None, op, rows, cols, kind, rng.choice(["bf16", "bf16", "fp32"]), kind == "layer",
                     op != "norm_fwd" and rng.random() < 0.5, rng.choice([0, 0, 8]))
    if op.startswith("linear"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        top = 14336 if dtype == "bf16" else 2048
        k, n = fit2(fit(_log(rng, 48, top))), fit2(fit(_log(rng, 48, top)))
        most = (1 << 36) if dtype == "bf16" else (1 << 30)
        rows = _log(rng, 1, max(1, min(8192, most // (k * n))))
        return _linear(None, op, rows, k, n, dtype, rng.choice(["none", "silu", "gelu", "gelu_tanh", "relu"]),
                       rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.4, rng.choice([0, 0, 8]),
                       op == "linear_fwd" and rng.random() < 0.4)
    return _coef(None, "mix", 0, rng.choice([1, 2, 3, 4, 8, 11, 16]), rng.choice([0.25, 0.5, 1.0]),
                 rng.choice(["bf16", "bf16", "fp32"]), rng.choice([4096, 16384, 65536]),
                 params=_log(rng, 1 << 16, 1 << 25), tensors=_log(rng, 1, 24))


# ---- inputs -------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)


def _normal(g, shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _matrix(v, pad):
    """v as the left columns of a wider buffer: a view whose rows are `pad` elements further apart"""
    if not pad:
        return v
    wide = torch.empty(v.shape[0], v.shape[1] + pad, dtype=v.dtype, device=v.device)
    wide.fill_(float("nan"))
    wide[:, :v.shape[1]] = v
    return wide[:, :v.shape[1]]


def _tensor_sizes(case):
    if case["shape"] != "mix":
        h, f, kv, biases = LAYERS[case["shape"]]
        one = [h * h, kv * h, kv * h, h * h, f * h, f * h, h * f, h, h] + ([h, kv, kv] if biases else [])
        return one * case["layers"]
    t, left = case["tensors"], case["params"]
    weights = [(i * 7 % 11) + 1 for i in range(t)]
    return [max(1, left * w // sum(weights)) for w in weights]


def _blocks(case):
    """(blocks of each tensor, elements in the last block of each)"""
    sizes = _tensor_sizes(case)
    nb = [-(-s // case["block"]) for s in sizes]
    return sizes, nb


def _stats(x, kind, eps):
    xf = x.float()
    mean = xf.mean(1) if kind == "layer" else torch.zeros(x.shape[0], device=x.device)
    var = (xf - mean[:, None]).square().mean(1)
    return mean, (var + eps).rsqrt()


def prepare(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if case["op"].startswith("norm"):
        m, d = case["rows"], case["cols"]
        strong = torch.ones(d, device="cuda")
        strong[torch.randperm(d, generator=g, device="cuda")[:max(1, d // 100)]] = 12.0
        x = _normal(g, (m, d)) * strong + 0.1
        s["x"] = _matrix(x.to(dt), case["pad"])
        s["w"] = (1.0 + _normal(g, (d,), 0.2)).to(dt)
        s["b"] = _normal(g, (d,), 0.1, dt) if case["bias"] else None
        s["eps"] = 1e-6
        if case["op"] != "norm_fwd":
            s["dy"] = _matrix(_normal(g, (m, d), 0.01, dt), case["pad"])
            s["add"] = _normal(g, (m, d), 0.01, dt) if case["add"] else None
        if case["op"] == "norm_bwd":
            s["mean"], s["rstd"] = _stats(s["x"], case["kind"], s["eps"])
    elif case["op"].startswith("linear"):
        m, k, n = case["rows"], case["k"], case["n"]
        s["x"] = _matrix(_normal(g, (m, k), 1.0, dt), case["pad"])
        s["w"] = _normal(g, (n, k), 0.02, dt)
        s["b"] = _normal(g, (n,), 0.1, dt) if case["bias"] else None
        s["mul"] = _normal(g, (m, n), 1.0, dt) if case["mul"] else None
        s["res"] = _normal(g, (m, n), 1.0, dt) if case["residual"] else None
        if case["op"] == "linear_bwd":
            s["dy"] = _matrix(_normal(g, (m, n), 0.01, dt), case["pad"])
            # the pre-activation that the forward pass kept
            s["pre"] = _normal(g, (m, n), 0.02 * math.sqrt(k), dt) if case["act"] != "none" or case["mul"] else None
    else:
        block, K = case["block"], case["K"]
        sizes, nb = _blocks(case)
        total = sum(nb)
        length = torch.tensor([min(block, s_ - j * block) for s_, q in zip(sizes, nb) for j in range(q)], device="cuda")
        inside = torch.arange(block, device="cuda")[None, :] < length[:, None]
        base = torch.where(inside, _normal(g, (total, block), 0.02), 0.0).to(dt)
        grad = torch.where(inside, _normal(g, (total, block), 1e-3), 0.0)
        active = torch.rand((K, total), generator=g, device="cuda") < case["active"]
        scale = torch.exp(_normal(g, (K, total)) + math.log(1e-3)) * active
        experts = torch.empty((K, total, block), dtype=dt, device="cuda")
        for i in range(K):  # one expert at a time: half the memory
            delta = torch.randn((total, block), generator=g, device="cuda") * scale[i][:, None] * inside
            experts[i] = (base.float() + delta).to(dt)
            grad -= (0.2 / K) * delta
        s["base"], s["experts"], s["grad"] = base, experts, grad.to(dt)
        tensor_of = torch.repeat_interleave(torch.arange(len(nb), device="cuda"), torch.tensor(nb, device="cuda"))
        s["onehot"] = torch.nn.functional.one_hot(tensor_of, len(nb)).float()
        if own:  # what a program has in hand after its merge: the family, its catalog and the plan
            import paper_2605_29489_gb300 as mp
            first = [sum(nb[:t]) * block for t in range(len(nb))]
            s["fam"] = mp.family(list(zip(first, sizes)), base.view(-1), [experts[i].view(-1) for i in range(K)], block,
                                 mp.MP_BF16 if case["dtype"] == "bf16" else mp.MP_F32, 0)
            op = mp.make_op(mp.MP_OP_TA, alpha=[0.3] * K)
            s["index"] = mp.mp_index_blocks(s["fam"], op)
            s["plan"] = mp.mp_plan(s["index"], op, mp.mp_budget_from_fraction(s["fam"], 1.0))
    return s


# ---- the plain forms ----------------------------------------------------------------------------


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))


def _act_grad(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0.0).to(z.dtype)
    if act == "silu":
        t = 1.0 / (1.0 + torch.exp(-z))
        return t * (1.0 + z * (1.0 - t))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * z * z)


def _norm_fwd_plain(s):
    c, x = s["case"], s["x"].float()
    mean = x.mean(1) if c["kind"] == "layer" else None
    xc = x if mean is None else x - mean[:, None]
    rstd = 1.0 / torch.sqrt(xc.square().mean(1) + s["eps"])
    y = xc * rstd[:, None] * s["w"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    out = {"y": y.to(s["x"].dtype), "rstd": rstd}
    if mean is not None:
        out["mean"] = mean
    return out


def _norm_bwd_plain(s, mean, rstd):
    c, dt = s["case"], s["x"].dtype
    x, dy = s["x"].float(), s["dy"].float()
    xh = (x - mean[:, None] if c["kind"] == "layer" else x) * rstd[:, None]
    g = dy * s["w"].float()
    dx = g - xh * (g * xh).mean(1)[:, None]
    if c["kind"] == "layer":
        dx = dx - g.mean(1)[:, None]
    dx = dx * rstd[:, None]
    if s["add"] is not None:
        dx = dx + s["add"].float()
    out = {"dx": dx.to(dt), "dw": (dy * xh).sum(0).to(dt)}
    if c["bias"]:
        out["db"] = dy.sum(0).to(dt)
    return out


def _linear_fwd_plain(s):
    c, dt = s["case"], s["x"].dtype
    z = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        z = z + s["b"].float()
    y = _act(z, c["act"])
    if s["mul"] is not None:
        y = y * s["mul"].float()
    if s["res"] is not None:
        y = y + s["res"].float()
    out = {"y": y.to(dt)}
    if c["keep"]:
        out["pre"] = z.to(dt)
    return out


def _linear_bwd_plain(s):
    c, dt = s["case"], s["x"].dtype
    dz = dy = s["dy"].float()
    if s["pre"] is not None:
        z = s["pre"].float()
        dz = dz * _act_grad(z, c["act"])
    if s["mul"] is not None:
        dz = dz * s["mul"].float()
    out = {"dx": (dz @ s["w"].float()).to(dt), "dw": (dz.t() @ s["x"].float()).to(dt)}
    if c["bias"]:
        out["db"] = dz.sum(0).to(dt)
    if s["mul"] is not None:
        out["dmul"] = (dy * _act(z, c["act"])).to(dt)
    return out


def _coef_plain(s):
    delta = s["experts"].float() - s["base"].float()
    per_block = (delta * s["grad"].float()).sum(2)
    return {"grad": per_block @ s["onehot"]}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "norm_fwd":
        return _norm_fwd_plain(state)
    if op == "norm_bwd":
        return _norm_bwd_plain(state, state["mean"], state["rstd"])
    if op == "norm_step":
        y = _norm_fwd_plain(state)
        return {**y, **_norm_bwd_plain(state, y.get("mean"), y["rstd"])}
    if op == "linear_fwd":
        return _linear_fwd_plain(state)
    if op == "linear_bwd":
        return _linear_bwd_plain(state)
    return _coef_plain(state)


def _run_own(s):
    import paper_2605_29489_gb300 as mp
    c = s["case"]
    op = c["op"]
    if op.startswith("norm"):
        kind = mp.MP_NORM_LAYER if c["kind"] == "layer" else mp.MP_NORM_RMS
        out = {}
        if op == "norm_bwd":
            mean, rstd = (s["mean"] if c["kind"] == "layer" else None), s["rstd"]
        else:
            y, mean, rstd = mp.mp_norm(s["x"], s["w"], s["b"], eps=s["eps"], kind=kind)
            out = {"y": y, "rstd": rstd}
            if mean is not None:
                out["mean"] = mean
        if op != "norm_fwd":
            out["dx"], out["dw"], db = mp.mp_norm_backward(s["dy"], s["x"], s["w"], mean, rstd, kind=kind,
                                                           bias=c["bias"], add=s["add"])
            if c["bias"]:
                out["db"] = db
        return out
    if op == "coef":
        return {"grad": mp.mp_coef_grad(s["fam"], s["index"], s["plan"], s["grad"])}
    act = {"none": mp.MP_ACT_NONE, "relu": mp.MP_ACT_RELU, "silu": mp.MP_ACT_SILU, "gelu": mp.MP_ACT_GELU,
           "gelu_tanh": mp.MP_ACT_GELU_TANH}[c["act"]]
    if op == "linear_fwd":
        y, pre = mp.mp_linear(s["x"], s["w"], s["b"], act=act, mul=s["mul"], residual=s["res"],
                              keep_pre=c["keep"])
        return {"y": y} if pre is None else {"y": y, "pre": pre}
    dx, dw, db, dmul = mp.mp_linear_backward(s["dy"], s["x"], s["w"], pre=s["pre"], act=act, mul=s["mul"],
                                             bias=c["bias"])
    out = {"dx": dx, "dw": dw}
    if db is not None:
        out["db"] = db
    if dmul is not None:
        out["dmul"] = dmul
    return out


# ---- what a pass cannot do without, and its result in 64 bits ------------------------------------


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op.startswith("norm"):
        m, d = case["rows"], case["cols"]
        stats = 4 * m * (2 if case["kind"] == "layer" else 1)
        vec = es * d
        fwd = es * 2 * m * d + vec * (2 if case["bias"] else 1) + stats
        bwd = es * m * d * (4 if case["add"] else 3) + 2 * vec + stats + (vec if case["bias"] else 0)
        if op == "norm_fwd":
            return {"bytes": fwd, "flops": 6 * m * d}
        if op == "norm_bwd":
            return {"bytes": bwd, "flops": 13 * m * d}
        return {"bytes": fwd + bwd, "flops": 19 * m * d}
    if op.startswith("linear"):
        m, k, n = case["rows"], case["k"], case["n"]
        kept = case["keep"] if op == "linear_fwd" else case["act"] != "none" or case["mul"]
        mn = m * n
        if op == "linear_fwd":
            b = m * k + n * k + mn * (1 + kept + case["mul"] + case["residual"]) + (n if case["bias"] else 0)
            return {"bytes": es * b, "flops": 2 * mn * k}
        b = 2 * m * k + 2 * n * k + mn * (1 + kept + 2 * case["mul"]) + (n if case["bias"] else 0)
        return {"bytes": es * b, "flops": 4 * mn * k}
    sizes, nb = _blocks(case)
    e, K, a = sum(sizes), case["K"], case["active"]
    touched = 1.0 - (1.0 - a) ** K
    return {"bytes": es * e * (2 * touched + K * a) + 4 * K * len(sizes), "flops": 3 * e * K * a}


def exact(case, seed):
    s = prepare(case, seed)
    op, D = case["op"], torch.float64
    if op.startswith("norm"):
        x, w = s["x"].to(D), s["w"].to(D)
        mu = x.sum(1, keepdim=True) / x.shape[1] if case["kind"] == "layer" else torch.zeros_like(x[:, :1])
        var = ((x - mu) ** 2).sum(1, keepdim=True) / x.shape[1]
        r = (var + s["eps"]) ** -0.5
        out = {}
        if op == "norm_bwd":
            mu, r = s["mean"].to(D)[:, None], s["rstd"].to(D)[:, None]
        else:
            y = w * ((x - mu) * r)
            out = {"y": y if s["b"] is None else y + s["b"].to(D), "rstd": r[:, 0]}
            if case["kind"] == "layer":
                out["mean"] = mu[:, 0]
        if op != "norm_fwd":
            dy = s["dy"].to(D)
            h = (x - mu) * r
            # the product of the row's Jacobian with dy, written as two projections taken out of g
            gr = dy * w
            proj = (gr * h).sum(1, keepdim=True) / x.shape[1]
            shift = gr.sum(1, keepdim=True) / x.shape[1] if case["kind"] == "layer" else 0.0
            dx = r * (gr - shift - h * proj)
            out["dx"] = dx if s["add"] is None else dx + s["add"].to(D)
            out["dw"] = torch.einsum("md,md->d", dy, h)
            if case["bias"]:
                out["db"] = torch.einsum("md->d", dy)
        return out
    if op.startswith("linear"):
        x, w, act = s["x"].to(D), s["w"].to(D), case["act"]
        one = torch.ones((), dtype=D, device=x.device)
        root = math.sqrt(2.0)

        def parts(z):
            """(act, act') as z * p and p + z p' of the gate p"""
            if act == "none":
                return z, one.expand_as(z)
            if act == "relu":
                p = (z > 0).to(D)
                return z * p, p
            if act == "silu":
                p = torch.sigmoid(z)
                return z * p, p + z * p * (1 - p)
            if act == "gelu":
                p = torch.special.ndtr(z)
                return z * p, p + z * torch.exp(-((z / root) ** 2)) / (root * math.sqrt(math.pi))
            u = 2.0 * math.sqrt(2.0 / math.pi) * z * (1 + 0.044715 * z ** 2)
            p = torch.sigmoid(u)
            return z * p, p + z * p * (1 - p) * 2.0 * math.sqrt(2.0 / math.pi) * (1 + 3 * 0.044715 * z ** 2)

        if op == "linear_fwd":
            z = torch.mm(x, w.t())
            if s["b"] is not None:
                z += s["b"].to(D)
            y = parts(z)[0]
            if s["mul"] is not None:
                y = y * s["mul"].to(D)
            if s["res"] is not None:
                y = y + s["res"].to(D)
            return {"y": y, "pre": z} if case["keep"] else {"y": y}
        dy = s["dy"].to(D)
        z = s["pre"].to(D) if s["pre"] is not None else None
        a, da = parts(z) if z is not None else (None, one)
        dz = dy * da * (s["mul"].to(D) if s["mul"] is not None else one)
        out = {"dx": torch.mm(dz, w), "dw": torch.mm(dz.t(), x)}
        if case["bias"]:
            out["db"] = dz.sum(0)
        if case["mul"]:
            out["dmul"] = dy * a
        return out
    out = torch.zeros((case["K"], s["onehot"].shape[1]), dtype=D, device="cuda")
    b, gr = s["base"].to(D), s["grad"].to(D)
    sizes, nb = _blocks(case)
    for i in range(case["K"]):
        per_block = ((s["experts"][i].to(D) - b) * gr).sum(1)
        at = 0
        for t, q in enumerate(nb):
            out[i, t] = per_block[at:at + q].sum()
            at += q
    return {"grad": out}
