"""The operators of a training step beside the forward layers, at the sizes programs call them.

Three operators: LayerNorm over rows of the single or the pair track, its backward pass with
the reduction of the affine weights' gradients, and the backward pass of the pair-biased gated
attention, which recomputes the probabilities from the inputs and the softmax state (m, l, acc)
that the forward saved. Inputs are synthetic: N(0, 1) activations with a channel offset,
N(0, 1/fan_in) weights, affine LayerNorms, gradients of a mean over the rows.

A case is a dict with a ``kind`` and that kind's sizes. ``run`` computes it from elementary
operations in 32 bits, or, where ``own`` is set, through the library's entry points.
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# The token-level attention's widths: the bf16 workloads', and the fp32 workload's.
BF16_WIDTHS = {"dtype": "bf16", "c_s": 384, "c_z": 128, "heads": 16, "head_dim": 24}
F32_WIDTHS = {"dtype": "f32", "c_s": 128, "c_z": 32, "heads": 4, "head_dim": 32}


def listed():
    return [
        # the single track of one protein of odd length, before its attention: latency counts
        {"name": "ln_bf16_tokens333", "kind": "ln", "dtype": "bf16", "rows": 333, "c": 384},
        # the fp32 workload's pair track
        {"name": "ln_f32_pairs128", "kind": "ln", "dtype": "f32", "rows": 128 * 128, "c": 32},
        # the whole pair track of a 1024-token layer
        {"name": "ln_bf16_pairs1024", "kind": "ln", "dtype": "bf16", "rows": 1024 * 1024, "c": 128},
        # gradients of the fp32 workload's single track: 128 rows, little but latency
        {"name": "ln_back_f32_tokens128", "kind": "ln_back", "dtype": "f32", "rows": 128, "c": 128},
        # gradients of the single track of a 24000-token assembly
        {"name": "ln_back_bf16_tokens24000", "kind": "ln_back", "dtype": "bf16", "rows": 24000, "c": 384},
        # gradients of the pair track of a 1024-token layer, the weights' summed over a million rows
        {"name": "ln_back_bf16_pairs1024", "kind": "ln_back", "dtype": "bf16", "rows": 1024 * 1024, "c": 128},
        # a training step's attention in the fp32 workload's widths: a chain of short kernels
        {"name": "attn_back_f32_n128", "kind": "attn_back", **F32_WIDTHS, "n": 128, "row0": 0, "rows": 128,
         "masked": 0},
        # an fp32 layer of a small complex at the pair track's full width, ragged, some padding
        {"name": "attn_back_f32_n601", "kind": "attn_back", "dtype": "f32", "c_s": 128, "c_z": 128, "heads": 4,
         "head_dim": 32, "n": 601, "row0": 0, "rows": 601, "masked": 9},
        # fine-tuning on one protein of odd length
        {"name": "attn_back_bf16_n333", "kind": "attn_back", **BF16_WIDTHS, "n": 333, "row0": 0, "rows": 333,
         "masked": 0},
        # 12 copies of an 85-residue subunit plus 4 padding tokens
        {"name": "attn_back_bf16_n1024", "kind": "attn_back", **BF16_WIDTHS, "n": 1024, "row0": 0, "rows": 1024,
         "masked": 4},
        # half the query rows of 60 copies of an 80-residue subunit, 5% of the keys masked
        {"name": "attn_back_bf16_half4800", "kind": "attn_back", **BF16_WIDTHS, "n": 4800, "row0": 2400, "rows": 2400,
         "masked": 240},
        # one of 16 query stripes of a 60 x 200 assembly
        {"name": "attn_back_bf16_stripe12000", "kind": "attn_back", **BF16_WIDTHS, "n": 12000, "row0": 3750,
         "rows": 750, "masked": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["ln", "ln_back", "attn_f32", "attn_bf16", "attn_bf16", "stripe"])
    if kind in ("ln", "ln_back"):
        c = rng.choice([32, 64, 128, 128, 384]) if rng.random() < 0.7 else _log(rng, 7, 1500)
        return {"kind": kind, "dtype": rng.choice(["bf16", "f32"]), "rows": _log(rng, 20, min(1 << 20, (1 << 26) // c)),
                "c": c}
    if kind == "attn_f32":
        n = _log(rng, 60, 900)
        h, d = rng.choice([(4, 32), (4, 32), (8, 16), (4, 16)])
        return {"kind": "attn_back", "dtype": "f32", "c_s": rng.choice([64, 128]), "c_z": rng.choice([32, 64, 128]),
                "heads": h, "head_dim": d, "n": n, "row0": 0, "rows": n, "masked": rng.choice([0, n // 20])}
    if kind == "attn_bf16":
        n = _log(rng, 100, 3300)
        return {"kind": "attn_back", **BF16_WIDTHS, "n": n, "row0": 0, "rows": n,
                "masked": rng.choice([0, 4, n // 20])}
    n = _log(rng, 2000, 12000)
    parts = rng.choice([16, 20, 25])
    rows = n // parts
    return {"kind": "attn_back", **BF16_WIDTHS, "n": n, "row0": rows * rng.randrange(parts), "rows": rows,
            "masked": rng.choice([0, n // 50])}


# ----------------------------------------------------------------------------- inputs
def _normal(g, shape, dtype=torch.float32, scale=1.0):
    x = torch.randn(shape, generator=g, dtype=dtype, device="cuda")
    return x if scale == 1.0 else x.mul_(scale)


def _track(g, rows, c, dt):
    """Activations with a mean of their own per channel, as a residual stream has."""
    return _normal(g, (rows, c), dt).add_(_normal(g, (c,), dt, 0.5))


def _inputs(case, seed):
    """The case's tensors, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 2)
    dt = DTYPES[case["dtype"]]
    if case["kind"] in ("ln", "ln_back"):
        x = {"x": _track(g, case["rows"], case["c"], dt), "gamma": 1.0 + _normal(g, (case["c"],), scale=0.25),
             "beta": _normal(g, (case["c"],), scale=0.25)}
        if case["kind"] == "ln_back":
            x["dy"] = _normal(g, (case["rows"], case["c"]), dt, 2.0 ** -10)
        return x
    n, rows, c_s, c_z, h, d = (case[k] for k in ("n", "rows", "c_s", "c_z", "heads", "head_dim"))
    x = {name: _normal(g, (h * d, c_s), scale=c_s ** -0.5) for name in ("w_q", "w_k", "w_v", "w_g")}
    x["w_b"] = _normal(g, (h, c_z), scale=c_z ** -0.5)
    x["gamma"] = 1.0 + _normal(g, (c_z,), scale=0.25)
    x["s"] = _normal(g, (n, c_s), dt)
    x["z"] = _track(g, rows * n, c_z, dt).view(rows, n, c_z)
    x["dout"] = _normal(g, (rows, h * d), dt, 2.0 ** -10)
    x["mask"] = None
    if case["masked"]:
        x["mask"] = torch.ones(n, dtype=torch.uint8, device="cuda")
        x["mask"][torch.randperm(n, generator=g, device="cuda")[:case["masked"]]] = 0
    return x


def _heads(x, h, d):
    return x.view(x.shape[0], h, d).permute(1, 0, 2).contiguous()  # [h, rows, d]


def _saved_state(case, x):
    """m, l [h, rows] and acc [rows, h, d], as a forward pass over all keys leaves them. The logits
    leave out the per-head constants that LayerNorm's beta and the bias projection's bias add."""
    rows, row0, h, d = (case[k] for k in ("rows", "row0", "heads", "head_dim"))
    s = x["s"].float()
    k, v = _heads(s @ x["w_k"].T, h, d), _heads(s @ x["w_v"].T, h, d)
    w = x["w_b"] * x["gamma"]
    m, l = (torch.empty((h, rows), device="cuda") for _ in range(2))
    acc = torch.empty((rows, h, d), device="cuda")
    step = max(1, (1 << 21) // case["n"])
    for r in range(0, rows, step):
        e = min(r + step, rows)
        z = x["z"][r:e].float()
        z = z - z.mean(dim=2, keepdim=True)
        z = z * torch.rsqrt(z.square().mean(dim=2, keepdim=True) + EPS)
        q = _heads(s[row0 + r:row0 + e] @ x["w_q"].T, h, d)
        logits = torch.bmm(q, k.transpose(1, 2).contiguous()) * d ** -0.5 + (z @ w.T).permute(2, 0, 1)
        if x["mask"] is not None:
            logits.masked_fill_(x["mask"] == 0, -math.inf)
        m[:, r:e] = logits.max(dim=2).values
        p = torch.exp(logits - m[:, r:e, None])
        l[:, r:e] = p.sum(dim=2)
        acc[r:e] = torch.bmm(p, v).permute(1, 0, 2)
    return m, l, acc


def prepare(case, seed):
    x = _inputs(case, seed)
    st = {"case": case, "x": x, "kept": {}}
    if case["kind"] == "attn_back":
        x["m"], x["l"], x["acc"] = _saved_state(case, x)
    return st


# ----------------------------------------------------------------------------- the library's calls
def _kept(st, name, make):
    """A buffer that a program allocates once: outputs and workspaces."""
    if name not in st["kept"]:
        st["kept"][name] = make()
    return st["kept"][name]


def _workspace(st, size):
    return _kept(st, "workspace", lambda: torch.empty(max(size(), 256), dtype=torch.uint8, device="cuda"))


def _own_layer_norm(st):
    import paper_2607_05439_amd as dcp
    case, x = st["case"], st["x"]
    code = dcp.DCP_BF16 if case["dtype"] == "bf16" else dcp.DCP_F32
    y = _kept(st, "y", lambda: torch.empty_like(x["x"]))
    dcp.dcp_layer_norm(case["rows"], case["c"], code, code, EPS, x["x"], x["gamma"], x["beta"], y)
    return y


def _own_layer_norm_backward(st):
    import paper_2607_05439_amd as dcp
    case, x = st["case"], st["x"]
    code = dcp.DCP_BF16 if case["dtype"] == "bf16" else dcp.DCP_F32
    dx = _kept(st, "dx", lambda: torch.empty_like(x["x"]))
    dgamma = _kept(st, "dgamma", lambda: torch.empty_like(x["gamma"]))
    dbeta = _kept(st, "dbeta", lambda: torch.empty_like(x["beta"]))
    ws = _workspace(st, lambda: dcp.dcp_layer_norm_backward_workspace_size(case["rows"], case["c"]))
    dcp.dcp_layer_norm_backward(case["rows"], case["c"], code, code, EPS, x["x"], x["gamma"], x["dy"], dx, dgamma,
                                dbeta, ws, ws.numel())
    return dx, dgamma, dbeta


def _own_attention_backward(st):
    import paper_2607_05439_amd as dcp
    case, x = st["case"], st["x"]
    code, dt = (dcp.DCP_BF16 if case["dtype"] == "bf16" else dcp.DCP_F32), DTYPES[case["dtype"]]

    def plan():
        shape = dcp.make_shape(case["n"], case["c_s"], case["c_z"], case["heads"], case["head_dim"], code, code, EPS)
        weights = dcp.make_weights(x["w_q"], x["w_k"], x["w_v"], x["w_g"], x["w_b"], None, x["gamma"], None)
        out = [torch.empty_like(x["z"]), torch.empty_like(x["s"])]
        out += [torch.empty_like(x[k], dtype=dt) for k in ("w_q", "w_k", "w_v", "w_g", "w_b", "gamma")]
        return shape, weights, out, dcp.make_gradients(*out, dtype=code)

    shape, weights, out, grads = _kept(st, "plan", plan)
    ws = _workspace(st, lambda: dcp.dcp_pair_bias_attention_backward_workspace_size(shape, case["rows"]))
    dcp.dcp_pair_bias_attention_backward(shape, weights, x["s"], x["z"], x["mask"], case["row0"], case["rows"],
                                         x["m"], x["l"], x["acc"], x["dout"], grads, ws, ws.numel())
    return out


# ----------------------------------------------------------------------------- the plain forms
def _normalised(x):
    x = x - x.mean(dim=-1, keepdim=True)
    rstd = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS)
    return x * rstd, rstd


def _plain_layer_norm(st):
    x = st["x"]
    xh, _ = _normalised(x["x"].float())
    return (xh * x["gamma"] + x["beta"]).to(x["x"].dtype)


def _plain_layer_norm_backward(st):
    x = st["x"]
    xh, rstd = _normalised(x["x"].float())
    dy = x["dy"].float()
    g = dy * x["gamma"]
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))
    # the rows' sums in 64 bits: a million terms that mostly cancel
    return (dx.to(x["x"].dtype), (dy * xh).sum(dim=0, dtype=torch.float64).float(),
            dy.sum(dim=0, dtype=torch.float64).float())


def _plain_attention_backward(st):
    case, x = st["case"], st["x"]
    n, rows, row0, c_z, h, d = (case[k] for k in ("n", "rows", "row0", "c_z", "heads", "head_dim"))
    dt = x["s"].dtype
    s = x["s"].float()
    sq = s[row0:row0 + rows]
    q, k, v = _heads(sq @ x["w_q"].T, h, d), _heads(s @ x["w_k"].T, h, d), _heads(s @ x["w_v"].T, h, d)
    gate = torch.sigmoid(sq @ x["w_g"].T).view(rows, h, d)
    zh, rstd = _normalised(x["z"].float())
    w = x["w_b"] * x["gamma"]
    logits = torch.bmm(q, k.transpose(1, 2).contiguous()) * d ** -0.5 + (zh.view(-1, c_z) @ w.T).view(rows, n, h).permute(2, 0, 1)
    p = torch.exp(logits - x["m"][:, :, None]) / x["l"][:, :, None]
    if x["mask"] is not None:
        p = p * (x["mask"] != 0)
    o = x["acc"] / x["l"].T[:, :, None]
    dout = x["dout"].float().view(rows, h, d)
    do = gate * dout
    dg = (dout * o * gate * (1.0 - gate)).view(rows, h * d)
    dot = (do * o).sum(dim=2)
    do = do.permute(1, 0, 2).contiguous()
    ds_ = p * (torch.bmm(do, v.transpose(1, 2).contiguous()) - dot.T[:, :, None])  # [h, rows, n]
    dq = (torch.bmm(ds_, k) * d ** -0.5).permute(1, 0, 2).reshape(rows, h * d)
    dk = (torch.bmm(ds_.transpose(1, 2).contiguous(), q) * d ** -0.5).permute(1, 0, 2).reshape(n, h * d)
    dv = torch.bmm(p.transpose(1, 2).contiguous(), do).permute(1, 0, 2).reshape(n, h * d)
    ds = dk @ x["w_k"] + dv @ x["w_v"]
    ds[row0:row0 + rows] += dq @ x["w_q"] + dg @ x["w_g"]
    db = ds_.permute(1, 2, 0).reshape(rows * n, h)
    t = db.T.contiguous() @ zh.view(-1, c_z)  # [h, c_z]
    dzh = (db @ w).view(rows, n, c_z)
    dz = rstd * (dzh - dzh.mean(dim=2, keepdim=True) - zh * (dzh * zh).mean(dim=2, keepdim=True))
    return [dz.to(dt), ds.to(dt), (dq.T @ sq).to(dt), (dk.T @ s).to(dt), (dv.T @ s).to(dt), (dg.T @ sq).to(dt),
            (x["gamma"] * t).to(dt), (x["w_b"] * t).sum(dim=0).to(dt)]


def run(st):
    kind = st["case"]["kind"]
    if kind == "ln":
        return _own_layer_norm(st) if own else _plain_layer_norm(st)
    if kind == "ln_back":
        return _own_layer_norm_backward(st) if own else _plain_layer_norm_backward(st)
    return _own_attention_backward(st) if own else _plain_attention_backward(st)


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "ln":
        return {"bytes": 2 * case["rows"] * case["c"] * size + 8 * case["c"], "flops": 7 * case["rows"] * case["c"]}
    if case["kind"] == "ln_back":
        return {"bytes": 3 * case["rows"] * case["c"] * size + 12 * case["c"], "flops": 16 * case["rows"] * case["c"]}
    n, rows, c_s, c_z, h, d = (case[k] for k in ("n", "rows", "c_s", "c_z", "heads", "head_dim"))
    valid, hd = n - case["masked"], h * d
    return {"bytes": rows * (valid + n) * c_z * size  # z of the keys that count, dz of all
            + 2 * n * c_s * size + 4 * hd * c_s * (4 + size) + h * c_z * (4 + size)  # s, ds, weights and their gradients
            + rows * (hd * (4 + size) + 8 * h),  # acc, dout, m, l
            # per pair: LayerNorm and its gradient, the bias and its two gradients, logits, dP, dq, dk, dv,
            # softmax; per token: q, k, v, g and two products of each projection's gradient
            "flops": rows * valid * (8 * c_z + 6 * h * c_z + 10 * hd + 12 * h) + 12 * (rows + n) * hd * c_s}


# ----------------------------------------------------------------------------- the same in 64 bits
def _layer(s, z, mask, row0, w, h, d):
    """The attention layer's output rows from its definition (the oracle of its gradients)."""
    rows, n = z.shape[:2]
    var, mu = torch.var_mean(z, dim=2, keepdim=True, correction=0)
    bias = ((z - mu) / (var + EPS).sqrt() * w["gamma"]) @ w["w_b"].T  # [rows, n, h]
    sq = s[row0:row0 + rows]
    q = (sq @ w["w_q"].T).view(rows, h, d).transpose(0, 1)
    k = (s @ w["w_k"].T).view(n, h, d).permute(1, 2, 0)
    v = (s @ w["w_v"].T).view(n, h, d).transpose(0, 1)
    logits = q @ k / math.sqrt(d) + bias.permute(2, 0, 1)
    if mask is not None:
        logits = logits.masked_fill(mask == 0, -math.inf)
    o = torch.softmax(logits, dim=2) @ v
    return torch.sigmoid(sq @ w["w_g"].T) * o.transpose(0, 1).reshape(rows, h * d)


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] == "ln":
        v = x["x"].double()
        var, mu = torch.var_mean(v, dim=1, keepdim=True, correction=0)
        return (v - mu) / (var + EPS).sqrt() * x["gamma"].double() + x["beta"].double()
    if case["kind"] == "ln_back":
        v, gamma, beta = (x[k].double().requires_grad_() for k in ("x", "gamma", "beta"))
        var, mu = torch.var_mean(v, dim=1, keepdim=True, correction=0)
        y = (v - mu) / (var + EPS).sqrt() * gamma + beta
        return torch.autograd.grad(y, [v, gamma, beta], x["dy"].double())
    names = ("w_q", "w_k", "w_v", "w_g", "w_b", "gamma")
    w = {k: x[k].double().requires_grad_() for k in names}
    s = x["s"].double().requires_grad_()
    rows, step = case["rows"], max(1, (1 << 20) // case["n"])
    dz = torch.empty(x["z"].shape, dtype=torch.float64, device="cuda")
    total = [torch.zeros_like(s)] + [torch.zeros_like(w[k]) for k in names]
    for r in range(0, rows, step):
        e = min(r + step, rows)
        z = x["z"][r:e].double().requires_grad_()
        out = _layer(s, z, x["mask"], case["row0"] + r, w, case["heads"], case["head_dim"])
        grads = torch.autograd.grad(out, [z, s] + [w[k] for k in names], x["dout"][r:e].double())
        dz[r:e] = grads[0]
        total = [a + b for a, b in zip(total, grads[1:])]
    return [dz] + total
