"""The operators that train the pair track beside its attention, at the sizes programs call them.

Four operators: the backward pass of the pair transition, whose input is given as it is or as an 8-bit
checkpoint; the checkpoint itself, written and read back; the relative position encoding of the pair
track, a sum of table rows by buckets of what two tokens' positions differ by; and its tables' gradient.
Inputs are synthetic: N(0, 1) activations with a channel offset, N(0, 1/fan_in) weights, affine
LayerNorms, gradients of a mean over the rows, tokens of several copies of chains.

A case is a dict with a ``kind`` and that kind's sizes. ``run`` computes it from elementary
operations in 32 bits, or, where ``own`` is set, through the library's entry points.
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32  # channels that share a power of two in a checkpoint

# The bf16 workloads' pair track and its transition, and the fp32 workload's.
BF16_TRANS = {"dtype": "bf16", "c": 128, "hidden": 512}
F32_TRANS = {"dtype": "f32", "c": 32, "hidden": 128}
# Residue and token offsets, chain hops, the same entity: the fields of the relative position encoding.
RADII = "32,32,2,0"


def listed():
    return [
        # fine-tuning on a peptide of odd length: latency counts
        {"name": "trans_back_bf16_n45", "kind": "trans_back", **BF16_TRANS, "pairs": 45 * 45, "checkpoint": False},
        # one protein of odd length
        {"name": "trans_back_bf16_n333", "kind": "trans_back", **BF16_TRANS, "pairs": 333 * 333, "checkpoint": False},
        # the whole pair track of a 1024-token layer
        {"name": "trans_back_bf16_n1024", "kind": "trans_back", **BF16_TRANS, "pairs": 1024 * 1024, "checkpoint": False},
        # a stripe of 100 rows of 4800 tokens, whose input was kept in 8 bits
        {"name": "trans_back_ckpt_bf16_stripe4800", "kind": "trans_back", **BF16_TRANS, "pairs": 100 * 4800, "checkpoint": True},
        # the fp32 workload's pair track
        {"name": "trans_back_f32_n128", "kind": "trans_back", **F32_TRANS, "pairs": 128 * 128, "checkpoint": False},
        # an fp32 model at the pair track's full width
        {"name": "trans_back_f32_n192", "kind": "trans_back", "dtype": "f32", "c": 128, "hidden": 512, "pairs": 192 * 192,
         "checkpoint": False},
        # a checkpoint of the single track of one protein, written and read back: latency counts
        {"name": "ckpt_bf16_tokens333", "kind": "ckpt", "dtype": "bf16", "rows": 333, "c": 384},
        # of the whole pair track of a 1024-token layer
        {"name": "ckpt_bf16_pairs1024", "kind": "ckpt", "dtype": "bf16", "rows": 1024 * 1024, "c": 128},
        # the fp32 workload's pair track, encoded once per pass
        {"name": "relpos_f32_n128", "kind": "relpos", "dtype": "f32", "c": 32, "n": 128, "row0": 0, "rows": 128,
         "copies": 2, "radii": RADII},
        # 12 copies of an 85-residue subunit and padding
        {"name": "relpos_bf16_n1024", "kind": "relpos", "dtype": "bf16", "c": 128, "n": 1024, "row0": 0, "rows": 1024,
         "copies": 12, "radii": RADII},
        # the tables' gradient for one protein of odd length
        {"name": "relpos_back_bf16_n333", "kind": "relpos_back", "dtype": "bf16", "c": 128, "n": 333, "row0": 0,
         "rows": 333, "copies": 1, "radii": RADII},
        # for a stripe of half the rows of 60 copies of an 80-residue subunit
        {"name": "relpos_back_bf16_half4800", "kind": "relpos_back", "dtype": "bf16", "c": 128, "n": 4800, "row0": 2400,
         "rows": 2400, "copies": 60, "radii": RADII},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["trans_bf16", "trans_bf16", "trans_f32", "ckpt", "relpos", "relpos_back"])
    if kind == "trans_bf16":
        return {"kind": "trans_back", **BF16_TRANS, "pairs": _log(rng, 300, 1 << 20), "checkpoint": rng.random() < 0.4}
    if kind == "trans_f32":
        c = rng.choice([32, 64, 128]) if rng.random() < 0.6 else rng.randrange(12, 140)
        hidden = rng.choice([2, 4]) * c
        most = min(1 << 17, (1 << 31) // (c * hidden))
        return {"kind": "trans_back", "dtype": "f32", "c": c, "hidden": hidden, "pairs": _log(rng, 300, most),
                "checkpoint": rng.random() < 0.3}
    c = rng.choice([32, 64, 128, 128]) if rng.random() < 0.7 else rng.randrange(9, 200)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "ckpt":
        c = rng.choice([c, 384])
        return {"kind": "ckpt", "dtype": dtype, "rows": _log(rng, 100, min(1 << 20, (1 << 26) // c)), "c": c}
    n = _log(rng, 60, 1800)
    rows = n if rng.random() < 0.6 else max(1, n // rng.choice([3, 4, 8]))
    radii = rng.choice([RADII, RADII, "32", "16,16", "48,32,2", "20,1,3,0"])
    return {"kind": kind, "dtype": dtype, "c": c, "n": n, "row0": rng.randrange(n - rows + 1), "rows": rows,
            "copies": rng.choice([1, 2, 3, 12, max(1, n // 80)]), "radii": radii}


# ----------------------------------------------------------------------------- inputs
def _normal(g, shape, dtype=torch.float32, scale=1.0):
    x = torch.randn(shape, generator=g, dtype=dtype, device="cuda")
    return x if scale == 1.0 else x.mul_(scale)


def _track(g, rows, c, dt):
    """Activations with a mean of their own per channel, as a residual stream has."""
    return _normal(g, (rows, c), dt).add_(_normal(g, (c,), dt, 0.5))


def _fields(case, g):
    """(positions, groups) per field, [n] int32 each: copies of one chain, whose residues are numbered
    with a few gaps and of which one in eight is split into tokens for each of its atoms."""
    n, copies = case["n"], min(case["copies"], case["n"])
    token = torch.arange(n, device="cuda")
    length = n // copies
    chain = torch.clamp(token // length, max=copies - 1)
    within = token - chain * length
    size = int(within.max()) + 1
    starts = torch.rand(size, generator=g, device="cuda") < 7 / 8
    gaps = 1 + 5 * (torch.rand(size, generator=g, device="cuda") < 0.02).long()
    number = torch.cumsum(torch.where(starts, gaps, torch.zeros_like(gaps)), dim=0)
    residue = number[within]
    entity, hop = chain % 2, chain // 2
    fields = [(residue, chain), (token, chain * (1 << 16) + residue), (hop, entity), (torch.zeros_like(token), entity)]
    return [(p.int(), q.int()) for p, q in fields[:len(case["radii"].split(","))]]


def _radii(case):
    return [int(r) for r in case["radii"].split(",")]


def _buckets(case):
    return sum(2 * r + 2 for r in _radii(case))


def _power(b):
    """2^(b - 127) of exponent bytes 1..254, from the bits of an fp32 number."""
    return (b.int() << 23).view(torch.float32)


def _blocks(x):
    """[rows, c] as [rows, blocks, 32], the last block filled up with zeros."""
    rows, c = x.shape
    return torch.nn.functional.pad(x, (0, -c % BLOCK)).view(rows, -1, BLOCK)


def _checkpoint(x):
    """Codes [rows, c] and exponents [rows, blocks]: in each block the least power of two of at least
    2^-126 by which no code is over 127, and the values over it, rounded to the nearest (even) number."""
    blocks = _blocks(x.float())
    top = blocks.abs().amax(dim=2)
    e = torch.where(top > 0, torch.frexp(top).exponent - 7, -126).clamp(min=-126)
    e = e + (torch.round(top / _power(e + 127)) > 127)
    codes = torch.round(blocks / _power(e + 127)[:, :, None])
    return codes.view(x.shape[0], -1)[:, :x.shape[1]].to(torch.int8).contiguous(), (e + 127).to(torch.uint8)


def _values(codes, exponents):
    return (_blocks(codes.float()) * _power(exponents)[:, :, None]).view(codes.shape[0], -1)[:, :codes.shape[1]]


def _inputs(case, seed):
    """The case's tensors, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 5)
    dt, c = DTYPES[case["dtype"]], case["c"]
    if case["kind"] == "ckpt":
        return {"x": _track(g, case["rows"], c, dt)}
    if case["kind"] == "trans_back":
        pairs, hidden = case["pairs"], case["hidden"]
        x = {"w1": _normal(g, (hidden, c), scale=c ** -0.5), "w2": _normal(g, (hidden, c), scale=c ** -0.5),
             "w3": _normal(g, (c, hidden), scale=hidden ** -0.5), "gamma": 1.0 + _normal(g, (c,), scale=0.25),
             "beta": _normal(g, (c,), scale=0.25), "z": _track(g, pairs, c, dt),
             "dout": _normal(g, (pairs, c), dt, 2.0 ** -10), "exponents": None}
        if case["checkpoint"]:
            x["z"], x["exponents"] = _checkpoint(x["z"])
        return x
    x = {"fields": _fields(case, g)}
    if case["kind"] == "relpos":
        x["table"] = _normal(g, (_buckets(case), c))
        x["z"] = _track(g, case["rows"] * case["n"], c, dt).view(case["rows"], case["n"], c)
    else:
        x["dz"] = _normal(g, (case["rows"], case["n"], c), dt, 2.0 ** -10)
    return x


def prepare(case, seed):
    return {"case": case, "x": _inputs(case, seed), "kept": {}}


# ----------------------------------------------------------------------------- the library's calls
def _kept(st, name, make):
    """What a program makes once: outputs, workspaces, descriptors."""
    if name not in st["kept"]:
        st["kept"][name] = make()
    return st["kept"][name]


def _workspace(st, size):
    return _kept(st, "workspace", lambda: torch.empty(max(size(), 256), dtype=torch.uint8, device="cuda"))


def _own_transition_backward(st):
    import paper_2607_05439_amd as dcp
    case, x = st["case"], st["x"]
    code, dt = (dcp.DCP_BF16 if case["dtype"] == "bf16" else dcp.DCP_F32), DTYPES[case["dtype"]]

    def plan():
        out = [torch.empty_like(x["dout"])]
        out += [torch.empty_like(x[k], dtype=dt) for k in ("w1", "w2", "w3", "gamma", "beta")]
        return out, dcp.make_transition_gradients(*out, dtype=code)

    out, grads = _kept(st, "plan", plan)
    ws = _workspace(st, lambda: dcp.dcp_pair_transition_backward_workspace_size(case["pairs"], case["c"], case["hidden"], code))
    dcp.dcp_pair_transition_backward(case["pairs"], case["c"], case["hidden"], code, EPS, x["w1"], x["w2"], x["w3"],
                                     x["gamma"], x["beta"], x["z"], x["exponents"], x["dout"], grads, ws, ws.numel())
    return out


def _own_checkpoint(st):
    import paper_2607_05439_amd as dcp
    case, x = st["case"], st["x"]["x"]
    rows, c, code = case["rows"], case["c"], dcp.DCP_BF16 if case["dtype"] == "bf16" else dcp.DCP_F32
    codes = _kept(st, "codes", lambda: torch.empty((rows, c), dtype=torch.int8, device="cuda"))
    exponents = _kept(st, "exponents", lambda: torch.empty((rows, -(-c // BLOCK)), dtype=torch.uint8, device="cuda"))
    y = _kept(st, "y", lambda: torch.empty_like(x))
    dcp.dcp_checkpoint_pack(rows, c, code, x, codes, exponents)
    dcp.dcp_checkpoint_unpack(rows, c, code, codes, exponents, y)
    return y


def _own_relative_position(st):
    import paper_2607_05439_amd as dcp
    case, x = st["case"], st["x"]
    code = dcp.DCP_BF16 if case["dtype"] == "bf16" else dcp.DCP_F32
    fields = _kept(st, "fields", lambda: dcp.make_relative_fields([(p, q, r) for (p, q), r in zip(x["fields"], _radii(case))]))
    if case["kind"] == "relpos":
        out = _kept(st, "out", lambda: torch.empty_like(x["z"]))
        dcp.dcp_relative_position(case["n"], case["row0"], case["rows"], case["c"], code, fields, x["table"], x["z"], out)
        return out
    out = _kept(st, "out", lambda: torch.empty((_buckets(case), case["c"]), device="cuda"))
    ws = _workspace(st, lambda: dcp.dcp_relative_position_backward_workspace_size(case["n"], case["rows"], case["c"], fields))
    dcp.dcp_relative_position_backward(case["n"], case["row0"], case["rows"], case["c"], code, fields, x["dz"], out, ws,
                                       ws.numel())
    return out


# ----------------------------------------------------------------------------- the plain forms
def _plain_transition_backward(st):
    x = st["x"]
    dt, gamma = x["dout"].dtype, x["gamma"]
    z = x["z"].float() if x["exponents"] is None else _values(x["z"], x["exponents"])
    z = z - z.mean(dim=1, keepdim=True)
    rstd = torch.rsqrt(z.square().mean(dim=1, keepdim=True) + EPS)
    zh = z * rstd
    nz = zh * gamma + x["beta"]
    a, b = nz @ x["w1"].T, nz @ x["w2"].T
    sig = 1.0 / (1.0 + torch.exp(-a))
    silu = a * sig
    dy = x["dout"].float()
    dw3 = dy.T @ (silu * b)
    dh = dy @ x["w3"]
    db = dh * silu
    da = dh * b * (sig + silu * (1.0 - sig))
    dn = da @ x["w1"] + db @ x["w2"]
    g = dn * gamma
    dz = dy + rstd * (g - g.mean(dim=1, keepdim=True) - zh * (g * zh).mean(dim=1, keepdim=True))
    # the affine weights' sums over the pairs in 64 bits: up to a million terms that mostly cancel
    out = [dz, da.T @ nz, db.T @ nz, dw3, (dn * zh).sum(dim=0, dtype=torch.float64), dn.sum(dim=0, dtype=torch.float64)]
    return [t.to(dt) for t in out]


def _plain_checkpoint(st):
    x = st["x"]["x"]
    return _values(*_checkpoint(x)).to(x.dtype)


def _bucket(st, f):
    """[rows, n] buckets of field f, counted from the table's first row: the clipped difference, or one
    more for tokens of different groups."""
    case = st["case"]
    radii = _radii(case)
    r, first = radii[f], sum(2 * k + 2 for k in radii[:f])
    position, group = (t.long() for t in st["x"]["fields"][f])
    rows = slice(case["row0"], case["row0"] + case["rows"])
    d = (position[rows, None] - position[None, :]).clamp(-r, r) + r
    return first + torch.where(group[rows, None] == group[None, :], d, torch.full_like(d, 2 * r + 1))


def _plain_relative_position(st):
    x = st["x"]
    table = x["table"]
    total = sum(table[_bucket(st, f)] for f in range(len(x["fields"])))
    return (x["z"].float() + total).to(x["z"].dtype)


def _plain_relative_position_backward(st):
    case, x = st["case"], st["x"]
    every = torch.arange(_buckets(case), device="cuda")[None, :, None]
    # a product per row of the stripe with the rows of zeros and ones, and the rows' sum in 64 bits
    hot = sum((_bucket(st, f)[:, None, :] == every).float() for f in range(len(x["fields"])))
    return torch.bmm(hot, x["dz"].float()).sum(dim=0, dtype=torch.float64).float()


def run(st):
    kind = st["case"]["kind"]
    if kind == "trans_back":
        return _own_transition_backward(st) if own else _plain_transition_backward(st)
    if kind == "ckpt":
        return _own_checkpoint(st) if own else _plain_checkpoint(st)
    if own:
        return _own_relative_position(st)
    return _plain_relative_position(st) if kind == "relpos" else _plain_relative_position_backward(st)


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    size, c = (2 if case["dtype"] == "bf16" else 4), case["c"]
    eight = c + -(-c // BLOCK)  # bytes of a row's checkpoint
    if case["kind"] == "trans_back":
        pairs, hidden = case["pairs"], case["hidden"]
        return {"bytes": pairs * ((eight if case["checkpoint"] else c * size) + 2 * c * size)
                + (3 * c * hidden + 2 * c) * (4 + size),
                # A, B, dH, two products each for dN and for the gradients of W1 and W2, one for that of W3;
                # about 20 operations per hidden unit and 25 per channel
                "flops": pairs * (16 * c * hidden + 20 * hidden + 25 * c)}
    if case["kind"] == "ckpt":
        return {"bytes": 2 * case["rows"] * (c * size + eight), "flops": 6 * case["rows"] * c}
    pairs, fields = case["rows"] * case["n"], len(_radii(case))
    passes = 2 if case["kind"] == "relpos" else 1  # z in and out, or dz
    return {"bytes": passes * pairs * c * size + 4 * _buckets(case) * c + 8 * fields * case["n"],
            "flops": pairs * c * (fields + 1 if case["kind"] == "relpos" else fields)}


# ----------------------------------------------------------------------------- the same in 64 bits
def _transition(z, w):
    """The transition from its definition (the oracle of its gradients)."""
    var, mu = torch.var_mean(z, dim=1, keepdim=True, correction=0)
    n = (z - mu) / (var + EPS).sqrt() * w["gamma"] + w["beta"]
    return z + (torch.nn.functional.silu(n @ w["w1"].T) * (n @ w["w2"].T)) @ w["w3"].T


def _exact_values(codes, exponents):
    powers = torch.pow(2.0, exponents.double() - 127.0).repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]
    return codes.double() * powers


def _exact_checkpoint(x):
    """Block by block of channels: the exponent from a logarithm, put right where it is one off."""
    y = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for k in range(0, x.shape[1], BLOCK):
        v = x[:, k:k + BLOCK].double()
        top = v.abs().max(dim=1, keepdim=True).values
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -300) / 128.0)) - 1
        for _ in range(4):
            e = torch.where(torch.round(top * torch.pow(2.0, -e)) > 127, e + 1, e)
        e = e.clamp(min=-126)
        y[:, k:k + BLOCK] = torch.round(v * torch.pow(2.0, -e)) * torch.pow(2.0, e)
    return y


def _exact_hot(case, x, i0, i1):
    """[i1 - i0, n, buckets] zeros and ones of the stripe's rows i0..i1."""
    n = case["n"]
    hot = torch.zeros((i1 - i0, n, _buckets(case)), dtype=torch.float64, device="cuda")
    first = 0
    for (position, group), r in zip(x["fields"], _radii(case)):
        i = slice(case["row0"] + i0, case["row0"] + i1)
        d = torch.minimum(torch.maximum(position[i].double()[:, None] - position.double()[None, :],
                                        torch.tensor(-float(r), device="cuda")), torch.tensor(float(r), device="cuda"))
        b = torch.where(group[i][:, None] != group[None, :], torch.tensor(r + 1.0, device="cuda"), d) + (r + first)
        hot.scatter_(2, b.long()[:, :, None], 1.0)
        first += 2 * r + 2
    return hot


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] == "ckpt":
        return _exact_checkpoint(x["x"])
    if case["kind"] == "trans_back":
        names = ("w1", "w2", "w3", "gamma", "beta")
        w = {k: x[k].double().requires_grad_() for k in names}
        total = [torch.zeros_like(w[k]) for k in names]
        dz = torch.empty(x["dout"].shape, dtype=torch.float64, device="cuda")
        step = 1 << 16
        for r in range(0, case["pairs"], step):
            part = slice(r, r + step)
            z = x["z"][part].double() if x["exponents"] is None else _exact_values(x["z"][part], x["exponents"][part])
            z.requires_grad_()
            grads = torch.autograd.grad(_transition(z, w), [z] + [w[k] for k in names], x["dout"][part].double())
            dz[part] = grads[0]
            total = [a + b for a, b in zip(total, grads[1:])]
        return [dz] + total
    n, c, rows = case["n"], case["c"], case["rows"]
    step = max(1, (1 << 27) // (n * _buckets(case)))
    if case["kind"] == "relpos":
        y = torch.empty(x["z"].shape, dtype=torch.float64, device="cuda")
        for i in range(0, rows, step):
            e = min(i + step, rows)
            hot = _exact_hot(case, x, i, e).view((e - i) * n, -1)
            y[i:e] = x["z"][i:e].double() + (hot @ x["table"].double()).view(e - i, n, c)
        return y
    total = torch.zeros((_buckets(case), c), dtype=torch.float64, device="cuda")
    for i in range(0, rows, step):
        e = min(i + step, rows)
        hot = _exact_hot(case, x, i, e).view((e - i) * n, -1)
        total += hot.T.contiguous() @ x["dz"][i:e].double().view((e - i) * n, c)
    return total
