"""A training step of the pair track as a program makes it: the relative position encoding gives z, the attention reads
it, an 8-bit checkpoint keeps it, the transition overwrites it in place; then the transition's backward pass from the
checkpoint, in place in the gradient's buffer, the attention's from z, and the gradients of the encoding's table,
the transition's weights and the attention's bias. Against 64 bits (GPU).

Tolerances, of the 2-norm of the error relative to that of the result. The reference takes z as the encoding rounds it, and
what the checkpoint reads back as the transition's input, so neither counts. fp32: 2e-5, twice that of one backward pass
alone. bf16: the table's gradient is a sum of two gradients, each rounded to bf16 with what its pass is off by (3.6e-3 the
transition's, 1e-2 the attention's), of independent errors: 1.1e-2; the others as in their own tests."""
import math

import pytest

pytestmark = pytest.mark.gpu

EPS = 1e-5
CASES = {"f32": dict(n=40, c_s=64, c_z=32, heads=4, d=16, hidden=80), "bf16": dict(n=90, c_s=384, c_z=128, heads=16, d=24, hidden=512)}
RADII = (32, 32, 2, 0)


def fields(n):
    import torch
    token = torch.arange(n)
    chain, within = token // 25, token % 25
    residue = (within * 7) // 10  # some residues of two tokens
    pos, grp = [residue, token, chain // 2, torch.zeros(n, dtype=torch.long)], [chain, 100 * chain + residue, chain % 2, chain % 2]
    return [(p.int().cuda(), g.int().cuda(), r) for p, g, r in zip(pos, grp, RADII)]


def attention(z, s, w, heads, d):
    """The gated attention of all rows from its definition."""
    import torch
    n = s.shape[0]
    mu = z.mean(dim=2, keepdim=True)
    zh = (z - mu) / torch.sqrt(((z - mu) ** 2).mean(dim=2, keepdim=True) + EPS)
    q, k, v = ((s @ w[x].T).view(n, heads, d).transpose(0, 1) for x in ("w_q", "w_k", "w_v"))
    logits = q @ k.transpose(1, 2).contiguous() / math.sqrt(d) + (zh @ w["w_b"].T).permute(2, 0, 1)
    o = torch.softmax(logits, dim=2) @ v
    return torch.sigmoid(s @ w["w_g"].T) * o.transpose(0, 1).reshape(n, heads * d)


def transition(z, w):
    import torch
    mu = z.mean(dim=-1, keepdim=True)
    n = (z - mu) / torch.sqrt(((z - mu) ** 2).mean(dim=-1, keepdim=True) + EPS) * w["gamma"] + w["beta"]
    a = n @ w["w1"].T
    return z + (a / (1 + torch.exp(-a)) * (n @ w["w2"].T)) @ w["w3"].T


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_a_step(t):
    import torch
    import paper_2607_05439_amd as dcp
    c = CASES[t]
    n, c_s, c_z, heads, d, hidden = (c[k] for k in ("n", "c_s", "c_z", "heads", "d", "hidden"))
    dt, code, pairs = (torch.float32, 0, n * n) if t == "f32" else (torch.bfloat16, 1, n * n)
    g = torch.Generator().manual_seed(21)
    r = lambda *s: torch.randn(s, generator=g).cuda()  # noqa: E731
    w = {k: r(heads * d, c_s) / c_s ** 0.5 for k in ("w_q", "w_k", "w_v", "w_g")}
    w["w_b"] = r(heads, c_z) / c_z ** 0.5
    tw = {"w1": r(hidden, c_z) / c_z ** 0.5, "w2": r(hidden, c_z) / c_z ** 0.5, "w3": r(c_z, hidden) / hidden ** 0.5,
          "gamma": 1 + r(c_z) / 4, "beta": r(c_z) / 4}
    fs = fields(n)
    table, s = r(sum(2 * q + 2 for q in RADII), c_z), r(n, c_s).to(dt)
    r_out, r_z = (r(n, heads * d) / 64).to(dt), (r(pairs, c_z) / 64).to(dt)
    f32 = dict(dtype=torch.float32, device="cuda")
    byte = lambda size: torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")  # noqa: E731

    # forward
    rel = dcp.make_relative_fields(fs)
    z = torch.empty((n, n, c_z), dtype=dt, device="cuda")
    dcp.dcp_relative_position(n, 0, n, c_z, code, rel, table, None, z)
    shape = dcp.make_shape(n, c_s, c_z, heads, d, code, code, EPS)
    weights = dcp.make_weights(w["w_q"], w["w_k"], w["w_v"], w["w_g"], w["w_b"])
    m, l, acc, gate = torch.empty((heads, n), **f32), torch.empty((heads, n), **f32), torch.empty((n, heads, d), **f32), torch.empty((n, heads * d), **f32)
    ws = byte(dcp.dcp_workspace_size(shape, n, 1))
    dcp.dcp_pair_bias_attention_partial(shape, weights, s, z, None, 0, n, 0, n, m, l, acc, gate, ws, ws.numel())
    codes, exps = torch.empty((pairs, c_z), dtype=torch.int8, device="cuda"), torch.empty((pairs, -(-c_z // 32)), dtype=torch.uint8, device="cuda")
    dcp.dcp_checkpoint_pack(pairs, c_z, code, z, codes, exps)
    z0 = z.clone()
    tws = byte(dcp.dcp_transition_workspace_size(c_z, hidden, code))
    dcp.dcp_pair_transition(pairs, c_z, hidden, code, EPS, tw["w1"], tw["w2"], tw["w3"], tw["gamma"], tw["beta"], z, z, tws, tws.numel())

    # backward
    grad = r_z.clone()
    dw = [torch.empty_like(tw[k]) for k in ("w1", "w2", "w3", "gamma", "beta")]
    bws = byte(dcp.dcp_pair_transition_backward_workspace_size(pairs, c_z, hidden, code))
    dcp.dcp_pair_transition_backward(pairs, c_z, hidden, code, EPS, tw["w1"], tw["w2"], tw["w3"], tw["gamma"], tw["beta"], codes, exps, grad,
                                     dcp.make_transition_gradients(grad, *dw), bws, bws.numel())
    read = torch.empty_like(z0)
    dcp.dcp_checkpoint_unpack(pairs, c_z, code, codes, exps, read)
    dz, dw_b = torch.empty_like(z0), torch.empty_like(w["w_b"])
    aws = byte(dcp.dcp_pair_bias_attention_backward_workspace_size(shape, n))
    dcp.dcp_pair_bias_attention_backward(shape, weights, s, z0, None, 0, n, m, l, acc, r_out, dcp.make_gradients(dz_rows=dz, dw_b=dw_b), aws, aws.numel())
    dz += grad.view(n, n, c_z)
    dtable = torch.empty_like(table)
    rws = byte(dcp.dcp_relative_position_backward_workspace_size(n, n, c_z, rel))
    dcp.dcp_relative_position_backward(n, 0, n, c_z, code, rel, dz, dtable, rws, rws.numel())

    # the same in 64 bits
    zd = z0.double().requires_grad_()
    w64, tw64 = ({k: v.double().requires_grad_() for k, v in x.items()} for x in (w, tw))
    want_z, want_b = torch.autograd.grad(attention(zd, s.double(), w64, heads, d), [zd, w64["w_b"]], r_out.double())
    kept = read.double().view(pairs, c_z).requires_grad_()
    back = torch.autograd.grad(transition(kept, tw64), [kept] + [tw64[k] for k in ("w1", "w2", "w3", "gamma", "beta")], r_z.double())
    total = (want_z + back[0].view(n, n, c_z)).view(pairs, c_z)
    want_table, hot = torch.zeros_like(table, dtype=torch.float64), torch.zeros((pairs, table.shape[0]), dtype=torch.float64, device="cuda")
    first = 0
    for pos, grp, q in fs:
        b = torch.clamp(pos[:, None].long() - pos[None, :].long(), -q, q) + q
        b[grp[:, None] != grp[None, :]] = 2 * q + 1
        hot.scatter_(1, (b + first).view(pairs, 1), 1.0)
        first += 2 * q + 2
    want_table = hot.T.contiguous() @ total
    z_want = hot @ table.double()
    assert ((z0.double().view(pairs, c_z) - z_want).abs() <= (2.0 ** -8 if t == "bf16" else 2.0 ** -20) * z_want.abs() + 1e-5).all()
    err = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    e = {"table": err(dtable, want_table), "w_b": err(dw_b, want_b), "grad": err(grad, back[0])}
    e.update({k: err(a, b) for k, a, b in zip(("w1", "w2", "w3", "gamma", "beta"), dw, back[1:])})
    print(t, {k: "%.2e" % v for k, v in e.items()}, flush=True)
    assert all(v <= (2e-5 if t == "f32" else 1.1e-2 if k == "table" else 1e-2 if k == "w_b" else 3.6e-3) for k, v in e.items()), e
