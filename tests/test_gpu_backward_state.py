"""The fused backward pass and the softmax state that it is given: the library's own, whose forward
multiplies bf16 q, k and v, and the exact one. The weights that the backward forms have rows that sum to 1,
and their gradients rows that sum to 0, whichever state it was and however large the logits (GPU).

Tolerances. u = 2^-11 is half a step of fp16, in which the backward multiplies. A logit of size L is a
sum of 24 products, each off by at most 2 u of itself, independently: 2 u L / sqrt(24) in the norm if every
rounding were at its worst. A weight is off by as much, relatively, and dS = P (dP - D) by that twice, for P and
for D: 4 u L / sqrt(24). The result's own rounding to bf16 adds at most 2^-8. The gate's gradient
dout o g (1 - g), which is dw_g and a part of ds, takes o = acc / l from the state, and is as exact as that is:
for a state of bf16 logits the same with u = 2^-8, half a step of bf16.
"""
import math

import pytest

from test_gpu_attention_backward import BF16, EPS, NAMES, Call, check, make, reference

pytestmark = pytest.mark.gpu


def forward_64(x):
    """Per head and row of the stripe, in 64 bits: the logits, the weights, o and the gate."""
    import torch
    n, row0, rows, _, _, _, h, d = x["dims"]
    w = {k: x[k].double() for k in ("w_q", "w_k", "w_v", "w_g", "w_b")}
    s, z = x["s"].double(), x["z"].double()
    z = z - z.mean(dim=2, keepdim=True)
    z = z / torch.sqrt((z ** 2).mean(dim=2, keepdim=True) + EPS)
    if x["gamma"] is not None:
        z = z * x["gamma"].double()
    sq = s[row0:row0 + rows]
    heads = lambda t: t.reshape(-1, h, d).transpose(0, 1).contiguous()  # noqa: E731
    q, k, v = heads(sq @ w["w_q"].T), heads(s @ w["w_k"].T), heads(s @ w["w_v"].T)
    logits = q @ k.transpose(1, 2) / math.sqrt(d) + (z @ w["w_b"].T).permute(2, 0, 1)
    if x["mask"] is not None:
        logits = logits.masked_fill(x["mask"] == 0, -math.inf)
    p = torch.softmax(logits, dim=2)
    return {"logits": logits, "p": p, "q": q, "v": v, "o": p @ v, "g": torch.sigmoid(sq @ w["w_g"].T)}


def exact_state(call, x):
    """In the place of what the library's forward saved: m, l and acc from the definition."""
    f = forward_64(x)
    m = f["logits"].max(dim=2).values
    l = (f["logits"] - m[:, :, None]).exp().sum(dim=2)
    call.m.copy_(m), call.l.copy_(l), call.acc.copy_((f["o"] * l[:, :, None]).transpose(0, 1))


def largest_logit(f):
    return float(f["logits"][f["logits"] > -math.inf].abs().max())


@pytest.mark.parametrize("state", ["own", "exact"])
@pytest.mark.parametrize("factor", [1.0, 2.0, 4.0, 8.0, 16.0])
def test_logits_of_any_size(factor, state):
    x = make(200, 30, 120, **BF16, masked=5, seed=50)
    x["w_q"] = x["w_q"] * factor
    call, want, top = Call(x), reference(x), largest_logit(forward_64(x))
    if state == "exact":
        exact_state(call, x)
    got = call()
    through_o = ("ds", "w_g") if state == "own" else ()
    for names, u in ((tuple(k for k in NAMES if k not in through_o), 2.0 ** -11), (through_o, 2.0 ** -8)):
        if names:
            check(got, {k: want[k] for k in names}, 2.0 ** -8 + 4 * u * top / math.sqrt(24), "largest logit %.0f" % top)


@pytest.mark.parametrize("state", ["own", "exact"])
@pytest.mark.parametrize("factor", [1.0, 8.0, 32.0])
@pytest.mark.parametrize("row", [0, 61, 96])
def test_rows_sum_to_one_and_their_gradients_to_zero(row, factor, state):
    """A stripe of one row, and single-track channel 0 the constant 1 of every token: that channel's
    column of dW_v is sum_j dv_j = do sum_j P_j, and of dW_k sum_j dk_j = q sum_j dS_j / sqrt(d). P is off by 2^-11
    of itself, do and dS by as much once more, the pairs of bf16 and the sums behind them by under 2^-13."""
    import torch
    x = make(97, row, 1, **BF16, masked=4, seed=51)
    x["w_q"] = x["w_q"] * factor
    x["s"][:, 0] = 1.0
    call, f = Call(x, grad_dtype=0), forward_64(x)
    if state == "exact":
        exact_state(call, x)
    got = call()
    do = f["g"] * x["dout"].double()  # [1, 384]
    u = 2 * 2.0 ** -11 + 2.0 ** -13
    err = (got["w_v"][:, 0].cpu().double() - do[0]).abs()
    print("row sums off by", float((err / do[0].abs()).max()), flush=True)
    assert (err <= u * do[0].abs()).all(), float((err / do[0].abs()).max())
    dp = (do.view(16, 1, 24) * f["v"]).sum(dim=2)  # [16, 97]
    ds = (f["p"][:, 0] * (dp - (f["p"][:, 0] * dp).sum(dim=1, keepdim=True))).abs().sum(dim=1)
    bound = u * ds[:, None] * f["q"][:, 0].abs() / math.sqrt(24)
    if factor == 1.0:  # a one-sided softmax has nearly no dS: its sum is then that of P's roundings alone
        assert (got["w_k"][:, 0].cpu().double().abs() <= bound.flatten()).all()
    # P's own rounding leaves 2^-11 of D there
    bound = bound + u * (f["p"][:, 0] * dp.abs()).sum(dim=1)[:, None] * f["q"][:, 0].abs() / math.sqrt(24)
    assert (got["w_k"][:, 0].cpu().double().abs() <= bound.flatten()).all()


def test_a_ring_s_merged_state():
    """The state of three key ranges, the last of them merged on: the gradients of the whole one's."""
    import torch
    import paper_2607_05439_amd as dcp
    x = make(130, 17, 70, **BF16, masked=6, seed=52)
    call = Call(x)
    g, f = call.x, dict(dtype=torch.float32, device="cuda")
    m, l, acc = torch.empty((3, 16, 70), **f), torch.empty((3, 16, 70), **f), torch.empty((3, 70, 16, 24), **f)
    ws = torch.empty(dcp.dcp_workspace_size(call.shape, 70, 1), dtype=torch.uint8, device="cuda")
    for i, (k0, k1) in enumerate(((0, 40), (40, 55), (55, 130))):
        dcp.dcp_pair_bias_attention_partial(call.shape, call.weights, g["s"], g["z"], g["mask"], 17, 70, k0, k1, m[i], l[i],
                                            acc[i], None, ws, ws.numel())
    dcp.dcp_block_merge(3, 70, 16, 24, m, l, acc, call.m, call.l, call.acc, None, None, 0)
    check(call(), reference(x), 1e-2)
