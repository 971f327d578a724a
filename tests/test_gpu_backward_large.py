"""The attention's backward pass at sizes where the sums are split: keys over parts of a row tile, rows over
parts of a key tile, tokens over parts of the weights' gradients (GPU). The reference is the layer's
definition, differentiated in 64 bits over chunks of rows; the tolerances are those of
test_gpu_attention_backward.py, whose logits these have."""
import pytest

from test_gpu_attention_backward import BF16, F32, NAMES, Call, check, layer, make

pytestmark = pytest.mark.gpu


def reference_in_chunks(x):
    import torch
    n, row0, rows = x["dims"][:3]
    x = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in x.items()}
    w = {k: x[k].double().requires_grad_() for k in ("w_q", "w_k", "w_v", "w_g", "w_b", "gamma")}
    s = x["s"].double().requires_grad_()
    total, dz = None, []
    step = max(1, (1 << 18) // n)
    for r in range(0, rows, step):
        e = min(r + step, rows)
        z = x["z"][r:e].double().requires_grad_()
        part = {**x, "dims": (n, row0 + r, e - r) + x["dims"][3:]}
        got = torch.autograd.grad(layer(part, w, s, z), [z, s] + [w[k] for k in NAMES[2:]], x["dout"][r:e].double())
        dz.append(got[0].cpu())
        total = list(got[1:]) if total is None else [a + b for a, b in zip(total, got[1:])]
    return dict(zip(NAMES, [torch.cat(dz)] + [t.cpu() for t in total]))


@pytest.mark.parametrize("n,row0,rows,masked", [(257, 0, 257, 0), (333, 0, 333, 0), (600, 200, 300, 11), (1030, 0, 1030, 7),
                                                (2500, 1003, 130, 100), (3001, 3000, 1, 0)])
def test_fused_shape(n, row0, rows, masked):
    x = make(n, row0, rows, **BF16, masked=masked, seed=n)
    check(Call(x)(), reference_in_chunks(x), 1e-2)


@pytest.mark.parametrize("case,dtype", [
    (dict(n=601, row0=0, rows=601, c_s=128, c_z=128, h=4, d=32, masked=9), "f32"),
    (dict(n=601, row0=0, rows=601, c_s=128, c_z=128, h=4, d=32, masked=9), "bf16"),
    (dict(n=300, row0=40, rows=211, c_s=64, c_z=256, h=16, d=8, masked=3), "f32"),
    (dict(n=300, row0=40, rows=211, c_s=64, c_z=256, h=16, d=8, masked=3), "bf16"),
    (dict(n=1100, row0=1000, rows=100, c_s=128, c_z=32, h=4, d=32), "f32"),
    (dict(n=700, row0=0, rows=90, c_s=128, c_z=64, h=8, d=16, masked=50), "bf16"),
], ids=lambda v: v if isinstance(v, str) else "-".join(str(k) for k in v.values()))
def test_general_path(case, dtype):
    x = make(**case, dtype=dtype, seed=case["n"])
    check(Call(x, out_dtype=0)(), reference_in_chunks(x), 2e-5 + (2.0 ** -8 if dtype == "bf16" else 0))


@pytest.mark.parametrize("widths", [F32, BF16], ids=["f32", "bf16"])
def test_biases_that_add_a_constant_per_head(widths):
    """b_b and ln_beta in the forward and the backward: the bits of a call without them."""
    import torch
    import paper_2607_05439_amd as dcp
    x = make(90, 5, 60, **widths, masked=3, seed=70)
    call = Call(x)
    want = call()
    g = call.x
    b_b, beta = torch.randn(widths["h"], device="cuda") * 3, torch.randn(widths["c_z"], device="cuda") * 3
    call.weights = dcp.make_weights(g["w_q"], g["w_k"], g["w_v"], g["w_g"], g["w_b"], b_b, g["gamma"], beta)
    for t in (call.m, call.l, call.acc):
        t.fill_(7.0)
    ws = torch.empty(dcp.dcp_workspace_size(call.shape, 60, 1), dtype=torch.uint8, device="cuda")
    dcp.dcp_pair_bias_attention_partial(call.shape, call.weights, g["s"], g["z"], g["mask"], 5, 60, 0, 90, call.m, call.l,
                                        call.acc, None, ws, ws.numel())
    got = call()
    assert all(torch.equal(got[k], want[k]) for k in NAMES)
