"""LayerNorm and its backward pass through the C-ABI against the same in 64 bits (GPU).

Tolerances. Both kernels work in fp32 on the inputs as given, so an output is off by the
rounding to its type (half a step: 2^-24 fp32, 2^-8 bf16 relative) and by the fp32 arithmetic.
The sums over c channels run in at most c / 2 + 8 sequential additions, each off by 2^-24 of a
partial sum that a random walk keeps near sqrt(c) of a term: a few 2^-24 times sqrt(c), 4e-6 of
the result's scale at c = 4096, and 1e-5 is asserted. For the sums over rows the same holds with
at most n_rows / 1024 + 20 additions in a chain."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 1e-5
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def dtypes():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def code(t):
    import paper_2607_05439_amd as dcp
    return dcp.DCP_BF16 if t == "bf16" else dcp.DCP_F32


def make(rows, c, x_type, y_type, seed=0, offset=0.5):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((rows, c), generator=g) + offset * torch.randn((c,), generator=g)).to(dtypes()[x_type])
    dy = (torch.randn((rows, c), generator=g) / 64).to(dtypes()[y_type])
    return x, dy, 1 + torch.randn((c,), generator=g) / 4, torch.randn((c,), generator=g) / 4


def reference(x, dy, gamma, beta):
    """y, dx, dgamma, dbeta in 64 bits from the definition."""
    import torch
    x = x.double().requires_grad_()
    gamma = (torch.ones(x.shape[1]) if gamma is None else gamma).double().requires_grad_()
    beta = (torch.zeros(x.shape[1]) if beta is None else beta).double().requires_grad_()
    mu = x.mean(dim=1, keepdim=True)
    var = ((x - mu) ** 2).mean(dim=1, keepdim=True)
    y = gamma * (x - mu) / torch.sqrt(var + EPS) + beta
    return [y.detach()] + [t.detach() for t in torch.autograd.grad(y, [x, gamma, beta], dy.double())]


def off(got, want, t):
    """Largest error beyond half a step of the type, relative to the tensor's largest value."""
    got, want = got.cpu().double().numpy(), want.numpy()
    scale = np.abs(want).max() if want.size else 1.0
    return float((np.abs(got - want) - STEP[t] * np.abs(want)).max(initial=0.0) / max(scale, 1e-300))


def forward(x, gamma, beta, y_type, out=None):
    import torch
    import paper_2607_05439_amd as dcp
    y = torch.full(x.shape, 7.0, dtype=dtypes()[y_type], device="cuda") if out is None else out
    x_type = "bf16" if x.dtype == torch.bfloat16 else "f32"
    dcp.dcp_layer_norm(x.shape[0], x.shape[1], code(x_type), code(y_type), EPS, x, gamma, beta, y)
    return y


def backward(x, gamma, dy, want=(True, True, True), dx=None):
    import torch
    import paper_2607_05439_amd as dcp
    n, c = x.shape
    t = {torch.bfloat16: code("bf16"), torch.float32: code("f32")}
    dx = torch.full_like(x, 7.0) if dx is None else dx
    dg, db = torch.full((c,), 7.0, device="cuda"), torch.full((c,), 7.0, device="cuda")
    ws = torch.full((max(dcp.dcp_layer_norm_backward_workspace_size(n, c), 256),), 255, dtype=torch.uint8, device="cuda")
    dcp.dcp_layer_norm_backward(n, c, t[x.dtype], t[dy.dtype], EPS, x, gamma, dy, dx if want[0] else None,
                                dg if want[1] else None, db if want[2] else None, ws, ws.numel())
    return dx, dg, db


SHAPES = [(1, 1), (1, 8), (3, 3), (2, 4), (5, 7), (17, 24), (130, 32), (333, 384), (64, 130), (9, 1000), (70, 1544),
          (3, 2047), (5, 4096), (1, 4095), (4099, 64), (6000, 128)]


@pytest.mark.parametrize("rows,c", SHAPES)
@pytest.mark.parametrize("x_type,y_type", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_matches_the_definition(rows, c, x_type, y_type):
    x, dy, gamma, beta = make(rows, c, x_type, y_type, seed=rows + c)
    want = reference(x, dy, gamma, beta)
    xd, dyd, gd, bd = (t.cuda() for t in (x, dy, gamma, beta))
    y = forward(xd, gd, bd, y_type)
    got = backward(xd, gd, dyd)
    errs = [off(y, want[0], y_type), off(got[0], want[1], x_type), off(got[1], want[2], "f32"), off(got[2], want[3], "f32")]
    print(rows, c, x_type, y_type, ["%.2e" % e for e in errs], flush=True)
    if c == 1:  # xh is 0: y = beta, dx = dgamma = 0 exactly
        assert errs[0] == 0 and not got[0].any() and not got[1].any()
    assert max(errs[i] for i in ((0, 3) if c == 1 else (0, 1, 2, 3))) <= 1e-5


def test_without_affine_weights():
    x, dy, _, _ = make(65, 96, "bf16", "bf16", seed=3)
    want = reference(x, dy, None, None)
    xd, dyd = x.cuda(), dy.cuda()
    assert off(forward(xd, None, None, "bf16"), want[0], "bf16") <= 1e-5
    got = backward(xd, None, dyd)
    assert off(got[0], want[1], "bf16") <= 1e-5 and off(got[1], want[2], "f32") <= 1e-5


def test_each_gradient_alone_has_the_same_bits():
    import torch
    x, dy, gamma, _ = (None if t is None else t.cuda() for t in make(300, 384, "bf16", "bf16", seed=4))
    all_three = backward(x, gamma, dy)
    for k in range(3):
        got = backward(x, gamma, dy, want=tuple(i == k for i in range(3)))
        for i in range(3):
            assert torch.equal(got[i], all_three[i]) if i == k else (got[i] == 7.0).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("c", [33, 384, 2000])
def test_in_place(t, c):
    import torch
    x, dy, gamma, beta = (v.cuda() for v in make(101, c, t, t, seed=5))
    y, (dx, dg, db) = forward(x, gamma, beta, t), backward(x, gamma, dy)
    for onto in ("x", "dy"):
        xc, dyc = x.clone(), dy.clone()
        got = backward(xc, gamma, dyc, dx=xc if onto == "x" else dyc)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dg) and torch.equal(got[2], db)
    assert torch.equal(forward(x, gamma, beta, t, out=x), y)


def test_unaligned_tensors():
    """Tensors off 16-byte alignment take one element at a time: the definition again, and nothing
    written outside."""
    import torch
    for t in ("f32", "bf16"):
        x, dy, gamma, beta = make(50, 64, t, t, seed=6)
        want = reference(x, dy, gamma, beta)
        flat = torch.full((50 * 64 + 2,), 7.0, dtype=dtypes()[t], device="cuda")
        xs, ys, ds = flat.clone(), flat.clone(), flat.clone()
        view = lambda v: v[1:-1].view(50, 64)  # noqa: E731
        view(xs).copy_(x), view(ds).copy_(dy)
        forward(view(xs), gamma.cuda(), beta.cuda(), t, out=view(ys))
        assert off(view(ys), want[0], t) <= 1e-5 and ys[0] == 7 and ys[-1] == 7
        got = backward(view(xs), gamma.cuda(), view(ds), dx=view(ys))
        assert off(got[0], want[1], t) <= 1e-5 and ys[0] == 7 and ys[-1] == 7
        assert off(got[1], want[2], "f32") <= 1e-5


def test_large_mean_and_constant_rows():
    """A mean far above the spread keeps its precision (the row is centred before it is squared);
    constant rows give beta and finite gradients."""
    import torch
    x, dy, gamma, beta = make(40, 128, "f32", "f32", seed=7)
    x = x + 1000.0
    x[5] = 3.0
    want = reference(x, dy, gamma, beta)
    y = forward(x.cuda(), gamma.cuda(), beta.cuda(), "f32")
    assert torch.equal(y[5].cpu(), beta)
    # the mean is off by up to 2^-24 of 1000, and with it the centred values of size 1
    assert off(y, want[0], "f32") <= 8 * 1000 * 2.0 ** -24
    dx = backward(x.cuda(), gamma.cuda(), dy.cuda())[0]
    rest = [i for i in range(40) if i != 5]
    assert off(dx[rest], want[1][rest], "f32") <= 8 * 1000 * 2.0 ** -24 and torch.isfinite(dx[5]).all()


def test_nan_stays_in_its_row():
    import torch
    x, dy, gamma, beta = make(37, 48, "f32", "f32", seed=8)
    want = reference(x, dy, gamma, beta)
    x[9, 3], x[20, 47] = float("nan"), float("inf")
    y, dx = forward(x.cuda(), gamma.cuda(), beta.cuda(), "f32"), backward(x.cuda(), gamma.cuda(), dy.cuda())[0]
    rest = [i for i in range(37) if i not in (9, 20)]
    assert torch.isnan(y[[9, 20]]).all() and torch.isnan(dx[[9, 20]]).all()
    assert off(y[rest], want[0][rest], "f32") <= 1e-5 and off(dx[rest], want[1][rest], "f32") <= 1e-5


def test_no_rows():
    import torch
    import paper_2607_05439_amd as dcp
    dg, db = torch.full((24,), 7.0, device="cuda"), torch.full((24,), 7.0, device="cuda")
    dcp.dcp_layer_norm(0, 24, 0, 0, EPS, None, None, None, None)
    dcp.dcp_layer_norm_backward(0, 24, 0, 0, EPS, None, None, None, None, dg, db, None, 0)
    assert not dg.any() and not db.any()


def test_gradient_against_differences():
    """dx along a random direction against the change of the loss."""
    import torch
    x, dy, gamma, beta = make(20, 96, "f32", "f32", seed=9)
    g = torch.Generator().manual_seed(1)
    v = torch.randn(x.shape, generator=g).double()
    loss = lambda t: float((reference(t, dy, gamma, beta)[0] * dy.double()).sum())  # noqa: E731
    h = 1e-4
    slope = (loss(x.double() + h * v) - loss(x.double() - h * v)) / (2 * h)
    dx = backward(x.cuda(), gamma.cuda(), dy.cuda())[0].cpu().double()
    # third derivatives of size 1 times h^2, and the gradient's 1e-5
    assert abs(float((dx * v).sum()) - slope) <= 1e-4 * float((dx.abs() * v.abs()).sum())


def test_replayed_on_another_stream():
    """Captured on a side stream and replayed with new inputs, the program's own eager calls between
    the replays."""
    import torch
    x, dy, gamma, beta = (v.cuda() for v in make(700, 384, "bf16", "bf16", seed=10))
    import paper_2607_05439_amd as dcp
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dg, db = torch.empty(384, device="cuda"), torch.empty(384, device="cuda")
    ws = torch.empty(dcp.dcp_layer_norm_backward_workspace_size(700, 384), dtype=torch.uint8, device="cuda")

    def call():
        dcp.dcp_layer_norm(700, 384, 1, 1, EPS, x, gamma, beta, y)
        dcp.dcp_layer_norm_backward(700, 384, 1, 1, EPS, x, gamma, dy, dx, dg, db, ws, ws.numel())

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        x.copy_(torch.randn(x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(k)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, forward(x, gamma, beta, "bf16"))
        assert all(torch.equal(a, b) for a, b in zip((dx, dg, db), backward(x, gamma, dy)))


def test_more_than_2_32_elements():
    """2^25 + 3 rows of 128: the last rows have the bits of a call on them alone, in place as well, and the
    sums over the rows are those in 64 bits: a chain of 2^25 / 2^14 additions leaves at most 2^-24 sqrt(2^11)
    of a partial sum, 3e-6, and 1e-5 is asserted of the norm."""
    import torch
    rows, c = 2 ** 25 + 3, 128
    gen = torch.Generator("cuda").manual_seed(5)
    x, dy = (torch.empty((rows, c), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for r in range(0, rows, 2 ** 22):
        for t in (x, dy):
            t[r:r + 2 ** 22] = torch.randn(t[r:r + 2 ** 22].shape, generator=gen, device="cuda")
    gamma, beta = (torch.rand(c, generator=gen, device="cuda") + 0.5 for _ in range(2))
    want = [torch.zeros(c, dtype=torch.float64, device="cuda") for _ in range(2)]
    for r in range(0, rows, 2 ** 20):
        a, b = x[r:r + 2 ** 20].double(), dy[r:r + 2 ** 20].double()
        a -= a.mean(dim=1, keepdim=True)
        a /= torch.sqrt((a ** 2).mean(dim=1, keepdim=True) + EPS)
        want[0] += (a * b).sum(dim=0)
        want[1] += b.sum(dim=0)
    tail = slice(rows - 1000, rows)
    y_tail = forward(x[tail].clone(), gamma, beta, "bf16")
    dx_tail = backward(x[tail].clone(), gamma, dy[tail].clone())[0]
    dx, dgamma, dbeta = backward(x, gamma, dy)
    assert torch.equal(dx[tail], dx_tail)
    for got, sum64 in zip((dgamma, dbeta), want):
        assert float((got.double() - sum64).norm()) <= 1e-5 * float(sum64.norm())
    del dx, dy
    assert torch.equal(forward(x, gamma, beta, "bf16", out=x)[tail], y_tail)
