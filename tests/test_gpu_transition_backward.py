"""The pair transition's backward pass through the C-ABI against the same in 64 bits, against
differences, and in the calls that a program makes of it (GPU).

Tolerances, of the 2-norm of the error relative to that of the result. fp32: every product and sum is
fp32; the longest chain of additions is the pairs of one share, n / (16 splits) steps of matrix-core
products and 512 shares at most, whose rounding errors (2^-24 each, of partial sums that grow like the
result) add up like a random walk: under 100 of them, 6e-6; 1e-5 is asserted. bf16: a result passes at
most a dozen roundings to 11 bits one after another (the weights twice, zh, dout, the sigmoid, A, B and dH, up to four in
the gate), and one to its own 8 bits. Each is off by at most half a step of its value, by 0.42 of that in the root mean
square over values spread evenly in their binade, and they are independent: sqrt(1 + 12 / 64) 0.42 2^-8 = 1.8e-3;
twice that, 3.6e-3, is asserted."""
import pytest

pytestmark = pytest.mark.gpu

EPS = 1e-5
TOL = {"f32": 1e-5, "bf16": 3.6e-3}
NAMES = ("dz", "dw1", "dw2", "dw3", "dgamma", "dbeta")


def dtypes():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def code(t):
    import paper_2607_05439_amd as dcp
    return dcp.DCP_BF16 if t == "bf16" else dcp.DCP_F32


def make(pairs, c, hidden, t, seed=0, affine=True, offset=0.5):
    import torch
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x = {"w1": r(hidden, c) / c ** 0.5, "w2": r(hidden, c) / c ** 0.5, "w3": r(c, hidden) / hidden ** 0.5,
         "gamma": 1 + r(c) / 4 if affine else None, "beta": r(c) / 4 if affine else None,
         "z": (r(pairs, c) + offset * r(c)).to(dtypes()[t]), "dout": (r(pairs, c) / 1024).to(dtypes()[t]), "exp": None}
    return {k: None if v is None else v.cuda() for k, v in x.items()}


def checkpointed(x):
    """The same with z as a checkpoint, written by the library."""
    import torch
    import paper_2607_05439_amd as dcp
    n, c = x["z"].shape
    codes = torch.empty((n, c), dtype=torch.int8, device="cuda")
    exp = torch.empty((n, -(-c // 32)), dtype=torch.uint8, device="cuda")
    dcp.dcp_checkpoint_pack(n, c, code("bf16" if x["z"].dtype == torch.bfloat16 else "f32"), x["z"], codes, exp)
    return {**x, "z": codes, "exp": exp}


def values(x):
    """z in 64 bits."""
    import torch
    if x["exp"] is None:
        return x["z"].double()
    p = torch.pow(2.0, x["exp"].double() - 127).repeat_interleave(32, dim=1)[:, :x["z"].shape[1]]
    return x["z"].double() * p


def layer(z, w):
    import torch
    mu = z.mean(dim=1, keepdim=True)
    n = (z - mu) / torch.sqrt(((z - mu) ** 2).mean(dim=1, keepdim=True) + EPS)
    if w["gamma"] is not None:
        n = n * w["gamma"]
    if w["beta"] is not None:
        n = n + w["beta"]
    a, b = n @ w["w1"].T, n @ w["w2"].T
    return z + (a / (1 + torch.exp(-a)) * b) @ w["w3"].T


def reference(x):
    """The six gradients in 64 bits from the definition."""
    import torch
    z = values(x).requires_grad_()
    c = z.shape[1]
    w = {k: x[k].double().requires_grad_() for k in ("w1", "w2", "w3")}
    w["gamma"] = (torch.ones(c, device="cuda") if x["gamma"] is None else x["gamma"]).double().requires_grad_()
    w["beta"] = (torch.zeros(c, device="cuda") if x["beta"] is None else x["beta"]).double().requires_grad_()
    names = ("w1", "w2", "w3", "gamma", "beta")
    return dict(zip(NAMES, torch.autograd.grad(layer(z, w), [z] + [w[k] for k in names], x["dout"].double())))


class Call:
    """The library's call with outputs and workspace of its own; `want`: the gradients asked for."""

    def __init__(self, x, grad_type=None, want=NAMES, in_place=False):
        import torch
        import paper_2607_05439_amd as dcp
        self.x, (n, c), hidden = x, x["dout"].shape, x["w1"].shape[0]
        self.t = "bf16" if x["dout"].dtype == torch.bfloat16 else "f32"
        gt = grad_type or self.t
        full = lambda *s: torch.full(s, 7.0, dtype=dtypes()[gt], device="cuda")  # noqa: E731
        self.out = {"dz": x["dout"] if in_place else torch.full_like(x["dout"], 7.0), "dw1": full(hidden, c),
                    "dw2": full(hidden, c), "dw3": full(c, hidden), "dgamma": full(c), "dbeta": full(c)}
        self.grads = dcp.make_transition_gradients(*[self.out[k] if k in want else None for k in NAMES], dtype=code(gt))
        size = dcp.dcp_pair_transition_backward_workspace_size(n, c, hidden, code(self.t))
        self.ws = torch.full((max(size, 256),), 255, dtype=torch.uint8, device="cuda")
        self.dims = (n, c, hidden)

    def __call__(self, stream=None, ws=None):
        import paper_2607_05439_amd as dcp
        x, ws = self.x, self.ws if ws is None else ws
        dcp.dcp_pair_transition_backward(*self.dims, code(self.t), EPS, x["w1"], x["w2"], x["w3"], x["gamma"], x["beta"],
                                         x["z"], x["exp"], x["dout"], self.grads, ws, ws.numel(), stream)
        return self.out


def errors(got, want):
    return {k: float((got[k].double() - want[k]).norm() / max(float(want[k].norm()), 1e-300)) for k in want}


def check(got, want, t, what):
    e = errors(got, want)
    print(what, {k: "%.2e" % v for k, v in e.items()}, flush=True)
    assert all(v <= TOL[t] for v in e.values()), (what, e)


F32_SHAPES = [(1, 2, 1), (1, 4, 16), (5, 3, 7), (16, 32, 128), (17, 32, 128), (33, 20, 50), (100, 64, 256), (70, 100, 400),
              (130, 128, 512), (40, 129, 260), (50, 256, 1024), (37, 255, 33), (4097, 32, 128), (9000, 64, 100)]


@pytest.mark.parametrize("saved", ["whole", "checkpoint"])
@pytest.mark.parametrize("pairs,c,hidden", F32_SHAPES)
def test_f32_matches_the_definition(pairs, c, hidden, saved):
    x = make(pairs, c, hidden, "f32", seed=pairs + c)
    x = checkpointed(x) if saved == "checkpoint" else x
    check(Call(x)(), reference(x), "f32", (pairs, c, hidden, saved))


@pytest.mark.parametrize("grad_type", ["f32", "bf16"])
@pytest.mark.parametrize("saved", ["whole", "checkpoint"])
@pytest.mark.parametrize("pairs", [1, 2, 15, 31, 32, 33, 255, 257, 1000, 2025, 16385, 70001])
def test_bf16_matches_the_definition(pairs, saved, grad_type):
    x = make(pairs, 128, 512, "bf16", seed=pairs)
    x = checkpointed(x) if saved == "checkpoint" else x
    check(Call(x, grad_type)(), reference(x), "bf16", (pairs, saved, grad_type))


def test_one_channel():
    """LayerNorm of one channel is beta: dz is dout, and dgamma 0."""
    import torch
    x = make(20, 1, 8, "f32", seed=1)
    got, want = Call(x)(), reference(x)
    assert torch.equal(got["dz"], x["dout"]) and not got["dgamma"].any()
    for k in ("dw1", "dw2", "dw3", "dbeta"):
        assert float((got[k].double() - want[k]).norm()) <= 1e-5 * float(want[k].norm())


@pytest.mark.parametrize("t,c,hidden", [("f32", 24, 40), ("bf16", 128, 512)])
def test_without_affine_weights(t, c, hidden):
    x = make(300, c, hidden, t, seed=3, affine=False)
    check(Call(x)(), reference(x), t, "no affine")


@pytest.mark.parametrize("pairs", [300, 9000, 40000])
@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("f32", 33, 70), ("bf16", 128, 512)])
def test_each_gradient_alone_and_in_place_have_the_same_bits(t, c, hidden, pairs):
    import torch
    x = make(pairs, c, hidden, t, seed=4)
    whole = {k: v.clone() for k, v in Call(x)().items()}
    for k in NAMES:
        got = Call(x, want=(k,))()
        for j in NAMES:
            assert torch.equal(got[j], whole[j]) if j == k else (got[j] == 7.0).all(), (k, j)
    got = Call({**x, "dout": x["dout"].clone()}, in_place=True)()
    assert all(torch.equal(got[k], whole[k]) for k in NAMES)


@pytest.mark.parametrize("t,c,hidden", [("f32", 20, 36), ("bf16", 128, 512)])
def test_against_differences(t, c, hidden):
    """The gradients' products with random directions against central differences of the definition
    in 64 bits: off by h^2 of the third derivative (1e-10 here) and by the gradients' tolerance, of a sum
    whose terms are those of the product: |gradient| |direction|."""
    import torch
    x = make(60, c, hidden, t, seed=5)
    got = Call(x)()
    w = {k: x[k].double() for k in ("w1", "w2", "w3", "gamma", "beta")}
    w["z"], dout, g = values(x), x["dout"].double(), torch.Generator(device="cuda").manual_seed(6)
    for k, name in zip(NAMES, ("z", "w1", "w2", "w3", "gamma", "beta")):
        v = torch.randn(w[name].shape, generator=g, device="cuda", dtype=torch.float64)
        f = lambda h: (layer(*((lambda q: (q["z"], q))({**w, name: w[name] + h * v}))) * dout).sum()  # noqa: B023, E731
        want, have = float((f(1e-5) - f(-1e-5)) / 2e-5), float((got[k].double() * v).sum())
        scale = float(got[k].double().norm() * v.norm())
        print(t, k, want, have, scale, flush=True)
        assert abs(want - have) <= (TOL[t] + 1e-8) * scale


@pytest.mark.parametrize("saved", ["whole", "checkpoint"])
@pytest.mark.parametrize("c", [32, 37])
def test_f32_tensors_off_16_byte_alignment(c, saved):
    """The definition, and nothing written outside."""
    import torch
    x = make(50, c, 48, "f32", seed=7)
    x = checkpointed(x) if saved == "checkpoint" else x
    want = reference(x)

    def off_by_one(t):
        flat = torch.full((t.numel() + 2,), 7, dtype=t.dtype, device="cuda")
        flat[1:-1] = t.flatten()
        return flat[1:-1].view(t.shape), flat

    y = {k: None if v is None else off_by_one(v)[0] for k, v in x.items()}
    call = Call(y)
    import paper_2607_05439_amd as dcp
    outs = {k: off_by_one(v) for k, v in call.out.items()}
    call.out = {k: v[0] for k, v in outs.items()}
    call.grads = dcp.make_transition_gradients(*[call.out[k] for k in NAMES], dtype=0)
    check(call(), want, "f32", "off by one")
    assert all(flat[0] == 7 and flat[-1] == 7 for _, flat in outs.values())


@pytest.mark.parametrize("pairs", [1, 33, 1000, 20011])
@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_nothing_is_written_behind_the_last_pair_or_the_workspace(t, c, hidden, pairs):
    import torch
    import paper_2607_05439_amd as dcp
    x = make(pairs, c, hidden, t, seed=8)
    call = Call(x)
    dz = torch.full((pairs + 300, c), 7.0, dtype=x["dout"].dtype, device="cuda")
    ws = torch.full((call.ws.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
    call.out["dz"] = dz[:pairs]
    call.grads = dcp.make_transition_gradients(*[call.out[k] for k in NAMES], dtype=code(t))
    size = call.ws.numel()
    dcp.dcp_pair_transition_backward(*call.dims, code(t), EPS, x["w1"], x["w2"], x["w3"], x["gamma"], x["beta"], x["z"], None,
                                     x["dout"], call.grads, ws, size, None)
    assert (dz[pairs:] == 7.0).all() and (ws[size:] == 255).all()
    check(call.out, reference(x), t, pairs)


@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_without_pairs_the_weights_gradients_are_zero(t, c, hidden):
    x = make(1, c, hidden, t)
    x = {**x, "z": x["z"][:0], "dout": x["dout"][:0]}
    got = Call(x)()
    assert all(not got[k].any() for k in NAMES[1:])


@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_zero_gradients_and_pairs_that_are_not_finite(t, c, hidden):
    """dout = 0 gives exact zeros. A NaN in one pair reaches its own dz and the weights' gradients, and
    no other pair."""
    import torch
    x = make(1000, c, hidden, t, seed=9)
    zero = Call({**x, "dout": torch.zeros_like(x["dout"])})()
    assert all(not v.any() for v in zero.values())
    want = Call(x)()["dz"].clone()
    for name in ("z", "dout"):
        y = {**x, name: x[name].clone()}
        y[name][517, 3] = float("nan")
        got = Call(y)()
        keep = torch.arange(1000, device="cuda") != 517
        assert torch.equal(got["dz"][keep], want[keep]) and got["dz"][517].isnan().any()
        assert got["dw1"].isnan().any() and got["dgamma"].isnan().any()


@pytest.mark.parametrize("what,factor", [("dout", 2.0 ** 80), ("dout", 2.0 ** -90), ("w3", 2.0 ** -24), ("w3", 2.0 ** 40),
                                         ("w1", 2.0 ** -30), ("w2", 2.0 ** -30), ("w2", 2.0 ** 30), ("gamma", 2.0 ** -20),
                                         ("gamma", 2.0 ** 6), ("w1", 16.0)])
@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_magnitudes(t, c, hidden, what, factor):
    """Every gradient that is not small against its parts keeps its relative precision at any size of the
    inputs. W1 or gamma many times as large make A so: sigmoid(A) and its slope are then off by |A| times
    A's relative error. A is a sum of c products whose operands are off by 2^-11 (bf16) or 2^-24: by
    2^-11 |A| at most in the norm, and largest |A| is taken times that on top of the tolerance."""
    x = make(500, c, hidden, t, seed=10)
    x[what] = x[what] * factor
    if what == "gamma":
        x["beta"] = x["beta"] * factor
    got, want = Call(x, "f32")(), reference(x)
    e = errors(got, want)
    n = values(x)
    n = n - n.mean(dim=1, keepdim=True)
    n = n / (n ** 2).mean(dim=1, keepdim=True).add(EPS).sqrt() * x["gamma"].double() + x["beta"].double()
    top = max(float((n @ x["w1"].double().T).abs().max()) - 4, 0.0)
    tol = TOL[t] + top * (2.0 ** -11 if t == "bf16" else 2.0 ** -22)
    print(t, what, factor, {k: "%.2e" % v for k, v in e.items()}, "largest A %.1f" % top, flush=True)
    assert all(v <= tol for v in e.values()), (e, tol)


def test_pairs_of_any_size_beside_each_other():
    """A pair whose gradient is 2^-40 of another's keeps its own precision in dz."""
    import torch
    x = make(640, 128, 512, "bf16", seed=11)
    x["dout"][::2] *= 2.0 ** -40
    got, want = Call(x)(), reference(x)
    for part in (slice(0, None, 2), slice(1, None, 2)):
        assert float((got["dz"][part].double() - want["dz"][part]).norm() / want["dz"][part].norm()) <= TOL["bf16"]


def test_large_mean_and_constant_rows():
    """A mean far above the spread keeps its precision; constant rows have finite gradients."""
    import torch
    x = make(300, 128, 512, "bf16", seed=12)
    x["z"] = (x["z"].float() + 64).to(torch.bfloat16)
    x["z"][7] = 3.0
    check(Call(x)(), reference(x), "bf16", "mean 64")


@pytest.mark.parametrize("t,c,hidden,pairs", [("f32", 32, 64, 5000), ("bf16", 128, 512, 3000), ("bf16", 128, 512, 50000)])
def test_bits_repeat_on_any_stream_and_in_graphs_that_share_a_workspace(t, c, hidden, pairs):
    import torch
    a, b = Call(make(pairs, c, hidden, t, seed=13)), Call(checkpointed(make(pairs // 2 + 1, c, hidden, t, seed=14)))
    want = [{k: v.clone() for k, v in call().items()} for call in (a, b)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for v in a.out.values():
        v.fill_(7.0)
    torch.cuda.synchronize()
    a(stream=side)
    side.synchronize()
    assert all(torch.equal(a.out[k], want[0][k]) for k in NAMES)
    graphs = []
    for call in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(ws=a.ws)
        graphs.append(g)
    for turn in range(3):
        for v in list(a.out.values()) + list(b.out.values()):
            v.fill_(7.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for call, w in zip((a, b), want):
            assert all(torch.equal(call.out[k], w[k]) for k in NAMES), turn


def test_stripes_add_up():
    """Two stripes' gradients of the weights add up to the whole's; dz are its rows."""
    import torch
    x = make(4001, 128, 512, "bf16", seed=15)
    whole = reference(x)
    parts = [Call({**x, "z": x["z"][s], "dout": x["dout"][s]}, "f32")() for s in (slice(0, 1500), slice(1500, None))]
    got = {k: parts[0][k].double() + parts[1][k].double() for k in NAMES[1:]}
    got["dz"] = torch.cat([p["dz"] for p in parts])
    check(got, whole, "bf16", "stripes")


def test_more_than_2_31_elements():
    """The last thousand pairs of 16.8 million, the others without a gradient."""
    import torch
    n, tail = (1 << 24) + 1003, 1000
    x = make(tail, 128, 512, "bf16", seed=16)
    big = {k: torch.zeros((n, 128), dtype=torch.bfloat16, device="cuda") for k in ("z", "dout")}
    for k in big:
        big[k][-tail:] = x[k]
    got = Call({**x, **big}, "f32")()
    want = reference(x)
    assert not got["dz"][:-tail].any()
    got["dz"] = got["dz"][-tail:]
    check(got, want, "bf16", "2^24 pairs")


@pytest.mark.parametrize("factor", [2.0 ** -12, 2.0 ** -70])
@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_pairs_without_a_gradient_beside_small_ones(t, c, hidden, factor):
    """Masked pairs: rows of zeros in dout get exact zeros and add nothing, however small the others are."""
    x = make(700, c, hidden, t, seed=17)
    x["dout"] = x["dout"] * factor
    x["dout"][::3] = 0.0
    got = Call(x, "f32")()
    assert not got["dz"][::3].any()
    check(got, reference(x), t, factor)


@pytest.mark.parametrize("what", ["w1", "w2", "w3", "all"])
@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_units_without_weights_beside_small_ones(t, c, hidden, what, monkeypatch):
    """A hidden width that is filled up with zeros: those units neither add anything nor cost the others their
    precision, however small the others' weights are. z is small and its LayerNorm without eps, so that what the
    weights make of dz is not hidden by dout; beta is left out, of which W1 and W2 would make values of other sizes."""
    import sys
    monkeypatch.setattr(sys.modules[__name__], "EPS", 0.0)
    x = make(400, c, hidden, t, seed=18)
    x["beta"] = None
    x["z"] = x["z"] * 2.0 ** -60
    for k in ("w1", "w2", "w3"):
        x[k] = x[k] * 2.0 ** -14
        if what in (k, "all"):
            (x[k].T if k == "w3" else x[k])[hidden // 3:] = 0.0
    got, want = Call(x, "f32")(), reference(x)
    assert float((want["dz"] - x["dout"].double()).norm()) > 8 * float(x["dout"].double().norm())
    check(got, want, t, what)


def test_f32_more_threads_than_one_launch_holds():
    """2^29 pairs and more, of which a thread takes an eighth of one. The last thousand, the others without a gradient."""
    import torch
    n, tail = (1 << 29) + 1003, 1000
    x = make(tail, 2, 3, "f32", seed=19)
    big = {k: torch.zeros((n, 2), device="cuda") for k in ("z", "dout")}
    for k in big:
        big[k][-tail:] = x[k]
    got, want = Call({**x, **big})(), reference(x)
    assert not got["dz"][:-tail].any()
    got["dz"] = got["dz"][-tail:]
    check(got, want, "f32", "2^29 pairs")


@pytest.mark.parametrize("saved", ["whole", "checkpoint"])
def test_more_pairs_than_are_taken_at_a_time_in_place(saved):
    """2^20 pairs and a few: in dout's place, and without dz, the bits of the call with a buffer of its own."""
    import torch
    n = (1 << 20) + 100
    x = make(1, 128, 512, "bf16", seed=20)
    g = torch.Generator(device="cuda").manual_seed(21)
    for k in ("z", "dout"):
        x[k] = torch.randn((n, 128), generator=g, device="cuda", dtype=torch.bfloat16)
    x = checkpointed(x) if saved == "checkpoint" else x
    want = {k: v.clone() for k, v in Call(x)().items()}
    sums = Call(x, want=NAMES[1:])()
    assert all(torch.equal(sums[k], want[k]) for k in NAMES[1:])
    got = Call({**x, "dout": x["dout"].clone()}, in_place=True)()
    assert all(torch.equal(got[k], want[k]) for k in NAMES)


@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_two_calls_at_once(t, c, hidden):
    """Calls on two streams with workspaces of their own do not touch each other."""
    import torch
    calls = [Call(make(20000 + 777 * k, c, hidden, t, seed=22 + k)) for k in range(2)]
    want = [{k: v.clone() for k, v in call().items()} for call in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for turn in range(3):
        for call in calls:
            for v in call.out.values():
                v.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(4):
            for call, stream in zip(calls, streams):
                call(stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(call.out[k], w[k]) for call, w in zip(calls, want) for k in NAMES), turn
