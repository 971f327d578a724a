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


# ----------------------------------------------------------------------------- each unit by itself
def unit_rows(grads):
    """[3, hidden, c]: each unit's row of W1's and W2's gradients and column of W3's, in 64 bits."""
    import torch
    return torch.stack([grads["dw1"].double(), grads["dw2"].double(), grads["dw3"].double().T])


def unit_scales(x):
    """[2, 3, hidden], of the terms dA N, dB N and H dout of each unit and of those terms' slopes in A: the root of the sum of
    their squares, or the norm of their sum where that is more."""
    import torch
    z, dout = values(x), x["dout"].double()
    zh = (z - z.mean(dim=1, keepdim=True)) / torch.sqrt(z.var(dim=1, keepdim=True, correction=0) + EPS)
    n = zh * x["gamma"].double() + x["beta"].double()
    a, b, dh = n @ x["w1"].double().T, n @ x["w2"].double().T, dout @ x["w3"].double()
    s = 1 / (1 + torch.exp(-a))
    silu, slope, bend = a * s, s + a * s * (1 - s), s * (1 - s) * (2 + a * (1 - 2 * s))
    terms = ((dh * b * slope, n), (dh * silu, n), (silu * b, dout)), ((dh * b * bend, n), (dh * slope, n), (slope * b, dout))
    return torch.stack([torch.stack([torch.maximum((f.square() * v.square().sum(dim=1)[:, None]).sum(dim=0).sqrt(), (f.T @ v).norm(dim=1))
                                     for f, v in t]) for t in terms])


def check_units(x, got, want, t, what, units=slice(None), off=None):
    """Each unit by itself. Its row is a sum over the pairs of terms of either sign, by chance far smaller than the terms make
    likely (with a beta of 4 each row is mostly beta times a sum of numbers, which may be near 0 for one unit of many), or up to
    three times larger. The errors of zh, dout and the gate are independent from pair to pair and add up to the terms' relative error
    times the root of the sum of their squares; those of a unit's weights are the same for all pairs and add up to that
    times the sum itself. The larger of the two is what the error is measured by. The terms' relative error is that of the
    tensors. Beside it stands that of A, `off`, which their slopes in A multiply alike. bf16: A is a sum of c products w zh of two operands of 11 bits, each off by
    0.42 2^-11 in the root mean square; here |w| < 0.3 and zh is about 1: 0.3 sqrt(2 128) 0.42 2^-11 = 1e-3; twice that, as
    for the tensors. fp32: A's partial sums are up to 60 here, and A is off by 2^-22 60 at most."""
    off = {"bf16": 2e-3, "f32": 60 * 2.0 ** -22}[t] if off is None else off
    error, (term, slope) = (unit_rows(got) - unit_rows(want)).norm(dim=2), unit_scales(x)
    most = (TOL[t] * term + off * slope).clamp(min=1e-300)
    part, rel = (error / most)[:, units], (error / term.clamp(min=1e-300))[:, units]
    print(what, "dw1, dw2, dw3: errors by the terms up to", ["%.2e" % float(v) for v in rel.max(dim=1).values],
          "of the limit up to", ["%.2f" % float(v) for v in part.max(dim=1).values], flush=True)
    assert float(part.max()) <= 1.0, what


@pytest.mark.parametrize("saved", ["whole", "checkpoint"])
@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_units_whose_gates_are_shut_keep_their_precision(t, c, hidden, saved):
    """Units with A ~ N(m, 1), m from 0 to -60: a shut gate's sigmoid is as small as e^-62, and so is all that its unit has of
    a gradient; of its own size that is as precise as any other's."""
    import torch
    x = make(3000, c, hidden, t, seed=30, offset=0.0)
    x["gamma"], x["beta"] = torch.ones(c, device="cuda"), torch.full((c,), 4.0, device="cuda")
    m = torch.tensor([0.0, -4.0, -8.0, -10.0, -12.0, -14.0, -16.0, -18.0, -22.0, -30.0, -45.0, -60.0], device="cuda")
    m = m[torch.arange(hidden, device="cuda") % len(m)]
    x["w1"] = x["w1"] - x["w1"].mean(dim=1, keepdim=True) + m[:, None] / (4 * c)
    x = checkpointed(x) if saved == "checkpoint" else x
    check_units(x, Call(x, "f32")(), reference(x), t, (t, saved))


@pytest.mark.parametrize("factor", [2.0 ** -10, 2.0 ** -14, 2.0 ** -18, 2.0 ** -26, 2.0 ** -40])
@pytest.mark.parametrize("shut", [0.0, -8.0, -16.0])
@pytest.mark.parametrize("t,c,hidden", [("f32", 32, 64), ("bf16", 128, 512)])
def test_small_pairs_count_where_the_large_have_no_part(t, c, hidden, shut, factor):
    """Every second pair has a gradient `factor` times as large as the others', whose gates are shut (A near -60) in every fourth
    unit: what those units have of a gradient is of the small pairs alone, and as precise as any. `shut`: A of the small pairs there."""
    import torch
    n = 3000
    x = make(n, c, hidden, t, seed=31, offset=0.0)
    units = torch.arange(hidden, device="cuda") % 4 == 0
    x["gamma"], x["beta"] = torch.ones(c, device="cuda"), torch.full((c,), 4.0, device="cuda")
    # z = +-(1, .., -1, ..) + half as much of a normal one that is orthogonal to it; 1.118 = sqrt(1.25), the root mean square of its
    # rows, so that A = shut - 30 -+ 30 in those units
    side = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1.0, -1.0)
    half = torch.cat([torch.ones(c // 2, device="cuda"), -torch.ones(c - c // 2, device="cuda")])
    z = x["z"].float()
    z = z - z.mean(dim=1, keepdim=True)
    z = z - (z @ half / c)[:, None] * half
    z = z / z.square().mean(dim=1, keepdim=True).sqrt()
    x["z"] = (z * 0.5 + side[:, None] * half).to(x["z"].dtype)
    w = x["w1"] - x["w1"].mean(dim=1, keepdim=True)
    w = w - (w @ half / c)[:, None] * half
    x["w1"] = torch.where(units[:, None], w - (30.0 / c) * 1.118 * half + (shut - 30.0) / (4 * c), w)
    x["dout"][1::2] *= factor
    got, want = Call(x, "f32")(), reference(x)
    check_units(x, got, want, t, (t, shut, factor, "units of the small pairs"), units)
    check_units(x, got, want, t, (t, shut, factor, "the others"), ~units)


@pytest.mark.parametrize("pairs", [2000, 20000, (1 << 20) + 5000])
@pytest.mark.parametrize("order", ["open", "shut", "any"])
def test_gates_that_open_or_shut_along_the_pairs(order, pairs):
    """A from -57 to -3 in every fourth unit, from pair to pair in order, backwards or in any: what is small at first is
    far more at the end, over steps, shares and the pairs that are taken at a time. The rows of z have a root mean square of 1
    up to their own rounding, and zh is z times 1 + d, |d| < 2^-9: rounded to 11 bits much of a row loses the same part of up to 2^-12,
    so its errors are not independent, and A's 30 of the first half against the second are off by 30 2^-12 at most."""
    import torch
    x = make(1, 128, 512, "bf16", seed=34)
    g = torch.Generator(device="cuda").manual_seed(35)
    x["gamma"], x["beta"] = torch.ones(128, device="cuda"), torch.full((128,), 4.0, device="cuda")
    half = torch.cat([torch.ones(64, device="cuda"), -torch.ones(64, device="cuda")])
    along = torch.linspace(-0.9, 0.9, pairs, device="cuda")
    along = along.flip(0) if order == "shut" else along[torch.randperm(pairs, generator=g, device="cuda")] if order == "any" else along
    z = torch.randn((pairs, 128), generator=g, device="cuda")
    z = z - z.mean(dim=1, keepdim=True)
    z = z - (z @ half / 128)[:, None] * half
    z = z / z.square().mean(dim=1, keepdim=True).sqrt()
    x["z"] = (along[:, None] * half + (1 - along.square()).sqrt()[:, None] * z).to(torch.bfloat16)
    x["dout"] = torch.randn((pairs, 128), generator=g, device="cuda", dtype=torch.bfloat16)
    units = torch.arange(512, device="cuda") % 4 == 0
    w = x["w1"] - x["w1"].mean(dim=1, keepdim=True)
    w = w - (w @ half / 128)[:, None] * half
    x["w1"] = torch.where(units[:, None], w + (30.0 / 128) * half - 30.0 / 512, w)
    got, want = Call(x, "f32")(), reference(x)
    check_units(x, got, want, "bf16", (order, pairs), off=30 * 2.0 ** -12)
    again = Call(x, "f32", want=NAMES[1:])()
    assert all(torch.equal(again[k], got[k]) for k in NAMES[1:])


def gradients_of_rounded_operands(x):
    """The gradients in 64 bits by the formulas, with zh and the rows of W1 diag(gamma), W2 diag(gamma) and W3^T (each of a
    power of two of its own) rounded to 11 bits as the products' operands are."""
    import torch
    half = lambda v: v.to(torch.float16).double()  # noqa: E731

    def rows(w):
        e = torch.frexp(w.abs().amax(dim=1, keepdim=True)).exponent.double()
        return half(w * torch.pow(2.0, -e)) * torch.pow(2.0, e)

    z, dout, ga, be = values(x), x["dout"].double(), x["gamma"].double(), x["beta"].double()
    mu = z.mean(dim=1, keepdim=True)
    rstd = 1 / torch.sqrt(((z - mu) ** 2).mean(dim=1, keepdim=True) + EPS)
    exact, zh = (z - mu) * rstd, half((z - mu) * rstd)
    w1, w2 = x["w1"].double(), x["w2"].double()
    r1, r2, r3 = rows(w1 * ga), rows(w2 * ga), rows(x["w3"].double().T.contiguous())
    a, b, dh = zh @ r1.T + w1 @ be, zh @ r2.T + w2 @ be, dout @ r3.T
    s = 1 / (1 + torch.exp(-a))
    h, db, da = a * s * b, dh * a * s, dh * b * (s + a * s * (1 - s))
    g = da @ r1 + db @ r2
    t1, t2, s1, s2 = da.T @ zh, db.T @ zh, da.sum(dim=0), db.sum(dim=0)
    return {"dz": dout + rstd * (g - g.mean(dim=1, keepdim=True) - exact * (g * exact).mean(dim=1, keepdim=True)),
            "dw1": t1 * ga + s1[:, None] * be, "dw2": t2 * ga + s2[:, None] * be, "dw3": dout.T @ h,
            "dgamma": (w1 * t1 + w2 * t2).sum(dim=0), "dbeta": w1.T @ s1 + w2.T @ s2}


@pytest.mark.parametrize("mean", [0.0, 3.0, 5.0, 8.0])
@pytest.mark.parametrize("factor", [1.0, 4.0, 16.0])
def test_open_and_saturated_gates(factor, mean):
    """Large W1, and gates that are open (A ~ N(mean, factor)): sigmoid and slope have the error of A's operands, |A| times
    theirs. Beside the gradients of operands that are rounded alike that is left out, and what remains are the roundings of the
    gate and of the results: within the tensors' tolerance, whatever A is."""
    import torch
    x = make(2000, 128, 512, "bf16", seed=32, offset=0.0)
    x["beta"] = torch.full((128,), 4.0, device="cuda")
    x["w1"] = (x["w1"] - x["w1"].mean(dim=1, keepdim=True)) * factor + mean / 512
    got, want = Call(x, "f32")(), gradients_of_rounded_operands(x)
    check(got, want, "bf16", (factor, mean))
    check_units(x, got, want, "bf16", (factor, mean), off=0.0)


MANY_WIDE_F32 = [(4097, 128, 512), (9000, 128, 512), (5000, 100, 400), (4113, 256, 1024), (4100, 129, 260), (8200, 65, 130)]


@pytest.mark.parametrize("saved", ["whole", "checkpoint"])
@pytest.mark.parametrize("pairs,c,hidden", MANY_WIDE_F32)
def test_f32_many_pairs_of_wide_rows(pairs, c, hidden, saved):
    """More pairs than the workgroups of one round hold: two tiles of pairs a workgroup in dz's kernel, several turns of the
    sums' loops."""
    x = make(pairs, c, hidden, "f32", seed=pairs + c)
    x = checkpointed(x) if saved == "checkpoint" else x
    check(Call(x)(), reference(x), "f32", (pairs, c, hidden, saved))


@pytest.mark.parametrize("pairs,c,hidden", [(300, 128, 512), (9000, 128, 512), (5000, 100, 400), (4500, 140, 300)])
def test_f32_wide_rows_in_place_alone_and_again(pairs, c, hidden):
    """The bits of a call that is repeated, of one in dout's place and of each gradient alone; nothing written behind dz and the
    workspace."""
    import torch
    import paper_2607_05439_amd as dcp
    x = make(pairs, c, hidden, "f32", seed=33)
    call = Call(x)
    dz = torch.full((pairs + 40, c), 7.0, device="cuda")
    ws = torch.full((call.ws.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
    call.out["dz"] = dz[:pairs]
    call.grads = dcp.make_transition_gradients(*[call.out[k] for k in NAMES], dtype=0)
    size, whole = call.ws.numel(), None
    for turn in range(3):
        dcp.dcp_pair_transition_backward(*call.dims, code("f32"), EPS, x["w1"], x["w2"], x["w3"], x["gamma"], x["beta"], x["z"],
                                         None, x["dout"], call.grads, ws, size, None)
        now = {k: v.clone() for k, v in call.out.items()}
        assert turn == 0 or all(torch.equal(now[k], whole[k]) for k in NAMES), turn
        whole = now
    assert (dz[pairs:] == 7.0).all() and (ws[size:] == 255).all()
    for k in NAMES:
        got = Call(x, want=(k,))()
        assert all(torch.equal(got[j], whole[j]) if j == k else (got[j] == 7.0).all() for j in NAMES), k
    got = Call({**x, "dout": x["dout"].clone()}, in_place=True)()
    assert all(torch.equal(got[k], whole[k]) for k in NAMES)
    check(whole, reference(x), "f32", (pairs, c, hidden))
