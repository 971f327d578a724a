"""The relative position encoding and its table's gradient through the C-ABI against the same in
64 bits (GPU).

Tolerances. Forward: up to four additions in fp32 of numbers of the size of the sum, then the rounding to the
result's type: 4 half steps of 2^-24 of the largest of them, and half a step of the type (2^-8 bf16). Backward: a sum of
fp32 additions: a chain has at most the pairs of one share in it, and its partial sums' roundings add up like a random walk,
under 2^-24 sqrt(chain length) of the result's scale, 1e-5 for chains up to 2^14 additions (asserted of each
bucket's row against the root of its number of pairs times the gradients' size, the scale of a sum of
random signs)."""
import pytest

pytestmark = pytest.mark.gpu

PAPER = (32, 32, 2, 0)


def dtypes():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def code(t):
    import paper_2607_05439_amd as dcp
    return dcp.DCP_BF16 if t == "bf16" else dcp.DCP_F32


def fields_of(n, radii, seed=0, order="chains"):
    """(position, group, radius) per field: chains of 80 residues, some split into tokens; or any order at all."""
    import torch
    g = torch.Generator().manual_seed(seed)
    token = torch.arange(n)
    if order == "any":
        pos = [torch.randint(-60, 60, (n,), generator=g) for _ in radii]
        grp = [torch.randint(0, 3, (n,), generator=g) for _ in radii]
    else:
        chain, within = token // 80, token % 80
        residue = torch.cumsum((torch.rand(80, generator=g) < 0.9).long(), 0)[within]
        pos = [residue, token, chain // 2, torch.zeros_like(token)]
        grp = [chain, chain * 1000 + residue, chain % 2, chain % 2]
    return [(p.int().cuda(), q.int().cuda(), r) for p, q, r in zip(pos, grp, radii)]


def n_buckets(fields):
    return sum(2 * r + 2 for _, _, r in fields)


def buckets(fields, row0, rows):
    """[rows, n] per field, from the table's first row."""
    import torch
    out, first = [], 0
    for pos, grp, r in fields:
        p = pos.long()
        grp = torch.zeros_like(p) if grp is None else grp.long()
        i = slice(row0, row0 + rows)
        d = torch.clamp(p[i, None] - p[None, :], min=-r, max=r) + r
        d[grp[i, None] != grp[None, :]] = 2 * r + 1
        out.append(d + first)
        first += 2 * r + 2
    return out


def forward(n, row0, rows, c, t, fields, table, z, out=None):
    import torch
    import paper_2607_05439_amd as dcp
    out = torch.full((rows, n, c), 7.0, dtype=dtypes()[t], device="cuda") if out is None else out
    dcp.dcp_relative_position(n, row0, rows, c, code(t), dcp.make_relative_fields(fields), table, z, out)
    return out


class Backward:
    def __init__(self, n, row0, rows, c, t, fields, dz):
        import torch
        import paper_2607_05439_amd as dcp
        self.args, self.dz = (n, row0, rows, c, code(t)), dz
        self.keep, self.fields = fields, dcp.make_relative_fields(fields)
        self.out = torch.full((n_buckets(fields), c), 7.0, device="cuda")
        size = dcp.dcp_relative_position_backward_workspace_size(n, rows, c, self.fields)
        self.ws = torch.full((max(size, 256),), 255, dtype=torch.uint8, device="cuda")

    def __call__(self, stream=None, ws=None):
        import paper_2607_05439_amd as dcp
        ws = self.ws if ws is None else ws
        dcp.dcp_relative_position_backward(*self.args, self.fields, self.dz, self.out, ws, ws.numel(), stream)
        return self.out


def gradient(fields, row0, rows, dz):
    """dtable in 64 bits and the number of pairs of each bucket."""
    import torch
    out = torch.zeros((n_buckets(fields), dz.shape[2]), dtype=torch.float64, device="cuda")
    count = torch.zeros(n_buckets(fields), dtype=torch.float64, device="cuda")
    flat = dz.reshape(-1, dz.shape[2]).double()
    for b in buckets(fields, row0, rows):
        hot = torch.zeros((out.shape[0], b.numel()), dtype=torch.float64, device="cuda").scatter_(0, b.flatten()[None], 1.0)
        out += hot @ flat
        count += hot.sum(dim=1)
    return out, count


def check_gradient(got, fields, row0, rows, dz, what):
    want, count = gradient(fields, row0, rows, dz)
    size = dz.double().square().mean().sqrt()
    off = (got.double() - want).norm(dim=1) / (size * (count * dz.shape[2]).sqrt()).clamp(min=1e-300)
    print(what, "largest error of a bucket %.2e, buckets without pairs %d" % (float(off.max()), int((count == 0).sum())), flush=True)
    assert not got[count == 0].any() and float(off.max()) <= 1e-5


CASES = [(1, 0, 1, 1, (0,)), (2, 1, 1, 8, (1, 0)), (63, 0, 63, 16, (5,)), (64, 3, 20, 32, PAPER), (65, 0, 65, 33, (3, 2)),
         (100, 50, 50, 7, (127, 127, 127, 127)), (130, 0, 130, 128, PAPER), (333, 100, 77, 128, PAPER), (257, 0, 40, 64, (16, 16)),
         (90, 0, 90, 200, (20, 1, 3, 0)), (70, 0, 9, 1024, (4,)), (81, 2, 30, 1000, (40, 32)), (301, 0, 301, 24, (48, 32, 2))]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["chains", "any"])
@pytest.mark.parametrize("n,row0,rows,c,radii", CASES)
def test_encoding_and_gradient(n, row0, rows, c, radii, order, t):
    import torch
    g = torch.Generator().manual_seed(n + c)
    fields = fields_of(n, radii, seed=n, order=order)
    table = torch.randn((n_buckets(fields), c), generator=g).cuda()
    z = torch.randn((rows, n, c), generator=g).to(dtypes()[t]).cuda()
    add = sum(table.double()[b] for b in buckets(fields, row0, rows))
    big = table.abs().max() * len(radii) + z.abs().max().float()
    for z_in in (z, None):
        want = add if z_in is None else add + z.double()
        got = forward(n, row0, rows, c, t, fields, table, z_in).double()
        tol = 4 * 2.0 ** -24 * big + (2.0 ** -8 if t == "bf16" else 2.0 ** -24) * want.abs()
        assert ((got - want).abs() <= tol).all()
    y = z.clone()
    assert torch.equal(forward(n, row0, rows, c, t, fields, table, y, out=y), forward(n, row0, rows, c, t, fields, table, z))
    dz = (z.float() / 512).to(z.dtype)
    check_gradient(Backward(n, row0, rows, c, t, fields, dz)(), fields, row0, rows, dz, (n, c, radii, order, t))


def test_one_group_and_far_positions():
    """A field without groups; positions whose difference passes 32 bits."""
    import torch
    pos = torch.tensor([-(1 << 31), (1 << 31) - 1, 0, 5, -5, (1 << 31) - 3], dtype=torch.int32).cuda()
    fields = [(pos, None, 3)]
    table = torch.randn((8, 16), generator=torch.Generator().manual_seed(1)).cuda()
    got = forward(6, 0, 6, 16, "f32", fields, table, None)
    assert torch.equal(got, table[buckets(fields, 0, 6)[0]])
    check_gradient(Backward(6, 0, 6, 16, "f32", fields, got)(), fields, 0, 6, got, "far")


def test_the_gradient_against_differences():
    """The encoding is linear in its table: its difference along a direction is the gradient's product with
    that, up to the roundings of both."""
    import torch
    g = torch.Generator().manual_seed(2)
    fields = fields_of(100, PAPER)
    table, v = (torch.randn((n_buckets(fields), 32), generator=g).cuda() for _ in range(2))
    dz = torch.randn((100, 100, 32), generator=g).cuda()
    f = lambda w: (forward(100, 0, 100, 32, "f32", fields, w, None).double() * dz.double()).sum()  # noqa: E731
    want, have = float(f(table + v) - f(table - v)) / 2, float((Backward(100, 0, 100, 32, "f32", fields, dz)().double() * v).sum())
    assert abs(want - have) <= 1e-5 * float(dz.norm() * 100 * 32 ** 0.5)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("c", [32, 128, 20])
def test_off_alignment_and_nothing_written_outside(c, t):
    import torch
    import paper_2607_05439_amd as dcp
    n, rows = 70, 30
    fields = fields_of(n, PAPER)
    g = torch.Generator().manual_seed(3)
    table = torch.randn((n_buckets(fields), c), generator=g).cuda()
    z = torch.randn((rows, n, c), generator=g).to(dtypes()[t]).cuda()
    want, back = forward(n, 10, rows, c, t, fields, table, z), Backward(n, 10, rows, c, t, fields, z)
    flat = [torch.full((v.numel() + 8,), 7.0, dtype=v.dtype, device="cuda") for v in (z, z, table, back.out)]
    zi, zo, tb, dt = (r[3:3 + v.numel()].view(v.shape) for r, v in zip(flat, (z, z, table, back.out)))
    zi.copy_(z), tb.copy_(table)
    forward(n, 10, rows, c, t, fields, tb, zi, out=zo)
    assert torch.equal(zo, want)
    size = back.ws.numel()
    ws = torch.full((size + 1024,), 255, dtype=torch.uint8, device="cuda")
    dcp.dcp_relative_position_backward(*back.args, back.fields, zi, dt, ws, size, None)
    check_gradient(dt, fields, 10, rows, z, "off alignment")
    assert (ws[size:] == 255).all()
    for r, v in zip(flat, (z, z, table, back.out)):
        assert (r[:3] == 7).all() and (r[3 + v.numel():] == 7).all()


def test_without_rows():
    import torch
    fields = fields_of(50, PAPER)
    back = Backward(50, 50, 0, 128, "bf16", fields, None)
    assert not back().any()
    forward(50, 20, 0, 128, "bf16", fields, torch.zeros((n_buckets(fields), 128), device="cuda"), None)


def test_values_that_are_not_finite_stay_in_their_buckets():
    import torch
    fields = fields_of(160, PAPER)
    dz = torch.randn((160, 160, 128), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    clean = Backward(160, 0, 160, 128, "bf16", fields, dz)().clone()
    dz[17, 90, 5] = float("inf")
    got = Backward(160, 0, 160, 128, "bf16", fields, dz)()
    hit = torch.zeros_like(clean, dtype=torch.bool)
    for b in buckets(fields, 17, 1):
        hit[b[0, 90], 5] = True
    assert (got[hit] == float("inf")).all() and torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("t,c", [("bf16", 128), ("f32", 32), ("f32", 13)])
def test_bits_repeat_on_any_stream_and_in_graphs_that_share_a_workspace(t, c):
    import torch
    g = torch.Generator().manual_seed(5)
    calls = []
    for n, rows in ((300, 300), (150, 40)):
        dz = torch.randn((rows, n, c), generator=g).to(dtypes()[t]).cuda()
        calls.append(Backward(n, 0, rows, c, t, fields_of(n, PAPER), dz))
    want = [call().clone() for call in calls]
    side = torch.cuda.Stream()
    calls[0].out.fill_(7.0)
    torch.cuda.synchronize()
    calls[0](stream=side)
    side.synchronize()
    assert torch.equal(calls[0].out, want[0])
    graphs = []
    for call in calls:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(ws=calls[0].ws)
        graphs.append(gr)
    for _ in range(3):
        for call in calls:
            call.out.fill_(7.0)
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(call.out, w) for call, w in zip(calls, want))


def test_stripes_add_up_and_long_sums():
    """Ones: every bucket's gradient is its number of pairs, exactly below 2^24."""
    import torch
    n, fields = 1501, fields_of(1501, PAPER)
    dz = torch.ones((n, n, 128), dtype=torch.bfloat16, device="cuda")
    got = Backward(n, 0, n, 128, "bf16", fields, dz)().clone()
    count = torch.zeros(n_buckets(fields), dtype=torch.long, device="cuda")
    for b in buckets(fields, 0, n):
        count += torch.bincount(b.flatten(), minlength=n_buckets(fields))
    assert torch.equal(got.long(), count[:, None].expand(-1, 128))
    parts = [Backward(n, r, e - r, 128, "bf16", fields, dz[r:e])().clone() for r, e in ((0, 700), (700, 701), (701, n))]
    assert torch.equal(sum(parts), got)


def test_more_than_2_32_elements():
    """The last two rows of a stripe of 5100 x 6600 pairs; the others hold zeros."""
    import torch
    n, rows, row0 = 6600, 5100, 1000
    fields = fields_of(n, PAPER)
    g = torch.Generator().manual_seed(6)
    z = torch.zeros((rows, n, 128), dtype=torch.bfloat16, device="cuda")
    z[-2:] = torch.randn((2, n, 128), generator=g).to(torch.bfloat16).cuda()
    got = Backward(n, row0, rows, 128, "bf16", fields, z)()
    check_gradient(got, fields, row0 + rows - 2, 2, z[-2:], "5100 x 6600")
    table = torch.randn((n_buckets(fields), 128), generator=g).cuda()
    want = forward(n, row0 + rows - 2, 2, 128, "bf16", fields, table, z[-2:])
    forward(n, row0, rows, 128, "bf16", fields, table, z, out=z)
    assert torch.equal(z[-2:], want)


def test_more_threads_than_one_launch_holds():
    """66000 tokens of one channel: more than 2^32 pairs, a lane each. Rows of all launches."""
    import torch
    import paper_2607_05439_amd as dcp
    n = 66000
    fields = [(torch.arange(n, dtype=torch.int32, device="cuda"), None, 1)]
    table = torch.tensor([[1.0], [2.0], [3.0], [4.0]], device="cuda")
    z = torch.full((n, n, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    dcp.dcp_relative_position(n, 0, n, 1, dcp.DCP_BF16, dcp.make_relative_fields(fields), table, None, z)
    for rows in (slice(0, 100), slice(30000, 30100), slice(n - 2000, n)):
        assert torch.equal(z[rows, :, 0].float(), table[:, 0][buckets(fields, rows.start, rows.stop - rows.start)[0]])


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("radii", [(0,), (32, 32, 2, 0), (127, 127)])
def test_long_runs_of_alike_pairs(radii, t):
    """Few groups, so that most blocks of pairs are alike in all fields, over rows and tiles, and the runs end in each way:
    at a group's end, at the diagonal, at a value that is not finite and at a workgroup's last pair."""
    import torch
    n = 700
    token = torch.arange(n)
    fields = [((token // 7).int().cuda(), (token // (100 * (f + 1))).int().cuda(), r) for f, r in enumerate(radii)]
    dz = torch.randn((n, n, 40), generator=torch.Generator().manual_seed(23)).to(dtypes()[t]).cuda()
    clean = Backward(n, 0, n, 40, t, fields, dz)().clone()
    check_gradient(clean, fields, 0, n, dz, (radii, t))
    dz[300, 650, 7] = float("-inf")
    got, hit = Backward(n, 0, n, 40, t, fields, dz)(), torch.zeros_like(clean, dtype=torch.bool)
    for b in buckets(fields, 300, 1):
        hit[b[0, 650], 7] = True
    assert (got[hit] == float("-inf")).all()
    dz[300, 650, 7] = 0.0
    assert torch.equal(got[~hit], Backward(n, 0, n, 40, t, fields, dz)()[~hit])


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("width", [16, 31, 32, 77])
def test_many_classes_of_alike_pairs(width, t):
    """Blocks of pairs with two kinds of buckets at most, but more kinds in a stripe than are summed side by side."""
    import torch
    n, rows = 650, 90
    token = torch.arange(n)
    fields = [((token // width).int().cuda(), None, 127), ((token // width % 5).int().cuda(), (token // width % 3).int().cuda(), 3)]
    dz = torch.randn((rows, n, 72), generator=torch.Generator().manual_seed(24)).to(dtypes()[t]).cuda()
    got = Backward(n, 500, rows, 72, t, fields, dz)().clone()
    check_gradient(got, fields, 500, rows, dz, (width, t))
    assert torch.equal(Backward(n, 500, rows, 72, t, fields, dz)(), got)


def test_sums_past_the_largest_number_stay_in_their_buckets():
    import torch
    n = 192
    token = torch.arange(n, dtype=torch.int32, device="cuda")
    fields = [(token // 64, None, 2)]
    dz = torch.ones((n, n, 32), dtype=torch.bfloat16, device="cuda")
    dz[64:128, :64, 3] = 3e38  # bucket 3: 1 to the left
    got = Backward(n, 0, n, 32, "bf16", fields, dz)()
    want = torch.tensor([1, 2, 3, 2, 1, 0], device="cuda")[:, None].expand(6, 32) * 4096.0
    assert got[3, 3] >= 3e38
    got[3, 3] = want[3, 3]
    assert torch.equal(got, want)


@pytest.mark.parametrize("t,c", [("f32", 32), ("bf16", 32), ("f32", 100), ("bf16", 128)])
@pytest.mark.parametrize("kinds", ["alike", "two kinds", "mixed"])
def test_sums_past_the_largest_number_are_infinite(kinds, t, c):
    """Of either sign, in their own bucket alone, whether the pairs are summed by kind or each by itself; the largest finite
    number alone stays itself."""
    import torch
    n = 192
    top = 3.4028234663852886e38 if t == "f32" else 3.3895313892515355e38
    token = torch.arange(n, dtype=torch.int32, device="cuda")
    width = {"alike": 64, "two kinds": 24, "mixed": 1}[kinds]
    fields = [(token // width, None, 2)]
    dz = torch.ones((n, n, c), device="cuda").to(dtypes()[t])
    where = buckets(fields, 0, n)[0]
    for b, channel, value in ((3, 3, 3e38), (1, 5, -3e38)):
        dz[..., channel] = torch.where(where == b, value, 1.0).to(dz.dtype)
    dz[..., 9] = 0.0
    i, j = (where == 4).nonzero()[0].tolist()
    dz[i, j, 9] = top
    got = Backward(n, 0, n, c, t, fields, dz)()
    want = torch.bincount(where.flatten(), minlength=6).float()[:, None].repeat(1, c)
    want[3, 3], want[1, 5], want[:, 9], want[4, 9] = float("inf"), float("-inf"), 0.0, top
    print(kinds, t, got[:, [0, 3, 5, 9]].tolist(), flush=True)
    assert torch.equal(got, want)


@pytest.mark.parametrize("t,c", [("f32", 32), ("bf16", 32), ("bf16", 128)])
def test_two_pairs_past_the_largest_number(t, c):
    """One workgroup's sum alone passes it, of pairs that are alike in all fields; the buckets beside it stay as they are."""
    import torch
    n = 64
    token = torch.arange(n, dtype=torch.int32, device="cuda")
    fields = [(token // 32, None, 1), (token * 0, None, 0)]
    dz = torch.ones((n, n, c), device="cuda").to(dtypes()[t])
    dz[40, 50:52, 3], dz[40, 50:52, 5] = 3e38, -3e38
    got = Backward(n, 0, n, c, t, fields, dz)()
    want = torch.cat([torch.bincount(b.flatten(), minlength=6).float() for b in buckets(fields, 0, n)]).view(2, 6).sum(dim=0)[:, None].repeat(1, c)
    for channel, value in ((3, float("inf")), (5, float("-inf"))):
        want[1, channel] = want[4, channel] = value
    assert torch.equal(got, want)
