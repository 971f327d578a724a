"""8-bit activation checkpoints through the C-ABI: codes, exponents and values read back are exactly the
definition's (powers of two leave nothing to round but the codes; GPU)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def code(t):
    import torch
    import paper_2607_05439_amd as dcp
    return dcp.DCP_BF16 if t == torch.bfloat16 else dcp.DCP_F32


def definition(x):
    """codes, exponent bytes and values of fp32 rows [n, c] in 64 bits, block by block."""
    n, c = x.shape
    blocks = -(-c // 32)
    codes, exps, vals = np.zeros((n, c), np.int8), np.zeros((n, blocks), np.uint8), np.zeros((n, c))
    for r in range(n):
        for b in range(blocks):
            s = slice(32 * b, min(32 * b + 32, c))
            v = x[r, s].astype(np.float64)
            if not np.isfinite(v).all():
                exps[r, b], vals[r, s] = 255, np.nan
                continue
            e = -126
            top = np.abs(v).max()
            if top > 0:
                e = max(int(np.frexp(top)[1]) - 9, -126)
                while np.rint(np.ldexp(top, -e)) > 127:
                    e += 1
                e = min(e, 121)  # one more would pass the largest fp32 number
            codes[r, s] = np.clip(np.rint(np.ldexp(v, -e)), -127, 127)
            exps[r, b], vals[r, s] = e + 127, np.ldexp(codes[r, s].astype(np.float64), e)
    return codes, exps, vals


def pack(x):
    import torch
    import paper_2607_05439_amd as dcp
    n, c = x.shape
    codes = torch.full((n, c), 99, dtype=torch.int8, device="cuda")
    exps = torch.full((n, -(-c // 32)), 99, dtype=torch.uint8, device="cuda")
    dcp.dcp_checkpoint_pack(n, c, code(x.dtype), x, codes, exps)
    return codes, exps


def unpack(codes, exps, dtype):
    import torch
    import paper_2607_05439_amd as dcp
    y = torch.full(codes.shape, 7.0, dtype=dtype, device="cuda")
    dcp.dcp_checkpoint_unpack(codes.shape[0], codes.shape[1], code(dtype), codes, exps, y)
    return y


def same(x):
    import torch
    host = x.float().cpu().numpy()
    want = definition(host)
    codes, exps = pack(x)
    finite = np.repeat(want[1] != 255, 32, axis=1)[:, :host.shape[1]]
    assert np.array_equal(codes.cpu().numpy()[finite], want[0][finite])
    assert np.array_equal(exps.cpu().numpy(), want[1])
    for dtype in (torch.float32, torch.bfloat16):
        y = unpack(codes, exps, dtype).double().cpu().numpy()
        assert np.array_equal(y, want[2], equal_nan=True), dtype
    return want


SHAPES = [(1, 1), (1, 32), (3, 31), (2, 33), (7, 64), (5, 100), (40, 128), (333, 384), (9, 1000), (130, 96), (4, 4096)]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
def test_is_the_definition(rows, c, t):
    import torch
    g = torch.Generator().manual_seed(rows + c)
    x = torch.randn((rows, c), generator=g) * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g).float())
    want = same(x.to(torch.float32 if t == "f32" else torch.bfloat16).cuda())
    assert np.abs(want[0]).max() <= 127


def test_borders():
    """Largest magnitudes around 127.5 steps, ties, zeros of either sign, the smallest and the largest
    numbers, subnormal ones, and what is not finite."""
    import torch
    rows = []
    for top in (127.0, 127.49, 127.5, 127.51, 128.0, 255.0, 255.02, 64.0, 63.75, 1.0):
        for e in (0, -126, -130, -149, 100, 120):
            v = np.float32(top) * 2.0 ** e
            if v < 3.4e38:
                rows.append([v, -v, 0.5 * 2.0 ** e, 1.5 * 2.0 ** e, 2.5 * 2.0 ** e, -2.5 * 2.0 ** e, 0.0, -0.0])
    for v in (0.0, -0.0, 1e-45, 1.2e-38, 3.4028235e38, -3.4028235e38, np.nan, np.inf, -np.inf):
        rows.append([v] + [1.0] * 7)
        rows.append([v] + [0.0] * 7)
    same(torch.tensor(np.array(rows, np.float32)).cuda())
    x = torch.zeros((6, 96), device="cuda")
    x[1, 40], x[2, 95], x[3, 0] = float("nan"), float("inf"), 1.0  # a block alone is lost
    same(x)


def test_the_error_is_at_most_half_a_step():
    """Half a step is 2^(e-1). e - 1 would not do: the largest magnitude is at least 127.5 2^(e-1), and half a
    step at most 1/127.5 of it."""
    import torch
    x = torch.randn((500, 128), generator=torch.Generator().manual_seed(1)).cuda()
    y = unpack(*pack(x), torch.float32)
    top = x.view(500, 4, 32).abs().amax(dim=2, keepdim=True)
    assert ((x - y).view(500, 4, 32).abs() <= top / 127.5).all() and ((x - y).abs() > 0).any()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("c", [32, 128, 100])
def test_off_alignment_and_nothing_written_outside(t, c):
    import torch
    dt = torch.float32 if t == "f32" else torch.bfloat16
    x = torch.randn((51, c), generator=torch.Generator().manual_seed(2)).to(dt).cuda()
    codes, exps = pack(x)
    y = unpack(codes, exps, dt)
    for off in (1, 2, 4):
        room = lambda like: torch.full((like.numel() + 8,), 7, dtype=like.dtype, device="cuda")  # noqa: E731
        rx, rc, re, ry = room(x), room(codes), room(exps), room(y)
        view = lambda r, like: r[off:off + like.numel()].view(like.shape)  # noqa: B023, E731
        import paper_2607_05439_amd as dcp
        view(rx, x).copy_(x)
        dcp.dcp_checkpoint_pack(51, c, code(dt), view(rx, x), view(rc, codes), view(re, exps))
        dcp.dcp_checkpoint_unpack(51, c, code(dt), view(rc, codes), view(re, exps), view(ry, y))
        assert torch.equal(view(rc, codes), codes) and torch.equal(view(re, exps), exps) and torch.equal(view(ry, y), y)
        for r, like in ((rc, codes), (re, exps), (ry, y)):
            assert (r[:off] == 7).all() and (r[off + like.numel():] == 7).all()


def test_more_than_2_32_elements():
    import torch
    n = (1 << 25) + 5
    x = torch.zeros((n, 128), dtype=torch.bfloat16, device="cuda")
    x[-7:] = torch.randn((7, 128), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    codes, exps = pack(x)
    want = definition(x[-7:].float().cpu().numpy())
    assert np.array_equal(codes[-7:].cpu().numpy(), want[0]) and np.array_equal(exps[-7:].cpu().numpy(), want[1])
    assert not codes[:-7].any() and (exps[:-7] == 1).all()
    del x
    y = unpack(codes, exps, torch.bfloat16)
    assert np.array_equal(y[-7:].double().cpu().numpy(), want[2]) and not y[:-7].any()


def test_in_a_graph_and_on_another_stream():
    import torch
    import paper_2607_05439_amd as dcp
    x = torch.randn((1000, 128), device="cuda").to(torch.bfloat16)
    codes, exps = pack(x)
    want = unpack(codes, exps, torch.bfloat16)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c2, e2, y2 = torch.empty_like(codes), torch.empty_like(exps), torch.empty_like(want)
    torch.cuda.synchronize()
    dcp.dcp_checkpoint_pack(1000, 128, 1, x, c2, e2, side)
    dcp.dcp_checkpoint_unpack(1000, 128, 1, c2, e2, y2, side)
    side.synchronize()
    assert torch.equal(y2, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dcp.dcp_checkpoint_pack(1000, 128, 1, x, c2, e2)
        dcp.dcp_checkpoint_unpack(1000, 128, 1, c2, e2, y2)
    for k in range(3):
        x.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y2, unpack(*pack(x), torch.bfloat16))


def test_more_threads_than_one_launch_holds():
    """A row a block of one channel: 2^27 rows are 2^32 threads. The last rows are written too."""
    import torch
    n, tail = (1 << 27) + 77, 1000
    x = torch.zeros((n, 1), dtype=torch.bfloat16, device="cuda")
    x[-tail:, 0] = torch.arange(1, tail + 1, device="cuda").to(torch.bfloat16)
    codes, exps = pack(x)
    assert not codes[:-tail].any() and (exps[:-tail] == 1).all()
    want = pack(x[-tail:].clone())
    assert torch.equal(codes[-tail:], want[0]) and torch.equal(exps[-tail:], want[1])
    y = unpack(codes, exps, torch.bfloat16)
    assert not y[:-tail].any() and torch.equal(y[-tail:], unpack(*want, torch.bfloat16))


def test_the_error_at_the_ends_of_the_range():
    """Blocks whose largest magnitude is below 63.75 2^-126: at most 2^-127, all of a value below that. Over 127.5 2^121: 127 2^121
    is the most that is read back, at most 2^121 less. Between the two ends, up to them, half a step."""
    import torch
    g = torch.Generator().manual_seed(4)
    x = torch.rand((200, 32), generator=g, dtype=torch.float64) * 2 - 1
    top = torch.cat([torch.logspace(-149, -121, 100, base=2, dtype=torch.float64), torch.linspace(100, 127.999, 100, dtype=torch.float64) * 2.0 ** 121])
    x = (x * top[:, None]).float()
    x[:, 0] = top.float()
    y = unpack(*pack(x.cuda()), torch.float32).double().cpu()
    off, most = (x.double() - y).abs().amax(dim=1), x.double().abs().amax(dim=1)
    low, high = most < 63.75 * 2.0 ** -126, most > 127.5 * 2.0 ** 121
    assert low.any() and high.any() and not (low | high).all()
    assert (off[low] <= 2.0 ** -127).all() and (off[high] <= 2.0 ** 121).all()
    assert (off[~(low | high)] <= most[~(low | high)] / 127.5).all()
    assert (y[most < 2.0 ** -127] == 0).all()
    assert (off[high] > 2.0 ** 120).any() and (off[low] > most[low] / 127.5).any()
