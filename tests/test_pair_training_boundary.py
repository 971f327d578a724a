"""The pair transition's backward pass, 8-bit checkpoints and relative positions on the host (CPU only):
workspace queries, and every refusal with its documented code before anything reaches the GPU."""
import ctypes

import pytest

import paper_2607_05439_amd as dcp

FAKE = 0x10000  # 256-byte aligned, never dereferenced on these paths
FAR = 1 << 45
BAD, UNSUPPORTED, WORKSPACE = dcp.DCP_ERR_INVALID_ARGUMENT, dcp.DCP_ERR_UNSUPPORTED, dcp.DCP_ERR_WORKSPACE
NAN = float("nan")
NAMES = ("dz", "dw1", "dw2", "dw3", "dln_gamma", "dln_beta")


def gradients(dtype=0, **kw):
    g = {k: FAR + (i << 40) for i, k in enumerate(NAMES)}
    g.update(kw)
    return dcp.make_transition_gradients(**g, dtype=dtype)


def backward(n=1000, c=128, hidden=512, t=1, eps=1e-5, w1=FAKE, w2=2 * FAKE * 16, w3=3 * FAKE * 16, gamma=None, beta=None,
             z=1 << 36, exps=None, dout=1 << 37, g=None, ws=1 << 38, ws_bytes=1 << 34):
    g = gradients() if g is None else g
    return dcp.lib().dcp_pair_transition_backward(n, c, hidden, t, eps, w1, w2, w3, gamma, beta, z, exps, dout,
                                                  ctypes.byref(g) if g else None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), BAD), (dict(n=(1 << 34) + 1), BAD), (dict(c=0), BAD), (dict(hidden=0), BAD), (dict(t=2), BAD),
    (dict(c=64), UNSUPPORTED), (dict(hidden=256), UNSUPPORTED), (dict(t=0, c=257), UNSUPPORTED),
    (dict(t=0, hidden=1025), UNSUPPORTED), (dict(eps=-1.0), BAD), (dict(eps=NAN), BAD), (dict(w1=None), BAD),
    (dict(w2=None), BAD), (dict(w3=None), BAD), (dict(z=None), BAD), (dict(dout=None), BAD), (dict(g=False), BAD),
    (dict(g=gradients(dtype=2)), BAD), (dict(g=gradients(**{k: None for k in NAMES})), BAD),
    (dict(z=(1 << 36) + 8), BAD), (dict(dout=(1 << 37) + 2), BAD), (dict(g=gradients(dz=FAR + 4)), BAD),
    (dict(t=0, z=(1 << 36) + 2), BAD), (dict(t=0, dout=(1 << 37) + 2), BAD), (dict(exps=(1 << 35) + 2), BAD),
    (dict(w1=FAKE + 2), BAD), (dict(gamma=FAKE + 1), BAD), (dict(beta=FAKE + 3), BAD), (dict(g=gradients(dw1=FAR * 2 + 2)), BAD),
    (dict(g=gradients(dtype=1, dln_beta=FAR * 2 + 1)), BAD), (dict(ws=None), WORKSPACE), (dict(ws=(1 << 38) + 16), WORKSPACE),
    (dict(ws_bytes=100), WORKSPACE),
])
def test_transition_backward_refusals(kw, code):
    assert backward(**kw) == code and dcp.dcp_last_error()


def test_transition_backward_overlaps():
    rows, w = 1000 * 128 * 2, 128 * 512 * 4
    for kw in (dict(g=gradients(dz=1 << 36)), dict(g=gradients(dz=(1 << 37) + 16)), dict(g=gradients(dz=(1 << 37) - 16)),
               dict(g=gradients(dw1=1 << 36)), dict(g=gradients(dw1=(1 << 36) + rows - 4)), dict(g=gradients(dw1=FAKE)),
               dict(g=gradients(dw2=FAKE + w - 4)), dict(g=gradients(dw3=1 << 37)), dict(g=gradients(dln_gamma=1 << 38)),
               dict(g=gradients(dw1=FAR, dz=FAR)), dict(g=gradients(dw1=FAR * 2, dw2=FAR * 2 + w - 4)),
               dict(g=gradients(dln_beta=1 << 35), gamma=1 << 35), dict(ws=1 << 36), dict(ws=1 << 37),
               dict(exps=1 << 38), dict(g=gradients(dz=1 << 35), exps=(1 << 35) + 16)):
        assert backward(**kw) == BAD and "overlap" in dcp.dcp_last_error(), kw


def test_transition_backward_workspace():
    size = dcp.dcp_pair_transition_backward_workspace_size
    need = size(1000, 128, 512, 1)
    assert need > 0 and backward(ws_bytes=need - 1) == WORKSPACE
    # bounded: shares' sums and, in bf16, 512 B for each of at most 2^20 pairs
    assert size(1 << 34, 128, 512, 1) == size(1 << 20, 128, 512, 1) < 640e6 and size(1 << 34, 32, 128, 0) < 256e6
    out, lib = ctypes.c_size_t(), dcp.lib()
    query = lib.dcp_pair_transition_backward_workspace_size
    assert query(10, 128, 512, 1, None) == BAD and query(-1, 128, 512, 1, ctypes.byref(out)) == BAD
    assert query(10, 64, 512, 1, ctypes.byref(out)) == UNSUPPORTED and query(10, 0, 512, 0, ctypes.byref(out)) == BAD


def test_only_dz_of_no_pairs_needs_nothing():
    assert backward(n=0, z=None, dout=None, ws=None, g=gradients(**{k: None for k in NAMES[1:]})) == dcp.DCP_OK


def pack(n=10, c=128, t=1, x=FAR, codes=2 * FAR, exps=3 * FAR):
    return dcp.lib().dcp_checkpoint_pack(n, c, t, x, codes, exps, None)


def unpack(n=10, c=128, t=1, x=FAR, codes=2 * FAR, exps=3 * FAR):
    return dcp.lib().dcp_checkpoint_unpack(n, c, t, codes, exps, x, None)


@pytest.mark.parametrize("call", [pack, unpack])
@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), BAD), (dict(n=(1 << 36) + 1), BAD), (dict(c=0), BAD), (dict(c=65537), UNSUPPORTED), (dict(t=2), BAD),
    (dict(x=None), BAD), (dict(codes=None), BAD), (dict(exps=None), BAD), (dict(x=FAR + 1), BAD), (dict(t=0, x=FAR + 2), BAD),
    (dict(codes=FAR), BAD), (dict(codes=FAR + 10 * 256 - 1), BAD), (dict(codes=FAR - 1), BAD), (dict(exps=FAR + 100), BAD),
])
def test_checkpoint_refusals(call, kw, code):
    assert call(**kw) == code and dcp.dcp_last_error()


def test_checkpoint_of_no_rows_needs_nothing_and_codes_lie_apart():
    assert pack(n=0, x=None, codes=None, exps=None) == dcp.DCP_OK and unpack(n=0, x=None, codes=None, exps=None) == dcp.DCP_OK
    assert pack(codes=3 * FAR - 1) == BAD and pack(exps=2 * FAR + 5) == BAD


def fields(*radii, position=FAKE, group=FAKE):
    return dcp.make_relative_fields([(position, group, r) for r in radii])


def encode(n=100, row0=0, rows=100, c=128, t=1, f=None, count=None, table=2 * FAR, z_in=3 * FAR, z_out=4 * FAR):
    f = fields(32, 0) if f is None else f
    return dcp.lib().dcp_relative_position(n, row0, rows, c, t, len(f) if count is None else count, f or None, table, z_in,
                                           z_out, None)


def encode_back(n=100, row0=0, rows=100, c=128, t=1, f=None, count=None, dz=3 * FAR, dtable=2 * FAR, ws=5 * FAR, ws_bytes=1 << 40):
    f = fields(32, 0) if f is None else f
    return dcp.lib().dcp_relative_position_backward(n, row0, rows, c, t, len(f) if count is None else count, f or None, dz,
                                                    dtable, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [encode, encode_back])
@pytest.mark.parametrize("kw,code", [
    (dict(n=0), BAD), (dict(n=1 << 31, rows=1), BAD), (dict(rows=-1), BAD), (dict(row0=-1), BAD), (dict(row0=1), BAD),
    (dict(rows=101), BAD), (dict(row0=(1 << 63) - 1, rows=1), BAD), (dict(n=1 << 20, rows=1 << 20), BAD), (dict(c=0), BAD),
    (dict(c=1025), UNSUPPORTED), (dict(t=2), BAD), (dict(count=0), BAD), (dict(f=fields(1, 1, 1, 1, 1)), UNSUPPORTED),
    (dict(f=[], count=1), BAD), (dict(f=fields(-1)), BAD), (dict(f=fields(128)), UNSUPPORTED),
    (dict(f=fields(1, position=None)), BAD), (dict(f=fields(1, position=FAKE + 2)), BAD), (dict(f=fields(1, group=FAKE + 1)), BAD),
])
def test_relative_refusals(call, kw, code):
    assert call(**kw) == code and dcp.dcp_last_error()


def test_relative_tensors():
    size = 100 * 100 * 128 * 2
    for kw in (dict(table=None), dict(table=2 * FAR + 2), dict(z_in=3 * FAR + 1), dict(z_out=None), dict(z_out=4 * FAR + 1),
               dict(z_out=3 * FAR + 2), dict(z_out=3 * FAR - size + 2), dict(z_out=2 * FAR), dict(table=4 * FAR + size - 4),
               dict(z_out=FAKE), dict(f=fields(3, position=4 * FAR)), dict(f=fields(3, group=4 * FAR + size - 4))):
        assert encode(**kw) == BAD, kw
    for kw in (dict(dz=None), dict(dtable=None), dict(dtable=2 * FAR + 2), dict(dz=3 * FAR + 1), dict(dtable=3 * FAR),
               dict(dtable=5 * FAR), dict(ws=3 * FAR), dict(dtable=FAKE), dict(f=fields(3, group=5 * FAR))):
        assert encode_back(**kw) == BAD, kw
    need = dcp.dcp_relative_position_backward_workspace_size(100, 100, 128, fields(32, 0))
    for kw in (dict(ws=None), dict(ws=5 * FAR + 16), dict(ws_bytes=need - 1)):
        assert encode_back(**kw) == WORKSPACE, kw
    out, lib = ctypes.c_size_t(), dcp.lib()
    query = lib.dcp_relative_position_backward_workspace_size
    assert query(100, 100, 128, 2, fields(32, 0), None) == BAD and query(100, 101, 128, 2, fields(32, 0), ctypes.byref(out)) == BAD
    assert query(100, 0, 128, 2, fields(32, 0), ctypes.byref(out)) == dcp.DCP_OK and out.value == 0


def test_encoding_of_no_rows_needs_nothing():
    assert encode(rows=0, table=None, z_in=None, z_out=None, f=fields(1, position=None)) == dcp.DCP_OK
