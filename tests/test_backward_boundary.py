"""LayerNorm and the backward passes on the host (CPU only): workspace queries, and every refusal with
its documented code before anything reaches the GPU."""
import ctypes

import pytest

import paper_2607_05439_amd as dcp

FAKE = 0x10000  # 256-byte aligned, never dereferenced on these paths
FAR = 1 << 45
BAD, UNSUPPORTED, WORKSPACE = dcp.DCP_ERR_INVALID_ARGUMENT, dcp.DCP_ERR_UNSUPPORTED, dcp.DCP_ERR_WORKSPACE
NAN = float("nan")


def layer_norm(n_rows=10, c=64, in_t=1, out_t=1, eps=1e-5, x=FAKE, gamma=None, beta=None, y=FAR):
    return dcp.lib().dcp_layer_norm(n_rows, c, in_t, out_t, eps, x, gamma, beta, y, None)


def layer_norm_back(n_rows=10, c=64, in_t=1, out_t=1, eps=1e-5, x=FAKE, gamma=None, dy=FAR, dx=2 * FAR, dgamma=3 * FAR,
                    dbeta=4 * FAR, ws=FAKE, ws_bytes=1 << 30):
    return dcp.lib().dcp_layer_norm_backward(n_rows, c, in_t, out_t, eps, x, gamma, dy, dx, dgamma, dbeta, ws, ws_bytes,
                                             None)


@pytest.mark.parametrize("call", [layer_norm, layer_norm_back])
@pytest.mark.parametrize("kw,code", [
    (dict(n_rows=-1), BAD), (dict(n_rows=(1 << 48) + 1), BAD), (dict(c=0), BAD), (dict(c=4097), UNSUPPORTED),
    (dict(in_t=2), BAD), (dict(out_t=-1), BAD), (dict(eps=-1.0), BAD), (dict(eps=NAN), BAD), (dict(eps=float("inf")), BAD),
    (dict(x=None), BAD), (dict(x=FAKE + 1), BAD), (dict(in_t=0, x=FAKE + 2), BAD), (dict(gamma=FAKE + 2), BAD),
])
def test_layer_norm_refusals(call, kw, code):
    assert call(**kw) == code and dcp.dcp_last_error()


def test_layer_norm_outputs_that_overlap():
    size = 10 * 64 * 2
    assert layer_norm(y=None) == BAD and layer_norm(y=FAR + 1) == BAD
    assert layer_norm(y=FAKE + size - 2) == BAD and layer_norm(y=FAKE - size + 2) == BAD
    assert layer_norm(y=FAKE, out_t=0) == BAD  # in place only in the same type
    for kw in (dict(dx=FAKE + 2), dict(dx=FAR - 2), dict(dx=FAKE, out_t=0, in_t=1, dy=FAKE + size - 4),
               dict(dx=FAR, out_t=0), dict(dy=None), dict(dy=FAR + 1), dict(dgamma=FAR + 2), dict(dbeta=1),
               dict(dx=None, dgamma=None, dbeta=None)):
        assert layer_norm_back(**kw) == BAD, kw


def test_layer_norm_workspace():
    size = dcp.dcp_layer_norm_backward_workspace_size
    assert size(0, 64) == 0 and 0 < size(1, 1) <= 256
    assert size(1 << 20, 128) == 1024 * 2 * 128 * 4 and size(1 << 40, 4096) == 1024 * 2 * 4096 * 4
    need = size(1000, 384)
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(ws_bytes=need - 1)):
        assert layer_norm_back(n_rows=1000, c=384, dx=5 * FAR, **kw) == WORKSPACE
    out = ctypes.c_size_t()
    L = dcp.lib()
    assert L.dcp_layer_norm_backward_workspace_size(10, 64, None) == BAD
    assert L.dcp_layer_norm_backward_workspace_size(-1, 64, ctypes.byref(out)) == BAD
    assert L.dcp_layer_norm_backward_workspace_size(10, 5000, ctypes.byref(out)) == UNSUPPORTED


def test_layer_norm_without_rows_needs_nothing():
    assert layer_norm(n_rows=0, x=None, y=None) == dcp.DCP_OK and dcp.dcp_last_error() == ""


FUSED = dict(n_tokens=24000, c_s=384, c_z=128, n_heads=16, head_dim=24, act_dtype=1, out_dtype=1, ln_eps=1e-5)
GENERAL = dict(n_tokens=601, c_s=128, c_z=128, n_heads=4, head_dim=32, act_dtype=0, out_dtype=0, ln_eps=1e-5)


def weights(**kw):
    w = {k: FAKE for k in ("w_q", "w_k", "w_v", "w_g", "w_b")}
    w.update(kw)
    return dcp.make_weights(**w)


def gradients(dtype=0, **kw):
    g = {k: FAR for k in ("dz_rows", "ds", "dw_q", "dw_k", "dw_v", "dw_g", "dw_b", "dln_gamma")}
    g.update(kw)
    return dcp.make_gradients(**g, dtype=dtype)


def backward(sh=None, w=None, s=FAKE, z=FAKE, q_row0=0, n_q=300, m=FAKE, l=FAKE, acc=FAKE, dout=FAKE, g=None, ws=FAKE,
             ws_bytes=1 << 45, base=GENERAL):
    sh = dcp.make_shape(**{**base, **(sh or {})})
    return dcp.lib().dcp_pair_bias_attention_backward(ctypes.byref(sh), ctypes.byref(w or weights()), s, z, None, q_row0,
                                                      n_q, m, l, acc, dout, ctypes.byref(g or gradients()), ws, ws_bytes,
                                                      None)


@pytest.mark.parametrize("base", [GENERAL, FUSED], ids=["general", "fused"])
@pytest.mark.parametrize("kw,code", [
    (dict(sh=dict(n_tokens=0)), BAD), (dict(sh=dict(c_z=0)), BAD), (dict(sh=dict(act_dtype=2)), BAD),
    (dict(sh=dict(out_dtype=2)), BAD), (dict(sh=dict(ln_eps=NAN)), BAD), (dict(sh=dict(c_z=300)), UNSUPPORTED),
    (dict(sh=dict(c_s=4200)), UNSUPPORTED), (dict(sh=dict(n_heads=20)), UNSUPPORTED),
    (dict(sh=dict(head_dim=65)), UNSUPPORTED), (dict(n_q=-1), BAD), (dict(q_row0=-1), BAD), (dict(n_q=24001), BAD),
    (dict(q_row0=23990, n_q=11), BAD), (dict(s=None), BAD), (dict(z=None), BAD), (dict(m=None), BAD), (dict(l=None), BAD),
    (dict(acc=None), BAD), (dict(dout=None), BAD), (dict(s=FAKE + 8), BAD), (dict(z=FAKE + 2), BAD), (dict(m=FAKE + 4), BAD),
    (dict(l=FAKE + 4), BAD), (dict(acc=FAKE + 8), BAD), (dict(dout=FAKE + 4), BAD), (dict(w=weights(w_g=None)), BAD),
    (dict(w=weights(w_b=None)), BAD), (dict(g=gradients(dtype=3)), BAD), (dict(g=gradients(ds=FAR + 4)), BAD),
    (dict(g=gradients(dz_rows=FAR + 2)), BAD), (dict(g=gradients(dln_gamma=FAR + 8)), BAD),
    (dict(g=dcp.make_gradients()), BAD), (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 128), WORKSPACE),
    (dict(ws_bytes=1000), WORKSPACE),
])
def test_attention_backward_refusals(base, kw, code):
    assert backward(base=base, **kw) == code and dcp.dcp_last_error()


def test_attention_backward_missing_structs():
    L, sh, w, g = dcp.lib(), dcp.make_shape(**GENERAL), weights(), gradients()
    tail = (FAKE, FAKE, None, 0, 10, FAKE, FAKE, FAKE, FAKE)
    assert L.dcp_pair_bias_attention_backward(None, ctypes.byref(w), *tail, ctypes.byref(g), FAKE, 1 << 40, None) == BAD
    assert L.dcp_pair_bias_attention_backward(ctypes.byref(sh), None, *tail, ctypes.byref(g), FAKE, 1 << 40, None) == BAD
    assert L.dcp_pair_bias_attention_backward(ctypes.byref(sh), ctypes.byref(w), *tail, None, FAKE, 1 << 40, None) == BAD


def test_fused_weights_are_aligned():
    for name in ("w_q", "w_k", "w_v", "w_g", "w_b", "ln_gamma"):
        assert backward(base=FUSED, w=weights(**{name: FAKE + 4})) == BAD


def test_attention_backward_workspace():
    def size(base, n_q, **kw):
        return dcp.dcp_pair_bias_attention_backward_workspace_size(dcp.make_shape(**{**base, **kw}), n_q)

    for base in (GENERAL, FUSED):
        assert size(base, 0) == 0
        n = base["n_tokens"]
        for n_q in (1, 16, 300, n):
            need = size(base, n_q)
            assert need > 0 and backward(base=base, n_q=n_q, ws_bytes=need - 1) == WORKSPACE
    # the room for probabilities is bounded, whatever the stripe: not n_q x N x H
    assert size(FUSED, 24000) < 4 << 30
    sh, out = dcp.make_shape(**GENERAL), ctypes.c_size_t()
    L = dcp.lib()
    assert L.dcp_pair_bias_attention_backward_workspace_size(ctypes.byref(sh), 10, None) == BAD
    assert L.dcp_pair_bias_attention_backward_workspace_size(None, 10, ctypes.byref(out)) == BAD
    assert L.dcp_pair_bias_attention_backward_workspace_size(ctypes.byref(sh), 602, ctypes.byref(out)) == BAD


# ----------------------------------------------------------------------------- gradients that overlap
PLACES = {"s": 1, "z": 2, "m": 3, "l": 4, "acc": 5, "dout": 6, "mask": 7, "w_q": 8, "w_k": 9, "w_v": 10, "w_g": 11, "w_b": 12,
          "ln_gamma": 13, "ws": 14, "dz_rows": 15, "ds": 16, "dw_q": 17, "dw_k": 18, "dw_v": 19, "dw_g": 20, "dw_b": 21,
          "dln_gamma": 22}
GRADS = ("dz_rows", "ds", "dw_q", "dw_k", "dw_v", "dw_g", "dw_b", "dln_gamma")
N_Q = 300


def sizes(base, grad):
    """Bytes of each tensor of a call of N_Q rows with gradients of `grad` bytes an element."""
    n, c_s, c_z, h, hd = base["n_tokens"], base["c_s"], base["c_z"], base["n_heads"], base["n_heads"] * base["head_dim"]
    act, out = (2 if base["act_dtype"] else 4), (2 if base["out_dtype"] else 4)
    b = {"s": n * c_s * act, "z": N_Q * n * c_z * act, "m": h * N_Q * 4, "l": h * N_Q * 4, "acc": N_Q * hd * 4,
         "dout": N_Q * hd * out, "mask": n, "w_b": h * c_z * 4, "ln_gamma": c_z * 4,
         "ws": dcp.dcp_pair_bias_attention_backward_workspace_size(dcp.make_shape(**base), N_Q),
         "dz_rows": N_Q * n * c_z * act, "ds": n * c_s * grad, "dw_b": h * c_z * grad, "dln_gamma": c_z * grad}
    b.update({k: hd * c_s * 4 for k in ("w_q", "w_k", "w_v", "w_g")})
    b.update({k: hd * c_s * grad for k in ("dw_q", "dw_k", "dw_v", "dw_g")})
    return b


def placed(base, grad_dtype, at):
    sh = dcp.make_shape(**base)
    w = dcp.make_weights(**{k: at[k] for k in ("w_q", "w_k", "w_v", "w_g", "w_b", "ln_gamma")})
    g = dcp.make_gradients(**{k: at[k] for k in GRADS}, dtype=grad_dtype)
    return dcp.lib().dcp_pair_bias_attention_backward(
        ctypes.byref(sh), ctypes.byref(w), at["s"], at["z"], at["mask"], 0, N_Q, at["m"], at["l"], at["acc"], at["dout"],
        ctypes.byref(g), at["ws"], 1 << 50, None)


@pytest.mark.parametrize("base", [GENERAL, FUSED], ids=["general", "fused"])
@pytest.mark.parametrize("grad_dtype", [0, 1])
def test_gradients_that_overlap_are_refused(base, grad_dtype):
    """Each gradient and the workspace at the start of every other tensor and at its last piece; a range
    that only touches another is none, so that the refusal names a third one, put on s."""
    apart = {k: v << 40 for k, v in PLACES.items()}
    size = sizes(base, 2 if grad_dtype else 4)
    for a in GRADS + ("ws",):
        for b in (k for k in PLACES if k != a):
            last = (size[b] - 1) // 256 * 256
            for at in (0, last):
                assert placed(base, grad_dtype, {**apart, a: apart[b] + at}) == BAD, (a, b)
                assert "overlap" in dcp.dcp_last_error(), (a, b, dcp.dcp_last_error())
            third = next(k for k in GRADS if k not in (a, b))
            assert placed(base, grad_dtype, {**apart, a: apart[b] + last + 256, third: apart["s"]}) == BAD
            assert third in dcp.dcp_last_error().replace(",", " ").split(), (a, b, third, dcp.dcp_last_error())


@pytest.mark.parametrize("in_t,out_t", [(0, 0), (1, 1), (0, 1), (1, 0)])
def test_layer_norm_s_sums_and_workspace_lie_apart(in_t, out_t):
    """dln_gamma, dln_beta and the workspace on each other and on the rows' tensors, and rows written onto
    weights: refused."""
    rows, c = 1000, 64
    at = {k: (i + 1) << 40 for i, k in enumerate(("x", "dy", "dx", "gamma", "dgamma", "dbeta", "ws"))}
    size = {"x": rows * c * (2 if in_t else 4), "dy": rows * c * (2 if out_t else 4), "dx": rows * c * (2 if in_t else 4),
            "gamma": c * 4, "dgamma": c * 4, "dbeta": c * 4, "ws": dcp.dcp_layer_norm_backward_workspace_size(rows, c)}
    for a, b in [(a, b) for a in ("dgamma", "dbeta", "ws") for b in at if b != a] + [("dx", "gamma")]:
        for off in (0, (size[b] - 1) // 256 * 256):
            assert layer_norm_back(rows, c, in_t, out_t, **{**at, a: at[b] + off}) == BAD, (a, b)
            assert "overlap" in dcp.dcp_last_error(), (a, b)
    for b in ("gamma", "beta"):
        assert layer_norm(rows, c, in_t, out_t, x=FAKE, y=FAR, **{b: FAR + 512}) == BAD and "overlap" in dcp.dcp_last_error()
