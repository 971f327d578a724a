"""The attention's backward pass where inputs are at the edge of what it accepts: no epsilon, values that are
not finite (GPU). The tolerances are those of test_gpu_attention_backward.py."""
import pytest

from test_gpu_attention_backward import BF16, F32, NAMES, Call, check, make, reference

pytestmark = pytest.mark.gpu
WIDTHS = pytest.mark.parametrize("widths,tol", [(F32, 2e-5), (BF16, 1e-2)], ids=["f32", "bf16"])


@WIDTHS
@pytest.mark.parametrize("row0,rows", [(0, 1), (3, 17), (0, 33)])
def test_without_epsilon(widths, tol, row0, rows):
    """ln_eps = 0 divides by the variance alone, which pairs of the stripe have: the tiles' rows past the
    stripe's last are no pairs. (The reference's 1e-5 of variances of size 1 moves the logits by 5e-6.)"""
    x = make(37, row0, rows, **widths, masked=2, seed=60)
    call = Call(x)
    call.shape.ln_eps = 0.0
    want = reference(x)
    check(call(), want, tol + 5e-6)


def other_heads(got, want, dims, tol, names=("w_q", "w_k", "w_v", "w_g")):
    """The rows of the projections' gradients that belong to heads 1 and up."""
    d = dims[7]
    check({k: got[k][d:] for k in names}, {k: want[k][d:] for k in names}, tol)


@WIDTHS
@pytest.mark.parametrize("scale", [2.0 ** -10, 2.0 ** -30])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_value_of_dout_that_is_not_finite_leaves_the_other_heads(widths, tol, scale, bad):
    """It belongs to head 0: the rows of dW_q, dW_k, dW_v and dW_g of the other heads hold what the
    finite values give, and dz of the other rows too."""
    x = make(60, 4, 40, **widths, masked=3, seed=61, dout_scale=scale)
    x["dout"][7, 3] = 0
    want = reference(x)
    x["dout"][7, 3] = bad
    got = Call(x)()
    other_heads(got, want, x["dims"], tol)
    rows = [r for r in range(40) if r != 7]
    check({"dz": got["dz"][rows]}, {"dz": want["dz"][rows]}, tol)


@WIDTHS
@pytest.mark.parametrize("factor", [1.0, 2.0 ** -24])
def test_a_query_that_is_not_finite(widths, tol, factor):
    """A padding token as a query row: masked as a key, its single track infinite. dz of the other rows is the
    definition's, with q of any size."""
    x = make(60, 0, 40, **widths, seed=62)
    import torch
    x["mask"] = torch.ones(60, dtype=torch.uint8)
    x["mask"][7] = 0
    x["w_q"], x["w_k"] = x["w_q"] * factor, x["w_k"] / factor
    want = reference(x)
    x["s"][7, 0] = float("inf")  # (all of a row: sums of both signs are NaN, not infinite)
    got = Call(x)()
    rows = [r for r in range(40) if r != 7]
    check({"dz": got["dz"][rows]}, {"dz": want["dz"][rows]}, tol)
