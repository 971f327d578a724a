"""LayerNorm over row counts on both sides of those where the backward takes more workgroups, and where a
workgroup's share of them is uneven (GPU). Tolerances and reference as in test_gpu_layer_norm.py."""
import pytest

from test_gpu_layer_norm import backward, forward, make, off, reference

pytestmark = pytest.mark.gpu


# rounds of rows: 512, 513, 1200, 1280, 1281; 1282 and 2600 of 128 channels; 1300 rows of a whole workgroup
@pytest.mark.parametrize("rows,c", [(2048, 384), (2049, 384), (4800, 384), (5120, 384), (5121, 384), (20500, 128),
                                    (41600, 128), (1300, 2000), (100001, 8)])
@pytest.mark.parametrize("x_type,y_type", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_matches_the_definition(rows, c, x_type, y_type):
    x, dy, gamma, beta = make(rows, c, x_type, y_type, seed=rows)
    want = reference(x, dy, gamma, beta)
    xd, dyd, gd, bd = (t.cuda() for t in (x, dy, gamma, beta))
    got = backward(xd, gd, dyd)
    errs = [off(forward(xd, gd, bd, y_type), want[0], y_type), off(got[0], want[1], x_type), off(got[1], want[2], "f32"),
            off(got[2], want[3], "f32")]
    print(rows, c, x_type, y_type, ["%.2e" % e for e in errs], flush=True)
    assert max(errs) <= 1e-5
