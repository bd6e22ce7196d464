"""Layer norm's gradients where several tokens share a workgroup, the last round of some teams
empty, and around the longest rows that registers hold.  Bounds as in test_gpu_layer_norm."""
import numpy as np
import pytest

from tests._gpu import darb, torch  # noqa: F401
from tests.test_gpu_layer_norm import run

pytestmark = pytest.mark.gpu

#: two, three and four teams, with and without an even end; rows of 1024 threads, and one longer
SHAPES = [(1500, 1025), (1100, 1536), (1500, 2049), (2048, 2051), (1030, 513), (3900, 1027), (8200, 5), (9216, 259),
          (12288, 3), (12290, 4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,B", SHAPES)
def test_layer_norm_teams(darb, H, B, dtype):  # noqa: F811
    rng = np.random.default_rng(H + B)
    x = rng.standard_normal((H, B)) * 1.5 + 0.3
    xd, dyd, w, (y, mean, rstd), (dx, dw, db) = run(darb, x, dtype, "f32", "tokens", rng, f"norm teams {H}x{B} {dtype}")
    for k in (0, 1):                         # in place, the same bits
        a = [dyd.clone(memory_format=torch.preserve_format), xd.clone(memory_format=torch.preserve_format)]
        got = darb.layer_norm_grad(a[0], a[1], mean, rstd, w, dx=a[k])
        assert got[0] is a[k] and all(torch.equal(p, q) for p, q in zip(got, (dx, dw, db)))
    only = darb.layer_norm_grad(dyd, xd, mean, rstd, w, need_x=False)
    assert only[0] is None and torch.equal(only[1], dw) and torch.equal(only[2], db)
