"""Layer norm's gradients of feature-major columns too long for a workgroup's registers at a
useful width, whose features are cut: around the sizes of tiles and chunks.  Bounds as in
test_gpu_layer_norm."""
import numpy as np
import pytest

from tests._gpu import darb, torch  # noqa: F401
from tests._train import TYPES
from tests.test_gpu_layer_norm import run

pytestmark = pytest.mark.gpu

SHAPES = [(2500, 8), (2500, 9), (2561, 63), (2560, 64), (3000, 65), (4096, 71), (4100, 129), (9216, 64), (9216, 200),
          (5003, 703), (12289, 31), (16640, 130)]


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("H,B", SHAPES)
def test_layer_norm_split(darb, H, B, dtype, wdtype):  # noqa: F811
    rng = np.random.default_rng(H + B)
    x = rng.standard_normal((H, B)) * 1.5 + 0.3
    seen = []
    for order in ("features", "features+"):
        xd, dyd, w, (y, mean, rstd), (dx, dw, db) = run(darb, x, dtype, wdtype, order, np.random.default_rng(B),
                                                        f"norm split {H}x{B} {dtype} {order}")
        seen.append((dx, dw, db))
    assert all(torch.equal(p, q) for p, q in zip(*seen))
    for k in (0, 1):                         # in place, and a workspace whose contents do not matter
        a = [dyd.clone(), xd.clone()]
        ws = torch.full((8 * H * min(B, 512) + 1024,), 255, dtype=torch.uint8, device="cuda")
        got = darb.layer_norm_grad(a[0], a[1], mean, rstd, w, dx=a[k], workspace=ws)
        assert got[0] is a[k] and all(torch.equal(p, q) for p, q in zip(got, (dx, dw, db)))
    only = darb.layer_norm_grad(dyd, xd, mean, rstd, w, need_x=False)
    assert only[0] is None and torch.equal(only[1], dw) and torch.equal(only[2], db)
    only = darb.layer_norm_grad(dyd, xd, mean, rstd, w, need_params=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None


def test_layer_norm_split_keeps_what_lies_beside(darb):  # noqa: F811
    H, B = 4099, 77
    for dtype in TYPES.values():
        x = torch.randn(H, B, device="cuda").to(dtype)
        wide = torch.full((H + 2, B + 9), 3.0, device="cuda").to(dtype)
        dx = wide[1:H + 1, 4:B + 4]
        y, mean, rstd = darb.layer_norm(x)
        got = darb.layer_norm_grad(x, x, mean, rstd, dx=dx)[0]
        assert torch.equal(got, darb.layer_norm_grad(x, x, mean, rstd)[0])
        wide[1:H + 1, 4:B + 4] = 3.0
        assert bool((wide == 3.0).all())
