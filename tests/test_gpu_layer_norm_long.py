"""Layer norm where an axis takes more than one launch."""
import pytest

from tests._gpu import darb, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def test_gradient_sums_of_more_features_than_a_launch_takes(darb):  # noqa: F811
    """2^27 features and some: dw and db are dy xh and dy, for one token."""
    H = (1 << 27) + 33
    say(f"layer norm: weights' gradients of {H} features")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((H, 1), device="cuda", generator=g)
    dy = torch.randn((H, 1), device="cuda", generator=g)
    mean, rstd = torch.tensor([0.25], device="cuda"), torch.tensor([2.0], device="cuda")
    dx, dw, db = darb.layer_norm_grad(dy, x, mean, rstd, need_x=False)
    assert dx is None and torch.equal(db, dy[:, 0])
    want = (x[:, 0] - 0.25).mul_(2.0)                # two roundings and the product's: 2^-22 relative
    want.mul_(dy[:, 0])
    assert bool(((dw - want).abs_() <= want.abs_().mul_(2.0 ** -21)).all())
