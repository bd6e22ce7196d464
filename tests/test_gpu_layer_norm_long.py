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


@pytest.mark.parametrize("H,B,order", [(8, (1 << 20) + 100, "tokens"), (2, (1 << 25) + 77, "features")])
def test_more_tokens_than_a_launch_takes(darb, H, B, order):  # noqa: F811
    """2^20 workgroups and some: rows of tokens, or tiles of 32."""
    say(f"layer norm: {H} x {B} {order}")
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((B, H) if order == "tokens" else (H, B), device="cuda", generator=g)
    dy = torch.randn(x.shape, device="cuda", generator=g)
    if order == "tokens":
        x, dy = x.t(), dy.t()
    y, mean, rstd = darb.layer_norm(x)
    dx, dw, db = darb.layer_norm_grad(dy, x, mean, rstd)
    x, dy = x.double(), dy.double()
    m = x.mean(0)
    r = (x.var(0, unbiased=False) + 1e-5).rsqrt()
    # two or eight features: the mean's rounding over the spread is what y is off by most
    size = x.abs().mean(0)
    assert bool(((mean - m).abs() <= 2.0 ** -22 * size + 1e-30).all())
    slip = 2.0 ** -22 * size * r
    xh = (x - m) * r
    assert bool(((y - xh).abs() <= 1e-5 * (xh.abs() + 1) + slip * (1 + slip * xh.abs())).all())
    m, r = mean.double(), rstd.double()
    xh = (x - m) * r
    t = dy * xh
    scale = r * (dy.abs() + dy.abs().mean(0) + xh.abs() * t.abs().mean(0))
    assert bool(((dx - r * (dy - dy.mean(0) - xh * t.mean(0))).abs() <= 2e-5 * scale).all())
    assert bool(((dw - t.sum(1)).abs() <= 1e-5 * t.abs().sum(1)).all())
    assert bool(((db - dy.sum(1)).abs() <= 1e-5 * dy.abs().sum(1)).all())
