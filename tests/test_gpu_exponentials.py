"""The exponentials of the policy loss and of the recurrence's gates over the whole range of fp32,
relative to themselves."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb, say  # noqa: E402,F401
from _train import wide  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
#: an exponential: the hardware's power of two by a unit in the last place (2 U), the step that puts its
#: argument right by a rounding; what that step leaves out is below 10^-5 of a U
EXP = 3.01 * U


def arguments(low, high, n=200_000):
    r = np.random.default_rng(11)
    some = np.concatenate([r.uniform(low, high, n), r.normal(size=n // 4), [0.0, low, high, 1.0, -1.0]])
    return some.astype(np.float32).clip(low, high)


def test_ratios(darb):
    """With no lower bound, an advantage of -1 and a weight of 1 the gradient is the ratio."""
    d = arguments(-87.0, 88.5)
    one = torch.ones(len(d), device="cuda")
    got = darb.policy_loss(torch.from_numpy(d).cuda(), torch.zeros_like(one), -one, weight=one, clip=(1.5, 0.2))
    want = np.exp(d.astype(np.float64))
    off = np.abs(wide(got.grad_logprob) - want) / want
    say("ratios", off.max() / U)
    assert off.max() <= EXP, d[off.argmax()]


@pytest.mark.parametrize("tokens", [1, 7])
def test_gates(darb, tokens):
    """f and 1 - f, and their product in dgate, each relative to itself.

    f = 1 / (1 + e) with e = e^-z: a sum (U), a reciprocal by a unit (2 U), and e's own part of 1 + e: half
    of e's error where z >= 0, all of it below.  1 - f is e f where z >= 0, a product more, and 1 - f
    below, where f <= 1/2 is off by as much as 1/2 or more is; dgate multiplies the two."""
    z = arguments(-86.0, 86.0)
    z = z[:len(z) // tokens * tokens]
    Z = torch.from_numpy(z).cuda().view(-1, tokens)
    H, batch = Z.shape[0], tokens           # one step
    zeros, ones = torch.zeros_like(Z), torch.ones_like(Z)
    small = 1 / (1 + np.exp(np.abs(z.astype(np.float64))))
    up = z >= 0
    f, u = np.where(up, 1 - small, small), np.where(up, small, 1 - small)
    ef = 3 * U + np.where(up, EXP / 2, EXP)
    eu = np.where(up, EXP + ef + U, ef + U)
    h = darb.gated_recurrence(Z, zeros, batch=batch, h0=ones)[0]            # f
    h1 = darb.gated_recurrence(Z, ones, batch=batch)[0]                     # 1 - f
    dgate, dx, dh0 = darb.gated_recurrence_grad(ones, Z, zeros, h, batch=batch, h0=ones)
    for got, want, bound, name in ((h, f, ef, "f"), (h1, u, eu, "1 - f"), (dx, u, eu, "dx"), (dh0, f, ef, "dh0"),
                                   (dgate, f * u, ef + eu + U, "dgate")):
        off = np.abs(wide(got).ravel() - want) / want
        say(name, (off / U).max())
        assert (off <= bound * (1 + 1e-5)).all(), (name, z[(off / bound).argmax()])
    # beyond fp32's range the gate is shut or open
    far = torch.tensor([[-200.0, 200.0, -np.inf, np.inf]], device="cuda")
    got = darb.gated_recurrence(far, torch.zeros_like(far), batch=4, h0=torch.ones_like(far))[0]
    assert got.tolist() == [[0.0, 1.0, 0.0, 1.0]]
    nan = darb.gated_recurrence(far * np.nan, torch.zeros_like(far), batch=4, h0=torch.ones_like(far))[0]
    assert torch.isnan(nan).all()
