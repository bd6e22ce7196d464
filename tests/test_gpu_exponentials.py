"""The exponentials of the policy loss over the whole range of fp32, relative to themselves."""
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
