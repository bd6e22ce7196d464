"""The policy loss where a ratio leaves the range of fp32."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb, say  # noqa: E402,F401
from _train import check, wide  # noqa: E402
from test_gpu_losses import f32, on, policy, tokens  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("n", [1, 700, 9001])
@pytest.mark.parametrize("far", [88.0, 89.0, 100.0, 3e38])
def test_advantages_of_0(darb, n, far):
    """A ratio of any finite size times an advantage of 0 is 0, in the loss and in its gradient."""
    r, lp, old, A, w, ref, ent = tokens(n, n)
    w = f32(w + 1e-3 / n)
    A[::5] = 0
    A[::10] = -0.0
    old[::5] = f32(lp[::5] - far)
    plain = np.where(A == 0, lp, old)       # a ratio of 1 in their place
    want = policy(lp, plain, A, w, 0.2, 0.2, None, 0.0, None, 0.0)
    got = darb.policy_loss(on(lp), on(old), on(A), weight=on(w))
    check(wide(got.loss), want[0], want[5] + U * abs(want[0]) + 1e-300, "loss")
    check(wide(got.clipped), want[2], U * abs(want[2]), "clipped")
    check(wide(got.grad_logprob), want[3], want[7], "dlp")
    assert not got.grad_logprob[::5].any()


def test_what_is_not_finite_stays(darb):
    """An advantage of 0 does not hide a NaN, nor an infinite ratio (0 times which is none)."""
    for lp, old in ((math.nan, -1.0), (-1.0, math.nan), (-1.0, -math.inf), (-math.inf, -math.inf)):
        got = darb.policy_loss(on([lp, -1.0]), on([old, -1.0]), on([0.0, 1.0]))
        assert torch.isnan(got.loss) and torch.isnan(got.grad_logprob[0]) and torch.isfinite(got.grad_logprob[1]), (lp, old)
    # a token of probability 0 now has a ratio of 0
    got = darb.policy_loss(on([-math.inf, -1.0]), on([-1.0, -1.0]), on([0.0, 1.0]))
    assert float(got.loss) == -0.5 and got.grad_logprob.tolist() == [0.0, -0.5]


@pytest.mark.parametrize("n", [1, 700, 9001])
@pytest.mark.parametrize("far", [89.0, 1e4, math.inf, -math.inf, math.nan])
def test_kl_that_is_only_reported(darb, n, far):
    """With a coefficient of 0 the reference changes kl, neither the loss nor its gradient."""
    r, lp, old, A, w, ref, ent = tokens(n, n)
    w = f32(w + 1e-3 / n)
    ref[::7] = far
    without = darb.policy_loss(on(lp), on(old), on(A), weight=on(w))
    got = darb.policy_loss(on(lp), on(old), on(A), weight=on(w), ref_logprob=on(ref), kl_coef=0.0)
    assert torch.isfinite(got.loss) and torch.equal(got.loss, without.loss) and torch.equal(got.clipped, without.clipped)
    assert torch.equal(got.grad_logprob, without.grad_logprob)
    # a reference of +inf has no value: e^q - 1 - q is infinity less infinity in the definition too
    assert torch.isnan(got.kl) if math.isnan(far) or far == math.inf else float(got.kl) == math.inf
