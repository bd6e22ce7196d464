"""Alternatives where many logits are equal, where few are left, and of rows of several parts;
the gradient written over the logits where a row of tokens ends inside a vector.

Values are compared as in test_gpu_logprobs (its bounds); indexes are equal."""
import numpy as np
import pytest

from tests._gpu import darb, torch  # noqa: F401
from tests.test_gpu_logprobs import run

pytestmark = pytest.mark.gpu

#: one workgroup a row (256, 512 and 1024 threads), several parts a row, feature-major
SHAPES = [("tokens", 1500, 3), ("tokens", 9001, 40), ("tokens", 20480, 300), ("tokens", 300001, 1),
          ("features", 3001, 5), ("features", 40000, 2), ("features", 1024, 130)]


def equal_but(V, B, kind):
    rng = np.random.default_rng(V + B)
    z = np.full((V, B), 1.0)
    if kind == "spikes":                     # fewer than asked for above the others, at the end too
        z[V - 1] = 2.0
        z[rng.integers(V, size=B), np.arange(B)] = 3.0
    elif kind == "left":                     # three classes left
        z[:] = -np.inf
        for b in range(B):
            z[rng.choice(V, 3, replace=False), b] = rng.standard_normal(3)
    elif kind == "halves":                   # the greatest value half of the time
        z[rng.random((V, B)) < 0.5] = 0.0
    elif kind == "special":                  # more NaN than asked for, and infinities between
        z[rng.random((V, B)) < 0.3] = np.nan
        z[rng.random((V, B)) < 0.3] = np.inf
    return z, rng.integers(0, V, B)


@pytest.mark.parametrize("kind", ["equal", "spikes", "left", "halves", "special"])
@pytest.mark.parametrize("order,V,B", SHAPES)
def test_equal_logits(darb, order, V, B, kind):  # noqa: F811
    z, t = equal_but(V, B, kind)
    for top, dtype in ((5, "f32"), (64, "f16")):
        run(darb, z, t, top, dtype, order, f"{kind} {V}x{B} {dtype} {order} top {top}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinity_beside_numbers(darb, dtype):  # noqa: F811
    # a thread that read an infinity keeps the order of its numbers
    rng = np.random.default_rng(11)
    V, B = 4096, 6
    z = np.round(rng.standard_normal((V, B)) * 8)
    for b in range(B):
        z[rng.choice(V, 3 + b, replace=False), b] = np.inf
    for order in ("tokens", "features"):
        run(darb, z, rng.integers(0, V, B), 8, dtype, order, f"infinities {dtype} {order}")


def test_many_long_rows(darb):  # noqa: F811
    # rows so long that they have several parts although there are enough rows for the card
    V, B, k = 64 * 8192 + 5001, 520, 7
    z = torch.zeros(B, V, dtype=torch.bfloat16, device="cuda")
    at = torch.stack([torch.randperm(V // 9, device="cuda")[:k] * 9 for _ in range(B)])
    z.scatter_(1, at, (torch.arange(k, 0, -1, device="cuda", dtype=torch.bfloat16) + 4).expand(B, k).contiguous())
    r = darb.token_logprobs(z.t(), at[:, 0].contiguous(), top=k + 2)
    high = np.arange(k, 0, -1) + 4.0
    lse = np.log(np.exp(high).sum() + (V - k))
    assert torch.equal(r.top_index[:, :k], at)
    for b in range(0, B, 37):                # then zeros, the lowest classes that hold one
        rest = np.setdiff1d(np.arange(k + 2), at[b].cpu().numpy())[:2]
        assert r.top_index[b, k:].tolist() == rest.tolist()
    want = np.concatenate([high, [0.0, 0.0]]) - lse
    assert np.abs(r.top_logprob.double().cpu().numpy() - want).max() < 1e-5 + 13 * 2.0 ** -23
    assert np.abs(r.logprob.double().cpu().numpy() - want[0]).max() < 1e-5 + 13 * 2.0 ** -23


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V,B", [(37, 2), (37, 3), (300, 7), (300, 9), (65, 701), (1000, 1021)])
def test_gradient_over_the_logits(darb, V, B, dtype):  # noqa: F811
    rng = np.random.default_rng(V * 7 + B)
    types = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
    wide = torch.from_numpy(rng.standard_normal((V, B + 3))).cuda().to(types[dtype])
    z = wide[:, 1:B + 1]
    t = torch.from_numpy(rng.integers(-1, V, B)).cuda()
    r = darb.token_logprobs(z, t)
    g = torch.from_numpy(rng.standard_normal((2, B)).astype(np.float32)).cuda()
    apart = darb.token_logprobs_grad(z, t, r.lse, g[0], r.entropy, g[1])
    edge = wide[:, [0, B + 1, B + 2]].clone()
    over = darb.token_logprobs_grad(z, t, r.lse, g[0], r.entropy, g[1], out=z)
    assert over.data_ptr() == z.data_ptr()
    assert torch.equal(over, apart)
    assert torch.equal(wide[:, [0, B + 1, B + 2]], edge)
