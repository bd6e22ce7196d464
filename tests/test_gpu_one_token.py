"""One token: each operand may be a contiguous vector or a column of a wider matrix, whatever the
others are.  Bounds as in the tests of the calls themselves."""
import itertools

import numpy as np
import pytest

from tests._gpu import darb, say, torch  # noqa: F401
from tests._train import TYPES, check, rounding, wide

pytestmark = pytest.mark.gpu
EPS = 1e-5


def column(a, strided, dtype):
    """[F, 1] with feature stride 1, or 5 inside a buffer of sevens."""
    if not strided:
        return torch.from_numpy(a).to(TYPES[dtype]).cuda()
    m = torch.full((a.shape[0], 5), 7.0, dtype=TYPES[dtype], device="cuda")
    m[:, 2:3] = torch.from_numpy(a).to(TYPES[dtype]).cuda()
    return m[:, 2:3]


def untouched(t):
    if t.stride(0) == 1:
        return True
    whole = t.as_strided((t.shape[0], 5), (5, 1), t.storage_offset() - 2)
    return bool((whole[:, [0, 1, 3, 4]] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H", [1, 3, 133, 5000])
def test_layer_norm_of_one_token(darb, H, dtype):  # noqa: F811
    rng = np.random.default_rng(H)
    a, b = rng.standard_normal((H, 1)), rng.standard_normal((H, 1))
    for sx, sy, sd in itertools.product([False, True], repeat=3):
        say(f"one token: norm {H} {dtype} strided x {sx} y, dx {sy} dy {sd}")
        x, dy = column(a, sx, dtype), column(b, sd, dtype)
        y, dx = column(np.zeros((H, 1)), sy, dtype), column(np.zeros((H, 1)), sy, dtype)
        x64, g = wide(x), wide(dy)
        out, mean, rstd = darb.layer_norm(x, y=y, eps=EPS)
        m, r = x64.mean(), 1 / np.sqrt(x64.var() + EPS)
        xh = (x64 - m) * r
        slip = 2.0 ** -22 * np.abs(x64).mean() * r
        assert out is y and untouched(y) and untouched(x)
        check(wide(y), xh, 1e-5 * (np.abs(xh) + 1) + slip * (1 + slip * np.abs(xh)) + rounding(xh, dtype), "y")
        m, r = wide(mean)[0], wide(rstd)[0]
        xh = (x64 - m) * r
        want = r * (g - g.mean() - xh * (g * xh).mean())
        scale = r * (np.abs(g) + np.abs(g).mean() + np.abs(xh) * np.abs(g * xh).mean())
        got, dw, db = darb.layer_norm_grad(dy, x, mean, rstd, dx=dx)
        assert got is dx and untouched(dx) and untouched(dy) and untouched(x)
        check(wide(dx), want, 2e-5 * scale + rounding(want, dtype), "dx")
        check(wide(dw), (g * xh)[:, 0], 1e-5 * np.abs(g * xh)[:, 0] + 1e-30, "dw")
        check(wide(db), g[:, 0], 1e-5 * np.abs(g)[:, 0] + 1e-30, "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 3, 133, 5000])
def test_logprob_gradient_of_one_token(darb, V, dtype):  # noqa: F811
    rng = np.random.default_rng(V)
    a = rng.standard_normal((V, 1)) * 2
    word = torch.tensor([V // 2], device="cuda")
    for sz, sd in itertools.product([False, True], repeat=2):
        say(f"one token: log probability gradient {V} {dtype} strided z {sz} dz {sd}")
        z, dz = column(a, sz, dtype), column(np.zeros((V, 1)), sd, dtype)
        z64 = wide(z)
        r = darb.token_logprobs(z, word)
        lp = z64 - wide(r.lse)
        p = np.exp(lp)
        hit = np.arange(V)[:, None] == V // 2
        g = torch.tensor([0.7], device="cuda")
        want = wide(g) * (hit - p)
        got = darb.token_logprobs_grad(z, word, r.lse, g, out=dz)
        assert got is dz and untouched(dz) and untouched(z)
        check(wide(dz), want, 1e-5 * (hit + p) + rounding(want, dtype), "dz")


def test_one_element_repeated(darb):  # noqa: F811
    """One token or one feature that is only read may repeat an element; one that is written may not."""
    for F, B in ((300, 1), (1, 300)):
        say(f"one element repeated: {F} x {B}")
        rng = np.random.default_rng(F)
        x = torch.from_numpy(rng.standard_normal((F, B)).astype(np.float32)).cuda()
        dy = torch.full((1, 1), 0.25, device="cuda").expand(F, B)
        y, mean, rstd = darb.layer_norm(x)
        got = darb.layer_norm_grad(dy, x, mean, rstd)
        for a, b in zip(got, darb.layer_norm_grad(dy.contiguous(), x, mean, rstd)):
            assert torch.allclose(a, b, rtol=1e-5, atol=1e-6)
        r, want = darb.token_logprobs(dy), darb.token_logprobs(dy.contiguous())
        assert torch.allclose(r.lse, want.lse, rtol=1e-6) and torch.allclose(r.entropy, want.entropy, rtol=1e-5)
        with pytest.raises(darb.DarbError):
            darb.layer_norm(x, y=torch.zeros(1, 1, device="cuda").expand(F, B))
        with pytest.raises(darb.DarbError):
            darb.token_logprobs_grad(x, None, r.lse, r.lse, out=torch.zeros(1, 1, device="cuda").expand(F, B))
