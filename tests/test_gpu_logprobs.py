"""Token log probabilities and their gradient against the definition in 64 bits.

Bounds.  A term e^(z - m) is off by at most (|z - m| + 2) 2^-23 relative (the rounded product
with log2 e, the exponential's last place); weighted by the terms' shares of the sum, which
leaves |z - m| below some 20, and with the sum's own roundings that is below 1e-5 in the log
sum, and 2e-5 in the entropy.  Values themselves carry two roundings of 2^-24.  A probability
in the gradient is off by (|log p| + 2) 2^-23 relative, below 1e-5 where it counts.
"""
import numpy as np
import pytest

from tests._gpu import darb, say, torch  # noqa: F401
from tests._train import ORDERS, check, place, rounding, wide

pytestmark = pytest.mark.gpu


def oracle(z, t, top):
    """fp64: logprob, entropy, lse, top_logprob, top_index of z [V, B] (float64 of the stored
    values)."""
    V, B = z.shape
    m = z.max(0)
    bad = np.isnan(z).any(0) | (z == np.inf).any(0)
    empty = (z == -np.inf).all(0)
    ms = np.where(empty | bad, 0.0, m)
    with np.errstate(all="ignore"):
        d = z - ms
        e = np.exp(d)
        S = e.sum(0)
        lse = np.where(empty, -np.inf, ms + np.log(S))
        H = np.where(empty, 0.0, np.log(S) - np.where(e > 0, e * d, 0.0).sum(0) / S)
        lse[bad] = H[bad] = np.nan
        y = z[np.clip(t, 0, V - 1), np.arange(B)] - lse
    y[empty] = -np.inf
    y[t < 0] = 0.0
    y[t >= V] = np.nan
    y[bad & (t >= 0)] = np.nan
    # NaN first, then by value, equal ones by the lower class
    key = np.where(np.isnan(z), np.inf, z)
    rank = np.lexsort((np.broadcast_to(np.arange(V)[:, None], z.shape), -key, ~np.isnan(z)), axis=0)
    index = rank[:top].T
    with np.errstate(all="ignore"):
        tl = np.take_along_axis(z, index.T, 0).T - lse[:, None]
    tl[empty] = -np.inf
    return y, H, lse, tl, index


def logits(rng, V, B, kind):
    z = rng.standard_normal((V, B)) * 3
    if kind == "masked":
        z[rng.random((V, B)) < 0.4] = -np.inf
        z[:, rng.random(B) < 0.2] = -np.inf              # nothing left
        z[rng.integers(V), :] = np.where(rng.random(B) < 0.5, 1.0, z[rng.integers(V), :])
    elif kind == "ties":
        z = np.round(z)
    elif kind == "lowest":
        z[rng.random((V, B)) < 0.5] = -60000.0
        z[:, ::2] = -60000.0                             # the same lowest value everywhere
    elif kind == "far":
        z = z * 400 + 3000
    return z


def targets(rng, V, B):
    t = rng.integers(0, V, B)
    t[rng.random(B) < 0.2] = -1
    t[rng.random(B) < 0.05] = V + 3
    return t.astype(np.int64)


def run(darb, z, t, top, dtype, order, label):  # noqa: F811
    zd = place(z, order, dtype)
    z64 = wide(zd)
    td = torch.from_numpy(t).cuda()
    say(label)
    r = darb.token_logprobs(zd, td, top=top)
    y, H, lse, tl, ti = oracle(z64, t, top)
    size = np.abs(np.where(np.isfinite(lse), lse, 0))
    check(wide(r.lse), lse, 1e-5 + 2.0 ** -22 * size, label + " lse")
    big = np.abs(np.where(np.isfinite(y), y, 0))
    check(wide(r.logprob), y, 1e-5 + 2.0 ** -22 * (size + big), label + " logprob")
    check(wide(r.entropy), H, 2e-5 * (1 + H), label + " entropy")
    if top:
        assert np.array_equal(r.top_index.cpu().numpy(), ti), label
        big = np.abs(np.where(np.isfinite(tl), tl, 0))
        check(wide(r.top_logprob), tl, 1e-5 + 2.0 ** -22 * (size[:, None] + big), label + " top")
    else:
        assert r.top_index is None and r.top_logprob is None
    return zd, z64, td, r, (y, H, lse)


def check_grad(darb, rng, zd, z64, td, r, dtype, label, entropy=True):  # noqa: F811
    V, B = z64.shape
    t = td.cpu().numpy()
    g = rng.standard_normal(B).astype(np.float32)
    ge = rng.standard_normal(B).astype(np.float32) if entropy else np.zeros(B, np.float32)
    lse, H = wide(r.lse), wide(r.entropy)
    with np.errstate(all="ignore"):
        lp = z64 - lse
        p = np.exp(lp)
        hit = np.arange(V)[:, None] == t
        gg = np.where(t < 0, 0.0, g.astype(np.float64))
        mixed = np.where(p > 0, p * (lp + H), p * 0)
        want = gg * (hit - p) - ge * mixed
        scale = np.abs(gg) * (hit + p) + np.abs(ge) * p * (np.abs(np.where(p > 0, lp, 0)) + H + 1)
    want[:, t >= V] = np.nan
    want[:, lse == -np.inf] = 0.0
    scale[:, lse == -np.inf] = 0.0
    scale = np.where(np.isfinite(scale), scale, 0)
    kw = dict(entropy=r.entropy, grad_entropy=torch.from_numpy(ge).cuda()) if entropy else {}
    before = zd.clone()
    dz = darb.token_logprobs_grad(zd, td, r.lse, torch.from_numpy(g).cuda(), **kw)
    assert dz.dtype == zd.dtype and torch.equal(zd.nan_to_num(5.0), before.nan_to_num(5.0))
    # e^x is flushed to zero below the smallest normal number
    check(wide(dz), want, 1e-5 * scale + rounding(want, dtype) + 2.0 ** -126 * np.abs(g), label + " dz")
    inplace = zd.clone(memory_format=torch.preserve_format)
    out = darb.token_logprobs_grad(inplace, td, r.lse, torch.from_numpy(g).cuda(), out=inplace, **kw)
    assert out is inplace and torch.equal(wide_t(out), wide_t(dz)), label


def wide_t(t):
    return t.float().nan_to_num(12345.0)


SIZES = [(1, 1, 1), (1, 5, 1), (2, 3, 2), (5, 1, 5), (7, 64, 3), (63, 2, 8), (64, 65, 64), (65, 7, 20),
         (255, 17, 5), (257, 130, 5), (1000, 33, 10), (4099, 9, 20), (2500, 260, 3), (20011, 3, 50)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V,B,top", SIZES)
def test_logprobs_orders(darb, V, B, top, dtype):  # noqa: F811
    rng = np.random.default_rng(V * 131 + B)
    z, t = logits(rng, V, B, "plain"), targets(rng, V, B)
    seen = []
    for order in ORDERS:
        label = f"logprobs {V}x{B} {dtype} {order}"
        zd, z64, td, r, _ = run(darb, z, t, top, dtype, order, label)
        check_grad(darb, rng, zd, z64, td, r, dtype, label, entropy=order != "tokens")
        seen.append(r)
    if V == 1 or B == 1:                     # a contiguous vector has both orders, a strided one
        return
    # an order's bits do not depend on the leading dimension or the alignment
    for a, b in ((0, 2), (1, 3)):
        for x, y in zip(seen[a], seen[b]):
            assert x is None and y is None or torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0))


@pytest.mark.parametrize("kind", ["masked", "ties", "lowest", "far"])
@pytest.mark.parametrize("order", ["features", "tokens"])
@pytest.mark.parametrize("V,B,top", [(3, 6, 3), (700, 21, 12), (1, 4, 1), (5000, 4, 64)])
def test_logprobs_masks(darb, V, B, top, order, kind):  # noqa: F811
    rng = np.random.default_rng(V + B)
    z, t = logits(rng, V, B, kind), targets(rng, V, B)
    for dtype in ("f32", "f16") if kind != "far" else ("f32",):
        label = f"logprobs {kind} {V}x{B} {dtype} {order}"
        zd, z64, td, r, _ = run(darb, z, t, top, dtype, order, label)
        check_grad(darb, rng, zd, z64, td, r, dtype, label)


@pytest.mark.parametrize("order", ["features", "tokens"])
def test_logprobs_nan_and_infinity(darb, order):  # noqa: F811
    rng = np.random.default_rng(5)
    V, B = 900, 8
    z = rng.standard_normal((V, B))
    z[17, 1] = np.nan
    z[[3, 800], 2] = np.nan
    z[40, 3] = np.inf
    z[:, 4] = -np.inf
    z[11, 4] = np.nan
    z[:, 5] = -np.inf
    z[899, 5] = 2.0                                  # one class left
    z[:, 6] = -np.inf
    run(darb, z, np.arange(B).astype(np.int64), 6, "f32", order, f"logprobs special {order}")
    zd = place(z, order, "f32")
    r = darb.token_logprobs(zd, torch.arange(B).cuda())
    ones = torch.ones(B, device="cuda")
    dz = wide(darb.token_logprobs_grad(zd, torch.arange(B).cuda(), r.lse, ones, r.entropy, ones))
    assert np.isnan(dz[:, [1, 2, 3, 4]]).all() and np.isfinite(dz[:, [0, 5, 6, 7]]).all()
    assert (dz[:, 6] == 0).all()
    # class 899 has all of column 5; its target, class 5, has none: the formula's 1 there
    assert dz[5, 5] == 1.0 and abs(dz[899, 5] + 1) < 1e-6 and np.count_nonzero(dz[:, 5]) == 2


@pytest.mark.parametrize("order", ["features", "tokens"])
def test_logprobs_extremes_of_fp32(darb, order):  # noqa: F811
    low = np.finfo(np.float32).min
    z = np.full((300, 3), low)
    z[:, 1] = -low
    z[7, 2] = 1.0
    y, H, lse, tl, ti = oracle(z, np.array([0, 1, 7]), 2)
    r = darb.token_logprobs(place(z, order, "f32"), torch.tensor([0, 1, 7]).cuda(), top=2)
    assert np.allclose(wide(r.entropy), H, rtol=1e-5, atol=1e-5)
    assert np.array_equal(r.top_index.cpu().numpy(), ti)
    assert np.allclose(wide(r.lse), lse, rtol=1e-6)
    assert abs(float(r.logprob[2])) < 1e-5


def test_logprobs_long(darb):  # noqa: F811
    rng = np.random.default_rng(3)
    for V, B, order in ((131073, 2, "tokens"), (131073, 1, "features"), (300001, 1, "tokens"),
                        (70001, 5, "features")):
        z, t = logits(rng, V, B, "plain"), targets(rng, V, B)
        z[V - 1, 0] = 30.0
        zd, z64, td, r, _ = run(darb, z, t, 20, "f32", order, f"logprobs long {V}x{B} {order}")
        check_grad(darb, rng, zd, z64, td, r, "f32", f"logprobs long {V}x{B}")


def test_logprobs_many_tokens(darb):  # noqa: F811
    # more rows, and more tiles of 64 tokens, than a grid's second axis holds
    V, B = 3, 65535 + 10
    rng = np.random.default_rng(4)
    z, t = rng.standard_normal((V, B)), rng.integers(0, V, B)
    for order in ("features", "tokens"):
        zd, z64, td, r, _ = run(darb, z, t, 2, "f16", order, f"logprobs {V}x{B} {order}")
        check_grad(darb, rng, zd, z64, td, r, "f16", "many tokens")
    z = torch.randn(1, 65535 * 64 + 70, device="cuda")
    r = darb.token_logprobs(z, top=1)
    assert bool((r.logprob == 0).all()) and bool((r.lse == z[0]).all())
    assert bool((r.top_index == 0).all()) and bool((r.entropy == 0).all())


def test_logprobs_repeat_and_streams(darb):  # noqa: F811
    rng = np.random.default_rng(8)
    z, t = logits(rng, 5000, 40, "plain"), targets(rng, 5000, 40)
    zd, td = place(z, "features", "f32"), torch.from_numpy(t).cuda()
    first = darb.token_logprobs(zd, td, top=4)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    ws = torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda")      # what it holds is not read
    torch.cuda.synchronize()
    again = darb.token_logprobs(zd, td, top=4, workspace=ws, stream=st)
    st.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))


def test_logprobs_gradient_by_differences(darb):  # noqa: F811
    # a central difference of the fp32 loss: h^2 / 6 times a third derivative of order 1, and
    # the loss's error 1e-5 over h
    rng = np.random.default_rng(6)
    V, B, h = 40, 6, 3e-2
    z, u = rng.standard_normal((V, B)), rng.standard_normal((V, B)) / 6
    t = rng.integers(0, V, B)
    g, ge = rng.random(B) + 0.5, rng.random(B)

    def loss(a):
        r = darb.token_logprobs(place(a, "features", "f32"), torch.from_numpy(t).cuda())
        return float((wide(r.logprob) * g + wide(r.entropy) * ge).sum())

    zd = place(z, "features", "f32")
    r = darb.token_logprobs(zd, torch.from_numpy(t).cuda())
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()              # noqa: E731
    dz = wide(darb.token_logprobs_grad(zd, torch.from_numpy(t).cuda(), r.lse, f(g), r.entropy, f(ge)))
    slope = (loss(z + h * u) - loss(z - h * u)) / (2 * h)
    assert abs(slope - (dz * u).sum()) < B * (h * h + 2e-5 / h)


@pytest.mark.parametrize("bad,err", [
    (lambda d, z, t: d.token_logprobs(z.cpu()), ValueError),
    (lambda d, z, t: d.token_logprobs(z.double()), TypeError),
    (lambda d, z, t: d.token_logprobs(z[0]), ValueError),
    (lambda d, z, t: d.token_logprobs(z[:, :0]), ValueError),
    (lambda d, z, t: d.token_logprobs(z[::2, ::2]), ValueError),
    (lambda d, z, t: d.token_logprobs(z[:1].expand(10, 8)), ValueError),
    (lambda d, z, t: d.token_logprobs(z, t[:-1]), ValueError),
    (lambda d, z, t: d.token_logprobs(z, t.int()), TypeError),
    (lambda d, z, t: d.token_logprobs(z, t.cpu()), ValueError),
    (lambda d, z, t: d.token_logprobs(z, t, top=11), "DarbError"),
    (lambda d, z, t: d.token_logprobs(z, t, top=-1), "DarbError"),
    (lambda d, z, t: d.token_logprobs(z, t, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), ValueError),
    (lambda d, z, t: d.token_logprobs_grad(z, t, t.float()), "DarbError"),
    (lambda d, z, t: d.token_logprobs_grad(z, t, t.float(), t.float(), entropy=t.float()), "DarbError"),
    (lambda d, z, t: d.token_logprobs_grad(z, t, t.half(), t.float()), TypeError),
    (lambda d, z, t: d.token_logprobs_grad(z, t, t.float(), t.float(), out=z.half()), TypeError),
    (lambda d, z, t: d.token_logprobs_grad(z, t, t.float(), t.float(), out=torch.empty(8, 10, device="cuda").t()), "DarbError"),
])
def test_logprobs_refusals(darb, bad, err):  # noqa: F811
    z, t = torch.zeros(10, 8, device="cuda"), torch.zeros(8, dtype=torch.int64, device="cuda")
    with pytest.raises(darb.DarbError if err == "DarbError" else err):
        bad(darb, z, t)
