"""Layer norm and its gradients against the definition in 64 bits.

Bounds.  The mean is off by some 2^-22 of the mean magnitude; y by a few roundings of its terms
(1e-5 of |xh w|, |w| and |b| together) and, where the mean is large beside the spread, by the
mean's own rounding times rstd w.  The gradients are sums of products with a few roundings each:
1e-5 (dx 2e-5) of the terms' magnitudes.  16-bit results add one rounding.
"""
import numpy as np
import pytest

from tests._gpu import darb, say, torch  # noqa: F401
from tests._train import ORDERS, TYPES, check, place, rounding, wide

pytestmark = pytest.mark.gpu
EPS = 1e-5


def oracle(x, w, b, eps=EPS):
    mean = x.mean(0)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(0) + eps)
    xh = (x - mean) * rstd
    return xh * w[:, None] + b[:, None], mean, rstd, xh


def params(rng, H, dtype):
    t = [torch.from_numpy(a.astype(np.float32)).to(TYPES[dtype]).cuda()
         for a in (1 + 0.3 * rng.standard_normal(H), 0.2 * rng.standard_normal(H))]
    return t[0], t[1], wide(t[0]), wide(t[1])


def run(darb, x, dtype, wdtype, order, rng, label, affine=True):  # noqa: F811
    H, B = x.shape
    xd = place(x, order, dtype)
    x64 = wide(xd)
    w, b, w64, b64 = params(rng, H, wdtype)
    if not affine:
        w, b, w64, b64 = None, None, np.ones(H), np.zeros(H)
    say(label)
    y, mean, rstd = darb.layer_norm(xd, w, b, eps=EPS)
    wy, wmean, wrstd, xh = oracle(x64, w64, b64)
    size = np.abs(x64).mean(0)
    check(wide(mean), wmean, 2.0 ** -22 * size + 1e-30, label + " mean")
    slip = 2.0 ** -22 * size * wrstd                     # the mean's rounding, in units of xh
    check(wide(rstd), wrstd, wrstd * (2e-6 + slip ** 2), label + " rstd")
    terms = np.abs(xh * w64[:, None]) + np.abs(w64[:, None]) + np.abs(b64[:, None])
    check(wide(y), wy, 1e-5 * terms + slip * np.abs(w64[:, None]) * (1 + slip * np.abs(xh)) + rounding(wy, dtype),
          label + " y")
    assert y.dtype == xd.dtype and y.shape == xd.shape
    # gradients, from the statistics as the call returned them
    dy = rng.standard_normal((H, B)) * 0.5
    dyd = place(dy, order, dtype)
    g = wide(dyd)
    m, r = wide(mean), wide(rstd)
    xh = (x64 - m) * r
    a = g * w64[:, None]
    dx = r * (a - a.mean(0) - xh * (a * xh).mean(0))
    scale = r * (np.abs(a) + np.abs(a).mean(0) + np.abs(xh) * np.abs(a * xh).mean(0))
    out = darb.layer_norm_grad(dyd, xd, mean, rstd, w)
    check(wide(out[0]), dx, 2e-5 * scale + rounding(dx, dtype), label + " dx")
    check(wide(out[1]), (g * xh).sum(1), 1e-5 * np.abs(g * xh).sum(1) + 1e-30, label + " dw")
    check(wide(out[2]), g.sum(1), 1e-5 * np.abs(g).sum(1) + 1e-30, label + " db")
    return xd, dyd, w, (y, mean, rstd), out


SHAPES = [(1, 1), (1, 70), (2, 3), (3, 64), (16, 1), (63, 5), (64, 64), (65, 9), (100, 300), (257, 33), (1000, 7),
          (1024, 32), (1500, 20), (2049, 5), (4096, 40), (5000, 3), (9216, 17), (16384, 4), (20000, 2), (33000, 1)]


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("f16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("H,B", SHAPES)
def test_layer_norm_orders(darb, H, B, dtype, wdtype):  # noqa: F811
    x = np.random.default_rng(H * 7 + B).standard_normal((H, B)) * 1.5 + 0.3
    seen = []
    for order in ORDERS:
        rng = np.random.default_rng(H + B)
        seen.append(run(darb, x, dtype, wdtype, order, rng, f"norm {H}x{B} {dtype} {order}")[3:])
    if H == 1 or B == 1:                     # a contiguous vector has both orders, a strided one
        return
    for a, b in ((0, 2), (1, 3)):            # bits do not depend on leading dimension or alignment
        for p, q in zip(seen[a], seen[b]):
            assert all(torch.equal(s, t) for s, t in zip(p, q)), (H, B, a)


@pytest.mark.parametrize("order", ["features", "tokens"])
@pytest.mark.parametrize("kind", ["offset", "constant", "tiny", "no affine", "many"])
def test_layer_norm_values(darb, kind, order):  # noqa: F811
    rng = np.random.default_rng(9)
    x = rng.standard_normal((300, 3000 if kind == "many" else 20))
    if kind == "offset":
        x += 4096.0
    elif kind == "constant":
        x[:, ::2] = 0.25                     # no spread: y is the bias, rstd 1 / sqrt(eps)
    elif kind == "tiny":
        x *= 1e-6                            # eps decides
    run(darb, x, "f32", "f32", order, rng, f"norm {kind} {order}", affine=kind != "no affine")


def test_layer_norm_outputs_of_choice(darb):  # noqa: F811
    rng = np.random.default_rng(1)
    for order in ("features", "tokens"):
        x = rng.standard_normal((130, 50))
        xd, dyd, w, (y, mean, rstd), (dx, dw, db) = run(darb, x, "f32", "f32", order, rng, f"norm choice {order}")
        only = darb.layer_norm_grad(dyd, xd, mean, rstd, w, need_params=False)
        assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
        only = darb.layer_norm_grad(dyd, xd, mean, rstd, w, need_x=False)
        assert only[0] is None and torch.equal(only[1], dw) and torch.equal(only[2], db)
        # in place, from either operand, and a workspace whose contents do not matter
        ws = torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
        for k in (0, 1):
            a = [dyd.clone(memory_format=torch.preserve_format), xd.clone(memory_format=torch.preserve_format)]
            got = darb.layer_norm_grad(a[0], a[1], mean, rstd, w, dx=a[k], workspace=ws)
            assert got[0] is a[k] and all(torch.equal(p, q) for p, q in zip(got, (dx, dw, db)))
        x2 = xd.clone(memory_format=torch.preserve_format)
        b = torch.zeros(130, device="cuda")
        want = darb.layer_norm(xd, w, b)[0]
        assert torch.equal(darb.layer_norm(x2, w, b, y=x2)[0], want)


@pytest.mark.parametrize("order", ["features", "tokens"])
def test_layer_norm_nan_stays_in_its_column(darb, order):  # noqa: F811
    rng = np.random.default_rng(2)
    x = rng.standard_normal((200, 9))
    x[3, 4], x[7, 6] = np.nan, np.inf
    xd = place(x, order, "f32")
    y, mean, rstd = darb.layer_norm(xd, torch.ones(200, device="cuda"), None)
    bad = np.isnan(wide(y))
    assert bad[:, [4, 6]].all() and not np.delete(bad, [4, 6], 1).any()
    dy = place(rng.standard_normal((200, 9)), order, "f32")
    dx, dw, db = darb.layer_norm_grad(dy, xd, mean, rstd)
    bad = np.isnan(wide(dx))
    assert bad[:, [4, 6]].all() and not np.delete(bad, [4, 6], 1).any()
    assert np.isnan(wide(dw)).all() and np.isfinite(wide(db)).all()


@pytest.mark.parametrize("order", ["features", "tokens"])
def test_layer_norm_gradient_by_differences(darb, order):  # noqa: F811
    # central differences of a loss summed in fp64 from fp32 results: h^2 and 1e-5 / h apart
    rng = np.random.default_rng(3)
    H, B, h = 48, 5, 2e-2
    x, u, r = rng.standard_normal((H, B)), rng.standard_normal((H, B)), rng.standard_normal((H, B))
    w, b = 1 + 0.2 * rng.standard_normal(H), 0.2 * rng.standard_normal(H)
    uw, ub = rng.standard_normal(H), rng.standard_normal(H)
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()              # noqa: E731

    def loss(x, w, b):
        return (wide(darb.layer_norm(place(x, order, "f32"), f(w), f(b))[0]) * r).sum()

    xd = place(x, order, "f32")
    _, mean, rstd = darb.layer_norm(xd, f(w), f(b))
    dx, dw, db = (wide(t) for t in darb.layer_norm_grad(place(r, order, "f32"), xd, mean, rstd, f(w)))
    bound = np.sqrt(H * B) * (4 * h * h + 1e-5 / h)
    for got, up, down in (((dx * u).sum(), (x + h * u, w, b), (x - h * u, w, b)),
                          ((dw * uw).sum(), (x, w + h * uw, b), (x, w - h * uw, b)),
                          ((db * ub).sum(), (x, w, b + h * ub), (x, w, b - h * ub))):
        assert abs((loss(*up) - loss(*down)) / (2 * h) - got) < bound


def test_layer_norm_stream(darb):  # noqa: F811
    x = torch.randn(512, 700, device="cuda")
    dy = torch.randn(512, 700, device="cuda")
    y, mean, rstd = darb.layer_norm(x)
    want = darb.layer_norm_grad(dy, x, mean, rstd)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y2, m2, r2 = darb.layer_norm(x, stream=st)
    got = darb.layer_norm_grad(dy, x, m2, r2, stream=st)
    st.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("bad,err", [
    (lambda d, x, v: d.layer_norm(x.cpu()), ValueError),
    (lambda d, x, v: d.layer_norm(x.double()), TypeError),
    (lambda d, x, v: d.layer_norm(x[::2, ::2]), ValueError),
    (lambda d, x, v: d.layer_norm(x[:, :0]), ValueError),
    (lambda d, x, v: d.layer_norm(x, v[:-1]), ValueError),
    (lambda d, x, v: d.layer_norm(x, v.half()), TypeError),
    (lambda d, x, v: d.layer_norm(x.half(), v, v.half()), TypeError),
    (lambda d, x, v: d.layer_norm(x, v, eps=-1.0), "DarbError"),
    (lambda d, x, v: d.layer_norm(x, v, eps=float("nan")), "DarbError"),
    (lambda d, x, v: d.layer_norm(x, y=x.half()), TypeError),
    (lambda d, x, v: d.layer_norm(x, y=torch.empty(8, 10, device="cuda").t()), "DarbError"),
    (lambda d, x, v: d.layer_norm(x, mean=v.half()), TypeError),
    (lambda d, x, v: d.layer_norm_grad(x[:, :-1], x, v, v), ValueError),
    (lambda d, x, v: d.layer_norm_grad(x.half(), x, v, v), TypeError),
    (lambda d, x, v: d.layer_norm_grad(x, x, v[:3], v), ValueError),
    (lambda d, x, v: d.layer_norm_grad(x[:, :1].expand(10, 8), x, v, v), ValueError),
    (lambda d, x, v: d.layer_norm_grad(x, x, v, v, need_x=False, need_params=False), "DarbError"),
    (lambda d, x, v: d.layer_norm_grad(x, x, v, v, dweight=v.half()), TypeError)])
def test_layer_norm_refusals(darb, bad, err):  # noqa: F811
    x, v = torch.zeros(10, 8, device="cuda"), torch.ones(10, device="cuda")
    with pytest.raises(darb.DarbError if err == "DarbError" else err):
        bad(darb, x, v)
