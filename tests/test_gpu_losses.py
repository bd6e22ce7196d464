"""The policy and preference losses against their definitions in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb, say  # noqa: E402,F401
from _train import check, wide  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def f32(a):
    return np.asarray(a, np.float32).astype(np.float64)


def on(a):
    return None if a is None else torch.from_numpy(np.asarray(a, np.float32)).cuda()


def policy(lp, old, A, w, low, high, ref, kl, ent, ec):
    """(loss, kl, clipped, dlp, dent) and bounds of the first two and of dlp: an exponential is off
    by 2 units and what its argument's rounding makes of it, a product or sum by 1."""
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        d = lp - old
        r = np.exp(d)
        top, bottom = math.log1p(high), math.log1p(-low) if low < 1 else -math.inf
        cut = ((A > 0) & (d > top)) | ((A < 0) & (d < bottom))
        ratio = np.where(cut, np.where(A > 0, 1 + high, 1 - low), r)
        L, g = -ratio * A, np.where(cut, 0.0, -r * A)
        unit = (6 + np.abs(d)) * U
        eL, eg = np.abs(L) * unit, np.abs(g) * unit
        k = np.zeros_like(lp)
        if ref is not None:
            q = ref - lp
            k = np.expm1(q) - q
            # near 0 the excess is a series of 8 terms, else a difference
            ek = np.where(np.abs(q) < 0.25, 24 * U * k, U * (4 * np.abs(np.expm1(q)) + np.abs(q) * (2 + np.exp(q))))
            L, g = L + kl * k, g - kl * np.expm1(q)
            eL = eL + kl * (ek + 2 * U * k) + U * np.abs(L)
            eg = eg + kl * U * (4 * np.abs(np.expm1(q)) + np.abs(q) * np.exp(q)) + U * np.abs(g)
        if ent is not None:
            L = L - ec * ent
            eL = eL + 2 * U * np.abs(ec * ent) + U * np.abs(L)
        live = w != 0
        add = lambda v: np.where(live, w * v, 0.0)                                   # noqa: E731
        ew = np.abs(add(eL)).sum()
        ekl = 0.0 if ref is None else add(ek + U * k).sum()
        return (add(L).sum(), add(k).sum(), add(cut).sum(), add(g), -ec * w, ew, ekl,
                np.abs(add(eg)) + 2 * U * np.abs(add(g)))


def tokens(n, seed):
    r = np.random.default_rng(seed)
    lp = f32(-np.abs(r.normal(size=n)) * 2)
    return (r, lp, f32(lp + 0.2 * r.normal(size=n)), f32(r.normal(size=n)),
            f32(np.where(r.random(n) < 0.2, 0, r.random(n) / n)), f32(lp + r.normal(size=n) * r.choice([1e-4, 0.3, 1], n)),
            f32(np.abs(r.normal(size=n))))


@pytest.mark.parametrize("n", [1, 2, 3, 5, 255, 700, 8191, 8192, 8193, 8200, 100_003])
def test_policy(darb, n):
    r, lp, old, A, w, ref, ent = tokens(n, n)
    for weight in (w, None):
        for rf, kl in ((None, 0.0), (ref, 0.05), (ref, 0.0)):
            for en, ec in ((None, 0.0), (ent, 0.01)):
                for clip in (0.2, (0.2, 0.28), (1.5, 0.0)):
                    label = f"n={n} weight={weight is not None} kl={kl} ec={ec} clip={clip}"
                    low, high = clip if isinstance(clip, tuple) else (clip, clip)
                    ww = f32(np.full(n, 1 / n)) if weight is None else weight
                    want = policy(lp, old, A, ww, low, high, rf, kl, en, ec)
                    got = darb.policy_loss(on(lp), on(old), on(A), weight=on(weight), clip=clip, ref_logprob=on(rf),
                                           kl_coef=kl, entropy=on(en), entropy_coef=ec)
                    check(wide(got.loss), want[0], want[5] + U * abs(want[0]) + 1e-300, label + " loss")
                    check(wide(got.kl), want[1], want[6] + U * want[1], label + " kl")
                    check(wide(got.clipped), want[2], U * abs(want[2]), label + " clipped")
                    check(wide(got.grad_logprob), want[3], want[7], label + " dlp")
                    if en is None:
                        assert got.grad_entropy is None
                    else:
                        check(wide(got.grad_entropy), want[4], 2 * U * np.abs(want[4]), label + " dent")


def test_policy_border(darb):
    """A ratio at its bound is not past it; the next number is."""
    low, high = 0.25, 0.5
    a = np.float32(math.log1p(high))
    d = np.array([np.nextafter(a, np.float32(v)) for v in (0, 9)] + [a], np.float32)
    b = np.float32(math.log1p(-low))
    d = np.concatenate([d, [np.nextafter(b, np.float32(v)) for v in (0, -9)], [b]]).astype(np.float32)
    for A in (1.0, -1.0, 0.0):
        want = policy(f32(d), np.zeros(6), np.full(6, A), np.ones(6), low, high, None, 0.0, None, 0.0)
        got = darb.policy_loss(on(d), on(np.zeros(6)), on(np.full(6, A)), weight=on(np.ones(6)), clip=(low, high))
        assert float(got.clipped) == want[2]
        assert np.array_equal(wide(got.grad_logprob) == 0, want[3] == 0)


def test_policy_masked_places(darb):
    """A weight of 0 leaves a token out, whatever it holds; no token left gives zeros."""
    n = 9001
    r, lp, old, A, w, ref, ent = tokens(n, 3)
    w[::7] = 0
    clean = darb.policy_loss(on(lp), on(old), on(A), weight=on(w), ref_logprob=on(ref), kl_coef=0.1, entropy=on(ent),
                             entropy_coef=0.02)
    for bad in (np.nan, np.inf, -np.inf, np.finfo(np.float32).min):
        args = [np.where(np.arange(n) % 7 == 0, bad, a) for a in (lp, old, A, ref, ent)]
        got = darb.policy_loss(on(args[0]), on(args[1]), on(args[2]), weight=on(w), ref_logprob=on(args[3]),
                               kl_coef=0.1, entropy=on(args[4]), entropy_coef=0.02)
        assert all(torch.equal(p, q) for p, q in zip(got, clean))
        assert not got.grad_logprob[::7].any() and not got.grad_entropy[::7].any()
    none = darb.policy_loss(on(lp), on(old), on(A), weight=on(np.zeros(n)))
    assert float(none.loss) == 0 and float(none.kl) == 0 and not none.grad_logprob.any()
    # a token that counts makes NaN of the loss
    lp[1], w[1] = np.nan, 0.5
    got = darb.policy_loss(on(lp), on(old), on(A), weight=on(w))
    assert torch.isnan(got.loss) and torch.isnan(got.grad_logprob[1]) and torch.isfinite(got.grad_logprob[2:]).all()


def test_policy_gradient_against_differences(darb):
    r, lp, old, A, w, ref, ent = tokens(40, 17)
    d = 1e-5
    # away from the bounds, where the loss has no derivative
    old = np.where(np.abs(np.abs(lp - old) - 0.2) < 0.03, lp - 0.1, old)
    old = f32(old)
    value = lambda x: policy(x, old, A, w, 0.2, 0.2, ref, 0.3, None, 0.0)[0]         # noqa: E731
    got = wide(darb.policy_loss(on(lp), on(old), on(A), weight=on(w), ref_logprob=on(ref), kl_coef=0.3).grad_logprob)
    for i in range(40):
        e = np.zeros(40)
        e[i] = d
        want = (value(lp + e) - value(lp - e)) / (2 * d)
        # third derivatives are below 100 w, the values' own rounding below 1e-15 / d
        assert abs(got[i] - want) <= 100 * w[i] * d * d + 1e-9 + 64 * U * abs(want), i


def softplus(x):
    return np.maximum(x, 0) + np.log1p(np.exp(-np.abs(x)))


def preference(sums, w, beta, e):
    """(loss, margin, coefficient of every sequence) and their bounds.  The margin is rounded once;
    the loss's derivative by it is at most 1, an exponential or logarithm is off by 2 units."""
    P = len(sums) // 2
    m = beta * (sums[:P] - sums[P:])
    em = 2 * U * np.abs(m)
    L = (1 - e) * softplus(-m) + e * softplus(m)
    eL = em + 8 * U * (np.abs(m) + 1)
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(m))
    c = (e - s) * beta * w
    ec = beta * np.abs(w) * (0.25 * em + 6 * U * (s + e)) + 3 * U * np.abs(c)
    return (w * L).sum(), m, np.concatenate([c, -c]), (np.abs(w) * (eL + 2 * U * L)).sum(), em, np.concatenate([ec, ec])


@pytest.mark.parametrize("P,L", [(1, 1), (1, 7), (3, 50), (4, 33), (5, 200), (64, 17), (257, 3), (2, 9000)])
def test_preference_padded(darb, P, L):
    r = np.random.default_rng(P * 100 + L)
    lp, ref = f32(-np.abs(r.normal(size=(L, 2 * P)))), f32(-np.abs(r.normal(size=(L, 2 * P))))
    for rf in (ref, None):
        for w in (None, f32(np.where(r.random(P) < 0.3, 0, r.random(P)))):
            for beta, e in ((0.1, 0.0), (0.4, 0.1)):
                label = f"P={P} L={L} ref={rf is not None} w={w is not None} beta={beta}"
                b = float(np.float32(beta))
                sums = (lp - (0 if rf is None else rf)).sum(0)
                ww = f32(np.full(P, 1 / P)) if w is None else w
                loss, m, c, el, em, ec = preference(sums, ww, b, float(np.float32(e)))
                got = darb.preference_loss(on(lp).view(-1), None if rf is None else on(rf).view(-1), batch=2 * P, beta=beta,
                                           label_smoothing=e, weight=on(w))
                check(wide(got.margin), m, em + 1e-300, label + " margin")
                check(wide(got.loss), loss, el + U * abs(loss) + 1e-300, label + " loss")
                check(wide(got.grad_logprob).reshape(L, -1), np.broadcast_to(c, (L, 2 * P)),
                      np.broadcast_to(ec, (L, 2 * P)), label + " dlp")


def packed(lengths, before, behind, seed):
    r = np.random.default_rng(seed)
    starts = before + np.concatenate([[0], np.cumsum(lengths)])
    n = int(starts[-1]) + behind
    return r, starts.astype(np.int64), f32(-np.abs(r.normal(size=n))), f32(-np.abs(r.normal(size=n)))


@pytest.mark.parametrize("lengths,before,behind", [
    ([1, 1], 0, 0), ([5, 0], 0, 3), ([0, 0, 1, 0], 0, 0), ([3, 100, 128, 129, 1000, 64], 0, 0), ([10] * 8, 5, 300),
    ([70000, 3, 1, 40000], 2, 1), (list(range(0, 500)), 1, 1000)])
def test_preference_packed(darb, lengths, before, behind):
    r, starts, lp, ref = packed(lengths, before, behind, len(lengths))
    P, n = len(lengths) // 2, len(lp)
    sums = np.array([(lp[a:b] - ref[a:b]).sum() for a, b in zip(starts[:-1], starts[1:])])
    loss, m, c, el, em, ec = preference(sums, f32(np.full(P, 1 / P)), float(np.float32(0.1)), 0.0)
    d, ed = np.zeros(n), np.zeros(n)
    for s, (a, b) in enumerate(zip(starts[:-1], starts[1:])):
        d[a:b], ed[a:b] = c[s], ec[s]
    got = darb.preference_loss(on(lp), on(ref), starts=torch.from_numpy(starts).cuda(), beta=0.1)
    check(wide(got.margin), m, em + 1e-300, "margin")
    check(wide(got.loss), loss, el + U * abs(loss), "loss")
    check(wide(got.grad_logprob), d, ed, "dlp")


def test_preference_wild_places(darb):
    """Starts outside the tokens are held inside them; masked pairs and infinite margins."""
    n = 100
    lp, ref = on(np.linspace(-3, 0, n)), on(np.linspace(-2, -1, n))
    wild = torch.tensor([-50, 40, 1 << 40], device="cuda")
    held = torch.tensor([0, 40, n], device="cuda")
    a, b = (darb.preference_loss(lp, ref, starts=s) for s in (wild, held))
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    # a pair of weight 0 adds nothing
    lp4 = torch.tensor([np.nan, -1.0, -2.0, -0.5], device="cuda", dtype=torch.float32)
    w = torch.tensor([0.0, 1.0], device="cuda")
    got = darb.preference_loss(lp4, batch=4, weight=w, beta=1.0)
    assert torch.isfinite(got.loss) and got.grad_logprob[0] == 0 and got.grad_logprob[2] == 0
    want = darb.preference_loss(lp4[1::2].contiguous(), batch=2, beta=1.0)
    assert torch.equal(got.loss, want.loss) and torch.equal(got.grad_logprob[1::2], want.grad_logprob)
    # a preferred sequence of probability 0 has an infinite loss and a whole gradient; the reverse none
    lp2 = torch.tensor([-np.inf, -1.0], device="cuda", dtype=torch.float32)
    got = darb.preference_loss(lp2, batch=2, beta=0.5)
    assert float(got.loss) == np.inf and got.grad_logprob.tolist() == [-0.5, 0.5]
    got = darb.preference_loss(lp2.flip(0), batch=2, beta=0.5)
    assert float(got.loss) == 0 and got.grad_logprob.tolist() == [0, 0]
    got = darb.preference_loss(lp2.flip(0), batch=2, beta=0.5, label_smoothing=0.25)
    assert float(got.loss) == np.inf


def test_preference_gradient_against_differences(darb):
    r, starts, lp, ref = packed([3, 1, 4, 2], 1, 1, 5)
    d = 1e-5

    def value(x):
        sums = np.array([(x[a:b] - ref[a:b]).sum() for a, b in zip(starts[:-1], starts[1:])])
        return preference(sums, np.array([0.5, 0.5]), float(np.float32(0.7)), float(np.float32(0.1)))[0]
    got = wide(darb.preference_loss(on(lp), on(ref), starts=torch.from_numpy(starts).cuda(), beta=0.7,
                                    label_smoothing=0.1).grad_logprob)
    for i in range(len(lp)):
        e = np.zeros(len(lp))
        e[i] = d
        want = (value(lp + e) - value(lp - e)) / (2 * d)
        assert abs(got[i] - want) <= d * d + 1e-9 + 32 * U * abs(want), i


def test_outputs_in_place(darb):
    for n in (700, 9001):
        r, lp, old, A, w, ref, ent = tokens(n, n)
        want = darb.policy_loss(on(lp), on(old), on(A), weight=on(w), ref_logprob=on(ref), kl_coef=0.1, entropy=on(ent),
                                entropy_coef=0.02)
        a, h = on(lp), on(ent)
        got = darb.policy_loss(a, on(old), on(A), weight=on(w), ref_logprob=on(ref), kl_coef=0.1, entropy=h,
                               entropy_coef=0.02, grad_logprob=a, grad_entropy=h)
        assert got.grad_logprob is a and got.grad_entropy is h and all(torch.equal(p, q) for p, q in zip(got, want))
        m = n // 10 * 10
        a = on(lp[:m])
        want = darb.preference_loss(a, on(ref[:m]), batch=10)
        got = darb.preference_loss(a, on(ref[:m]), batch=10, grad_logprob=a)
        assert got.grad_logprob is a and all(torch.equal(p, q) for p, q in zip(got, want))


def test_streams_and_graphs(darb):
    from _streams import Busy, copies, same
    busy = Busy()
    n = 40000
    r, lp, old, A, w, ref, ent = (on(a) if isinstance(a, np.ndarray) else a for a in tokens(n, 1))
    starts = torch.tensor([0, 100, 20000, 20000, n - 7], device="cuda")

    def every(stream=None):
        return (darb.policy_loss(lp, old, A, weight=w, ref_logprob=ref, kl_coef=0.1, entropy=ent, entropy_coef=0.1,
                                 stream=stream),
                darb.preference_loss(lp, ref, batch=100, stream=stream),
                darb.preference_loss(lp, ref, starts=starts, stream=stream))
    want = copies(every())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy.queue()
    got = every(side)
    side.synchronize()
    assert same(copies(got), want)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        every()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = every()
    for k in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert same(copies(out), want), k
        every()
    A.mul_(2.0)
    g.replay()
    assert same(copies(out), copies(every()))
