"""The orthogonalised update against its definition in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb, say  # noqa: E402,F401
from _train import ROUND, TYPES, check, wide  # noqa: E402

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
U = 2.0 ** -24


def poly(s):
    return A * s + B * s ** 3 + C * s ** 5


def exact(G, steps, eps):
    """The orthogonalised G in 64 bits, through its singular values."""
    x = G / (np.linalg.norm(G) + eps)
    u, s, v = np.linalg.svd(x, full_matrices=False)
    for _ in range(steps):
        s = poly(s)
    return (u * s) @ v


def stretch(s, wide):
    """How much a step can enlarge a small change of X, in the Frobenius norm: an odd function of the
    singular values changes by its divided differences over them and their negatives (and over 0 where
    the matrix is not square)."""
    s = np.concatenate([s, [0.0]]) if wide else s
    a, b = np.meshgrid(s, s)
    near, sum_ = np.abs(a - b) < 1e-9, a + b
    slope = A + 3 * B * a ** 2 + 5 * C * a ** 4
    with np.errstate(divide="ignore", invalid="ignore"):
        d = np.where(near, slope, (poly(a) - poly(b)) / np.where(near, 1, a - b))
        e = np.where(sum_ < 1e-9, A, (poly(a) + poly(b)) / np.where(sum_ < 1e-9, 1, sum_))
    return max(np.abs(d).max(), np.abs(e).max())


def bound(G, steps, eps, full):
    """A bound of the error's Frobenius norm before the result is rounded to its type.

    An fp32 result: hi + lo holds 22 bits, so each operand is off by 2^-22 of itself, the product of
    the lo parts is left out (2^-22) and a sum of K terms off by (K + 2) 2^-24 of the terms'
    magnitudes (two more sums of as many): c = 3 2^-22 + 3 (K + 2) 2^-24 of them, whose matrix has at
    most the product of the factors' Frobenius norms.  A 16-bit one: the factors of A and of the
    last product are rounded to 2^-11 each, independently, so that an element of a product of m and K
    is off by less than 6 standard deviations, 6 2^-11 sqrt(2 / 3) of the root of the sum of the
    terms' squares; A A's are as before.  X itself is held in 22 bits.  A's error reaches X by
    (b + 2 c A) X, that of A A by c X, that of the last product as it is."""
    x = G / (np.linalg.norm(G) + eps)
    u, s, v = np.linalg.svd(x, full_matrices=False)
    m, n = min(G.shape), max(G.shape)
    total = (2 * 2.0 ** -22 + (2 + math.log2(m * n)) * 2.0 ** -53) * 1.0
    for _ in range(steps):
        xk = (u * s) @ v
        xk = xk if xk.shape[0] <= xk.shape[1] else xk.T
        a = xk @ xk.T
        q = B * a + C * a @ a
        big = s.max()

        def product(p, r, single):
            exactly = (3 * 2.0 ** -22 + 3 * (p.shape[1] + 2) * U) * np.linalg.norm(p) * np.linalg.norm(r)
            if not single:
                return exactly
            return exactly + 6 * 2.0 ** -11 * math.sqrt(2 / 3) * np.sqrt((p ** 2 @ r.T ** 2).sum())
        da = product(xk, xk, not full) + 2.0 ** -22 * np.linalg.norm(a)
        dq = (abs(B) + 2 * C * big ** 2) * da + abs(C) * product(a, a, False) + \
            (2.0 ** -22 if full else 2.0 ** -11) * np.linalg.norm(q) * (1.0 if full else 0.0) + 2.0 ** -22 * np.linalg.norm(q)
        dx = big * dq + product(q, xk.T, not full) + 2.0 ** -22 * np.linalg.norm(xk)
        total = total * stretch(s, m != n) + dx
        s = poly(s)
    return total


def matrix(m, n, kind, seed):
    r = np.random.default_rng(seed)
    g = r.normal(size=(m, n))
    if kind == "flat":                      # singular values between 0.7 and 1 of each other
        u, s, v = np.linalg.svd(g, full_matrices=False)
        g = (u * np.linspace(0.7, 1, len(s))) @ v
    if kind == "low":
        k = max(1, min(m, n) // 4)
        g = r.normal(size=(m, k)) @ r.normal(size=(k, n)) + 0.5 * g
    return g


SHAPES = [(1, 1), (1, 7), (5, 1), (3, 4), (17, 17), (40, 90), (130, 70), (128, 128), (129, 257), (64, 700), (300, 300)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["flat", "low"])
def test_orthogonalize(darb, dtype, kind):
    for n, (rows, cols) in enumerate(SHAPES):
        G = torch.from_numpy(matrix(rows, cols, kind, n) * 10.0 ** (n % 5 - 2)).to(TYPES[dtype])
        g = G.double().numpy()
        want = exact(g, 5, 1e-7)
        got = wide(darb.orthogonalize(G.cuda()))
        limit = bound(g, 5, 1e-7, dtype == "f32")
        rounded = ROUND[dtype][0] * np.linalg.norm(want) + ROUND[dtype][1] * math.sqrt(want.size)
        off = np.linalg.norm(got - want)
        say(f"{dtype} {kind} {rows}x{cols}: {off / np.linalg.norm(want):.2e} of the result, bound "
            f"{(limit + rounded) / np.linalg.norm(want):.2e}")
        assert np.isfinite(got).all() and off <= limit + rounded


@pytest.mark.parametrize("dtype", list(TYPES))
def test_every_tile(darb, dtype):
    """Each kind of tile that a product may go by, where tiles hang over, and where the sums are shorter
    than the stages that are loaded ahead."""
    import ctypes
    P, I64, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    call = darb.lib().darb_test_orthogonalize
    call.argtypes, call.restype = [P, I64, I, ctypes.c_double, P, I64, I, I, I, P], I
    code = {"f32": 0, "f16": 1, "bf16": 2}[dtype]
    shapes = [(64, 64), (70, 900), (290, 300), (520, 270), (400, 590), (333, 1100)]
    mats = [torch.from_numpy(matrix(*s, "flat", 70 + i)).to(TYPES[dtype]).cuda() for i, s in enumerate(shapes)]
    want = [exact(wide(g), 5, 1e-7) for g in mats]
    limit = [bound(wide(g), 5, 1e-7, dtype == "f32") for g in mats]
    for kinds in ((0, 0, 0), (2, 2, 1), (2, 2, 2), (3, 3, 3), (4, 4, 4), (4, 0, 1)):
        for only in (None, 3):
            table = (darb._MuonTensor * len(mats))()
            out = [torch.empty_like(g) for g in mats]
            chosen = [i for i in range(len(mats)) if only in (None, i)]
            for j, i in enumerate(chosen):
                r, c = shapes[i]
                table[j] = darb._MuonTensor(out[i].data_ptr(), None, mats[i].data_ptr(), None, r, c, c, c, 1.0, 0.0, code, code)
            n = ctypes.c_int64()
            assert darb.lib().darb_muon_workspace(table, len(chosen), ctypes.byref(n)) == 0
            # what the call does not write itself would show as NaN
            ws = torch.full((n.value // 4,), math.nan, device="cuda")
            for again in range(2):
                say(dtype, kinds, only, again)
                assert call(table, len(chosen), 5, 1e-7, ws.data_ptr(), n.value, *kinds,
                            torch.cuda.current_stream().cuda_stream) == 0
                for i in chosen:
                    got = wide(out[i])
                    off = np.linalg.norm(got - want[i])
                    rounded = ROUND[dtype][0] * np.linalg.norm(want[i]) + ROUND[dtype][1] * math.sqrt(got.size)
                    assert off <= limit[i] + rounded, (kinds, shapes[i], off, limit[i])
                    # no element is off by itself: a product's error is spread over a row and a column
                    worst = np.abs(got - want[i]).max()
                    assert worst <= 0.02 + ROUND[dtype][0] * np.abs(want[i]).max(), (kinds, shapes[i], worst)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_large(darb, dtype):
    """Sizes that the rules give each kind of tile, against the steps in 64 bits."""
    for rows, cols in ((1536, 4608), (2048, 2048), (4100, 1000)):
        g = torch.randn(rows, cols, device="cuda", dtype=torch.float32).to(TYPES[dtype])
        x = g.double()
        x = x / (x.norm() + 1e-7)
        x = x if rows <= cols else x.t().contiguous()
        for _ in range(5):
            a = x @ x.t()
            x = A * x + (B * a + C * (a @ a)) @ x
        x = x if rows <= cols else x.t()
        for again in range(3):
            got = darb.orthogonalize(g).double()
            off = float((got - x).norm() / x.norm())
            say(dtype, rows, cols, off)
            # fp32: 22 bits an operand, sums of up to 4608 terms, stretched by less than 3.4445 a step while
            # values are small: 2^-22 sqrt(3) 5 3.5; 16 bits: as the call's documentation has it, and its rounding
            assert off <= (2.0 ** -22 * 31 if dtype == "f32" else 3e-3 + ROUND[dtype][0])
            assert float((got - x).abs().max()) <= 40 * off * float(x.square().mean().sqrt()) + 1e-6 + \
                ROUND[dtype][0] * float(x.abs().max())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_what_it_does(darb, dtype):
    """Singular values from 0.01 of the norm up land between 0.68 and 1.21, the vectors stay."""
    r = np.random.default_rng(2)
    u, _, v = np.linalg.svd(r.normal(size=(200, 333)), full_matrices=False)
    s = np.exp(np.linspace(math.log(0.02), 0, 200))
    s = s / np.linalg.norm(s)
    G = (u * s) @ v
    got = wide(darb.orthogonalize(torch.from_numpy(G).to(TYPES[dtype]).cuda()))
    # with 3 10^-3 of the norm off, and an input rounded to its type, whose small values grow by up
    # to 3.4445^5 = 485
    inside = u.T @ got @ v.T
    kept = np.diag(inside)
    room = 3e-3 * math.sqrt(200) + 485 * ROUND[dtype][0]
    big = s > 0.01
    assert big.any() and (kept[big] > 0.68 - room).all() and (kept[big] < 1.21 + room).all()


def test_layouts(darb):
    """Batches, transposed and strided matrices, and a result in the input's own place."""
    g = torch.from_numpy(np.random.default_rng(5).normal(size=(3, 70, 130))).float().cuda()
    one = [darb.orthogonalize(x) for x in g]
    got = darb.orthogonalize(g)
    # a matrix among others is summed in other places: each is within the bound of the exact result
    assert got.shape == g.shape
    for x, a, b in zip(g, got, one):
        off = np.linalg.norm(wide(a) - wide(b))
        assert off <= 2 * (bound(wide(x), 5, 1e-7, True) + U * np.linalg.norm(wide(a)))
    turned = darb.orthogonalize(g.mT)
    assert turned.stride() == (70 * 130, 1, 130) and torch.equal(turned.mT, got)
    assert torch.equal(darb.orthogonalize(g[0].t().contiguous()), one[0].t())
    room = torch.full((3, 75, 141), 7.0, device="cuda")
    view = room[:, 2:72, 5:135]
    view.copy_(g)
    out = torch.full((3, 80, 150), 9.0, device="cuda")
    into = out[:, 1:71, 3:133]
    assert darb.orthogonalize(view, out=into) is into and torch.equal(into, got)
    into.fill_(9.0)
    assert bool((out == 9.0).all())
    same = g.clone()
    assert torch.equal(darb.orthogonalize(same, out=same), got)
    for shape in ((1, 40), (40, 1)):
        x = torch.randn(shape, device="cuda")
        assert torch.equal(darb.orthogonalize(x).t(), darb.orthogonalize(x.t()))


def test_special_matrices(darb):
    for dtype in TYPES.values():
        zero = darb.orthogonalize(torch.zeros(33, 150, dtype=dtype, device="cuda"))
        assert not zero.any()
        x = torch.randn(33, 150, device="cuda").to(dtype)
        for bad in (math.nan, math.inf):
            y = x.clone()
            y[3, 7] = bad
            assert torch.isnan(darb.orthogonalize(y)).all()
    # far from 1 in magnitude the norm is still right
    x = torch.randn(60, 100, device="cuda")
    want = darb.orthogonalize(x, eps=1e-300)
    for scale in (2.0 ** 100, 2.0 ** -100):
        assert torch.equal(darb.orthogonalize(x * scale, eps=1e-300), want)
    # columns of zeros, and one column alone
    y = torch.zeros(60, 100, device="cuda")
    y[:, 9] = x[:, 9]
    got = darb.orthogonalize(y)
    assert not got[:, :9].any() and not got[:, 10:].any()


def reference_step(p, m, g, lr, mu, nesterov, decay, scale, steps, eps):
    m = mu * m + (1 - mu) * g
    u = mu * m + (1 - mu) * g if nesterov else m
    O = exact(u, steps, eps)
    return p * (1 - lr * decay) - lr * scale * O, m, u


MODEL = [(40, 40), (96, 40), (40, 96), (1, 9), (130, 130), (7, 200)]


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype,gdtype,masters", [("f32", "f32", False), ("f32", "bf16", False), ("f16", "f32", False),
                                                  ("bf16", "bf16", True), ("f16", "f16", True), ("bf16", "bf16", False)])
def test_steps(darb, dtype, gdtype, masters, nesterov):
    r = np.random.default_rng(9)
    lr, mu, decay = 0.03, 0.9, 0.1
    start = [r.normal(size=s) * 0.1 for s in MODEL]
    params = [torch.from_numpy(p).to(TYPES[dtype]).cuda() for p in start]
    opt = darb.Muon(params, lr=lr, momentum=mu, nesterov=nesterov, weight_decay=decay, masters=masters)
    p = [wide(t) for t in (opt.masters if masters else params)]
    m = [np.zeros(s) for s in MODEL]
    limit, mlimit = [0.0] * len(MODEL), [np.zeros(s) for s in MODEL]
    full = dtype == "f32" or masters
    kept = "f32" if full else dtype
    for step in range(3):
        grads = [torch.from_numpy(matrix(*s, "flat", 50 + step) * 1e-3).to(TYPES[gdtype]).cuda() for s in MODEL]
        left_out = step == 1
        if left_out:
            grads[2] = None
        before = [params[2].clone(), opt.momenta[2].clone()]
        opt.step(grads)
        if left_out:
            assert torch.equal(params[2], before[0]) and torch.equal(opt.momenta[2], before[1])
        for i, g in enumerate(grads):
            if g is None:
                continue
            scale = math.sqrt(max(1, MODEL[i][0] / MODEL[i][1]))
            # u from the momentum as it is held, whose own error is measured apart
            mi = wide(opt.momenta[i])
            wp, wm, _ = reference_step(p[i], m[i], wide(g), lr, mu, nesterov, decay, scale, 5, 1e-7)
            mlimit[i] = mu * mlimit[i] + 4 * U * (np.abs(mu * m[i]) + np.abs((1 - mu) * wide(g)))
            check(mi, wm, mlimit[i] + 1e-300, f"momentum {i} step {step}")
            u = mu * mi + (1 - mu) * wide(g) if nesterov else mi
            O = exact(u, 5, 1e-7)
            wp = p[i] * (1 - lr * decay) - lr * scale * O
            # u is rounded to fp32, by 3 units of it at most, and stretched with everything else
            s0 = np.linalg.svd(u / np.linalg.norm(u), compute_uv=False)
            grown = 4 * U
            for _ in range(5):
                grown *= stretch(s0, u.shape[0] != u.shape[1])
                s0 = poly(s0)
            off = lr * scale * (bound(u, 5, 1e-7, full) + grown)
            step_rounding = 4 * U * (np.linalg.norm(p[i]) + np.linalg.norm(wp)) + \
                ROUND[kept][0] * np.linalg.norm(wp) + ROUND[kept][1] * math.sqrt(wp.size)
            got = wide(opt.masters[i] if masters else params[i])
            assert np.linalg.norm(got - wp) <= off + step_rounding, f"parameter {i} step {step}"
            if masters:
                assert torch.equal(params[i], opt.masters[i].to(TYPES[dtype]))
            p[i], m[i] = got, mi


def test_grad_scale_and_state(darb):
    """A loss scale is taken out, a state goes on, and a list of more matrices than go together."""
    r = np.random.default_rng(4)
    shapes = [(20 + i, 33) for i in range(61)]
    grads = [torch.from_numpy(r.normal(size=s)).float().cuda() for s in shapes]
    make = lambda **kw: darb.Muon([torch.ones(s, device="cuda") for s in shapes], lr=0.1, **kw)      # noqa: E731
    a, b = make(), make()
    a.step(grads)
    b.step([g * 1024 for g in grads], grad_scale=torch.tensor([2.0 ** -10], device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(a.params + a.momenta, b.params + b.momenta))
    c = darb.Muon([p.clone() for p in a.params], lr=0.1, state=[m.clone() for m in a.momenta])
    a.step(grads, lr=0.05)
    c.step(grads, lr=0.05)
    assert all(torch.equal(x, y) for x, y in zip(a.params, c.params))
    # one alone gives the same as among others, but for the places its sums are cut at: each is within
    # the bound of the exact step, 0.1 of the result's and two roundings of values below 1.2
    d = darb.Muon([torch.ones(shapes[60], device="cuda")], lr=0.1)
    d.step([grads[60]])
    off = np.linalg.norm(wide(d.params[0]) - wide(b.params[60]))
    assert off <= 2 * (0.1 * bound(wide(b.momenta[60]), 5, 1e-7, True) + 2 * 1.2 * U * math.sqrt(d.params[0].numel()))
    # strided gradients
    e = make()
    e.step([torch.cat([g, g], 1)[:, :g.shape[1]] for g in grads])
    assert all(torch.equal(x, y) for x, y in zip(e.params, b.params))


def test_streams_and_graphs(darb):
    from _streams import Busy, copies, same
    busy = Busy()
    g = torch.randn(2, 150, 90, device="cuda")
    want = darb.orthogonalize(g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy.queue()
    got = darb.orthogonalize(g, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    make = lambda: darb.Muon([torch.ones(150, 90, device="cuda"), torch.ones(40, 200, device="cuda")])   # noqa: E731
    grads = [g[0], torch.randn(40, 200, device="cuda")]
    plain, graphed = make(), make()
    for _ in range(5):
        plain.step(grads)
    with torch.cuda.stream(side):
        darb.orthogonalize(g)
        graphed.step(grads)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step(grads)
        out = darb.orthogonalize(g)
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), k
        darb.orthogonalize(g * 2)
    assert same(copies(graphed.params + graphed.momenta), copies(plain.params + plain.momenta))
