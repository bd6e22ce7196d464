"""The AdamW step: bit for bit the documented sequence of correctly rounded fp32 operations (and
8-bit codes), and within a few roundings of the formula in 64 bits."""
import math

import numpy as np
import pytest

from tests import _adamw as ref
from tests._gpu import darb, say, torch  # noqa: F401
from tests._train import TYPES, place, wide  # noqa: F401

pytestmark = pytest.mark.gpu
f32 = np.float32
HYPER = dict(lr=2e-3, betas=(0.9, 0.999), eps=1e-8)


def back(t):
    torch.cuda.synchronize()
    return t.float().cpu().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def tensors(rng, sizes, dtype, spread=1.0):
    return [torch.from_numpy((rng.standard_normal(n) * spread).astype(f32)).to(TYPES[dtype]).cuda() for n in sizes]


SIZES = [1, 3, 255, 256, 257, 1000, 4095, 4096, 4097, 70001, 0, 12]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,gdtype,masters", [("f32", "f32", None), ("f32", "bf16", None), ("f16", "f16", None),
                                                  ("f16", "f32", True), ("bf16", "bf16", True), ("bf16", "f32", None)])
def test_adamw_steps_bit_for_bit(darb, bits, dtype, gdtype, masters):  # noqa: F811
    rng = np.random.default_rng(bits)
    params = tensors(rng, SIZES, dtype, 0.1)
    decay = [0.0 if n < 300 else 0.03 for n in SIZES]
    opt = darb.AdamW(params, weight_decay=decay, state_bits=bits, masters=masters, seed=77, **HYPER)
    state = []
    for p, k in zip(params, opt.masters):
        x = back(p if k is None else k)
        state.append([x, np.zeros(len(x), f32), np.zeros(len(x), f32)])
    for t in range(1, 5):
        grads = tensors(rng, SIZES, gdtype, 10.0 ** -t)
        grads[2] = None if t == 2 else grads[2]
        scale = torch.tensor([0.5], device="cuda") if t == 3 else None
        say(f"adamw {bits} {dtype} {gdtype} step {t}")
        opt.step(grads, grad_scale=scale)
        for i, (s, g) in enumerate(zip(state, grads)):
            if g is None:
                continue
            if opt.masters[i] is None:
                s[0] = torch.from_numpy(s[0]).to(TYPES[dtype]).float().numpy()
            s[:] = ref.step(s[0], back(g), s[1], s[2], t, decay=decay[i], scale=0.5 if t == 3 else 1.0, **HYPER)
            if bits == 8:
                rm, rv = ref.random_of(len(s[0]), ref.seed_of(77, t, i))
                cm, sm = ref.encode(s[1], rm, True)
                cv, sv = ref.encode(s[2], rv, False)
                got = [x.cpu().numpy() for x in opt.state_tensors[i]]
                assert same(got[2], sm) and same(got[3], sv), i
                assert same(got[0], cm) and same(got[1], cv), i
                s[1], s[2] = ref.decode(cm, sm, True), ref.decode(cv, sv, False)
            stored = torch.from_numpy(s[0]).to(TYPES[dtype]).float().numpy()
            assert same(back(params[i]), stored), i
            if opt.masters[i] is not None:
                assert same(back(opt.masters[i]), s[0]), i
        m, v = opt.moments()
        for i, s in enumerate(state):
            assert same(back(m[i]), s[1]) and same(back(v[i]), s[2]), i
    assert opt.steps == 4


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_against_64_bits(darb, bits):  # noqa: F811
    # one step from given moments: four roundings of m, v and their quotient, two of p
    rng = np.random.default_rng(3)
    n, t0 = 5000, 20
    p, g = rng.standard_normal(n).astype(f32), rng.standard_normal(n).astype(f32)
    m, v = (rng.standard_normal(n) * 0.1).astype(f32), (rng.random(n) + 0.01).astype(f32)
    d = lambda a: torch.from_numpy(a).cuda()                                     # noqa: E731
    if bits == 8:
        zero = np.zeros(n, np.int64)
        (cm, sm), (cv, sv) = ref.encode(m, zero, True), ref.encode(v, zero, False)
        m, v = ref.decode(cm, sm, True), ref.decode(cv, sv, False)
        state = [(d(cm), d(cv), d(sm), d(sv))]
    else:
        state = [(d(m), d(v))]
    pd = d(p)
    darb.AdamW([pd], weight_decay=0.1, state_bits=bits, state=state, steps=t0, **HYPER).step([d(g)])
    p, g, m, v = (a.astype(np.float64) for a in (p, g, m, v))
    m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g * g
    t = t0 + 1
    step = HYPER["lr"] * (m / (1 - 0.9 ** t)) / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
    want = p * (1 - HYPER["lr"] * 0.1) - step
    scale = np.abs(p) + HYPER["lr"] * (0.9 * np.abs(m) + 0.1 * np.abs(g)) * 10 / np.sqrt(v)
    assert (np.abs(wide(pd) - want) <= 2.0 ** -21 * scale).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_views_at_odd_addresses(darb, bits):  # noqa: F811
    # tensors cut out of one buffer at odd elements, beside each other: the same bits, and
    # nothing beside them is touched
    rng = np.random.default_rng(5)
    sizes = [257, 5, 1030, 4099]
    own = tensors(rng, sizes, "f16")
    grads = tensors(rng, sizes, "f16")
    cut = lambda flat: [flat[a:a + n] for a, n in zip(np.cumsum([1] + [n + 3 for n in sizes[:-1]]), sizes)]  # noqa: E731
    flat, gflat = (torch.full((sum(sizes) + 3 * len(sizes) + 8,), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    for v, t in zip(cut(flat), own):
        v.copy_(t)
    for v, t in zip(cut(gflat), grads):
        v.copy_(t)
    a = darb.AdamW(own, state_bits=bits, masters=True)
    b = darb.AdamW(cut(flat), state_bits=bits, masters=True)
    for _ in range(2):
        a.step(grads)
        b.step(cut(gflat))
    assert all(torch.equal(x, y) for x, y in zip(own, cut(flat)))
    assert all(torch.equal(x, y) for s, u in zip(a.state_tensors, b.state_tensors) for x, y in zip(s, u))
    mask = torch.ones_like(flat, dtype=torch.bool)
    for v in cut(mask):
        v.fill_(False)
    assert bool((flat[mask] == 9.0).all())


def test_adamw_more_tensors_than_one_launch_takes(darb):  # noqa: F811
    rng = np.random.default_rng(6)
    sizes = [int(n) for n in rng.integers(1, 600, 1000)]
    params, grads = tensors(rng, sizes, "f32"), tensors(rng, sizes, "f32")
    before = [back(p) for p in params]
    opt = darb.AdamW(params, weight_decay=0.01, state_bits=8, **HYPER)
    opt.step(grads)
    m, v = opt.moments()
    for i in range(0, len(sizes), 37):
        p, _, _ = ref.step(before[i], back(grads[i]), np.zeros(sizes[i], f32), np.zeros(sizes[i], f32), 1, decay=0.01, **HYPER)
        assert same(back(params[i]), p)
    i = len(sizes) - 1
    _, wm, wv = ref.step(before[i], back(grads[i]), np.zeros(sizes[i], f32), np.zeros(sizes[i], f32), 1, decay=0.01, **HYPER)
    rm, rv = ref.random_of(sizes[i], ref.seed_of(0, 1, i))
    assert same(back(m[i]), ref.decode(*ref.encode(wm, rm, True), True))
    assert same(back(v[i]), ref.decode(*ref.encode(wv, rv, False), False))


def test_adamw_infinite_gradients_stay_in_their_block(darb):  # noqa: F811
    g = torch.ones(1000, device="cuda")
    g[300] = math.inf
    p = torch.zeros(1000, device="cuda")
    opt = darb.AdamW([p], state_bits=8, **HYPER)
    opt.step([g])
    m, v = (back(x[0]) for x in opt.moments())
    block = np.zeros(1000, bool)
    block[256:512] = True
    assert np.array_equal(np.isnan(m), block) and np.array_equal(np.isnan(v), block)
    assert np.isfinite(back(p)[~block]).all()


def test_adamw_resumes(darb):  # noqa: F811
    # steps, states and seeds carried over: the same bits as one run
    rng = np.random.default_rng(7)
    sizes = [700, 40]
    grads = [tensors(rng, sizes, "f32") for _ in range(4)]
    start = tensors(rng, sizes, "bf16")
    one = [p.clone() for p in start]
    a = darb.AdamW(one, state_bits=8, masters=True, seed=5)
    for g in grads:
        a.step(g)
    two = [p.clone() for p in start]
    b = darb.AdamW(two, state_bits=8, masters=True, seed=5)
    for g in grads[:2]:
        b.step(g)
    c = darb.AdamW(two, state_bits=8, masters=b.masters, state=b.state_tensors, steps=b.steps, seed=5)
    for g in grads[2:]:
        c.step(g)
    assert all(torch.equal(x, y) for x, y in zip(one, two)) and c.steps == 4
    assert all(torch.equal(x, y) for s, u in zip(a.state_tensors, c.state_tensors) for x, y in zip(s, u))


def test_adamw_stream_and_graph(darb):  # noqa: F811
    # captured, a step replays with the gradients that then lie at the same addresses
    p, g = torch.ones(5000, device="cuda"), torch.zeros(5000, device="cuda")
    q = p.clone()
    a, b = darb.AdamW([p], **HYPER), darb.AdamW([q], **HYPER)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        a.step([g])
    for k in range(3):
        g.copy_(torch.randn(5000, device="cuda"))
        graph.replay()
        b.steps = 0                                  # the captured step's number
        b.step([g])
        torch.cuda.synchronize()
        assert torch.equal(p, q), k


@pytest.mark.parametrize("bad,err", [
    (lambda d, p: d.AdamW([]), ValueError),
    (lambda d, p: d.AdamW([p.cpu()]), ValueError),
    (lambda d, p: d.AdamW([p.double()]), TypeError),
    (lambda d, p: d.AdamW([p.view(4, 5).t()]), ValueError),
    (lambda d, p: d.AdamW([p], state_bits=16), ValueError),
    (lambda d, p: d.AdamW([p], weight_decay=[0.1, 0.1]), ValueError),
    (lambda d, p: d.AdamW([p], weight_decay=-0.1), "DarbError"),
    (lambda d, p: d.AdamW([p], state=[(p, p[:3])]), ValueError),
    (lambda d, p: d.AdamW([p], state=[(p.half(), p)]), TypeError),
    (lambda d, p: d.AdamW([p], masters=[p.half()]), TypeError),
    (lambda d, p: d.AdamW([p]).step([]), ValueError),
    (lambda d, p: d.AdamW([p]).step([p[:3]]), ValueError),
    (lambda d, p: d.AdamW([p]).step([p.cpu()]), ValueError),
    (lambda d, p: d.AdamW([p]).step([p.int()]), TypeError),
    (lambda d, p: d.AdamW([p], lr=-1.0).step([p]), "DarbError"),
    (lambda d, p: d.AdamW([p], betas=(0.9, 1.0)).step([p]), "DarbError"),
    (lambda d, p: d.AdamW([p], eps=float("nan")).step([p]), "DarbError"),
    (lambda d, p: d.AdamW([p]).step([p], grad_scale=p.half()), TypeError),
    (lambda d, p: d.AdamW([p]).moments(out=([p[:3]], [p])), ValueError)])
def test_adamw_refusals(darb, bad, err):  # noqa: F811
    p = torch.zeros(20, device="cuda")
    with pytest.raises(darb.DarbError if err == "DarbError" else err):
        bad(darb, p)
    assert bool((p == 0).all())
