"""The gated recurrence against its definition in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb, say  # noqa: E402,F401
from _recurrence import backward, forward  # noqa: E402
from _train import ORDERS, TYPES, check, place, rounding, wide  # noqa: E402

pytestmark = pytest.mark.gpu

#: one element, one step, odd sizes, rows read whole through LDS (few sequences), many tiles and
#: slabs of time, more lanes than a workgroup's
SIZES = [(1, 1, 1), (5, 1, 1), (1, 9, 1), (3, 1, 7), (16, 7, 3), (3, 130, 1), (9, 300, 5), (7, 2500, 1),
         (64, 9, 20), (33, 600, 2), (130, 1100, 1), (20, 70, 33), (300, 3, 64), (2, 5000, 16)]


def data(H, T, batch, form, resets, seed, dtype, scale=1.5):
    r = np.random.default_rng(seed)
    z = r.normal(1.0, scale, (H, T * batch))
    if form == "linear":
        z = np.tanh(z)
    x = r.normal(size=z.shape)
    as_typed = lambda a: torch.from_numpy(a).to(TYPES[dtype]).double().numpy()       # noqa: E731
    h0 = r.normal(size=(H, batch)).astype(np.float32)
    starts = (r.random(T * batch) < 0.1).astype(np.uint8) if resets else None
    return as_typed(z), as_typed(x), h0, starts, r


def state(a, order):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t if order.startswith("features") else t.t().contiguous().t()


def on(a):
    return None if a is None else torch.from_numpy(a).cuda()


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("form", ["gate", "linear"])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_forward(darb, dtype, form, order):
    for n, (H, T, batch) in enumerate(SIZES):
        for resets in (False, True):
            label = f"{dtype} {form} {order} H={H} T={T} batch={batch} resets={resets}"
            say(label)
            z, x, h0, starts, _ = data(H, T, batch, form, resets, n, dtype)
            want, last, bound, lbound = forward(z, x, h0, starts, batch, form)
            h, hl = darb.gated_recurrence(place(z, order, dtype), place(x, order, dtype), batch=batch,
                                          h0=state(h0, order), resets=on(starts), form=form)
            check(wide(h), want, bound + rounding(np.abs(want) + bound, dtype), label)
            check(wide(hl), last, lbound + 2.0 ** -24 * np.abs(last), label + " last")


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("form", ["gate", "linear"])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_backward(darb, dtype, form, order):
    for n, (H, T, batch) in enumerate(SIZES):
        for resets in (False, True):
            label = f"{dtype} {form} {order} H={H} T={T} batch={batch} resets={resets}"
            say(label)
            z, x, h0, starts, r = data(H, T, batch, form, resets, 100 + n, dtype)
            h = torch.from_numpy(forward(z, x, h0, starts, batch, form)[0]).to(TYPES[dtype]).double().numpy()
            dh = torch.from_numpy(r.normal(size=z.shape)).to(TYPES[dtype]).double().numpy()
            dl = r.normal(size=h0.shape).astype(np.float32)
            dz, dx, d0, bz, bx, b0 = backward(dh, z, x, h, h0, dl, starts, batch, form)
            got = darb.gated_recurrence_grad(place(dh, order, dtype), place(z, order, dtype), place(x, order, dtype),
                                             place(h, order, dtype), batch=batch, h0=state(h0, order),
                                             resets=on(starts), dh_last=state(dl, order), form=form)
            for g, w, b, name in zip(got, (dz, dx, d0), (bz, bx, b0), ("dgate", "dx", "dh0")):
                b = b + rounding(np.abs(w) + b, dtype if name != "dh0" else "f32")
                check(wide(g), w, b, f"{label} {name}")


@pytest.mark.parametrize("H,T,batch,order", [(3, 20000, 1, "features"), (2, 9001, 3, "features"), (5, 3001, 1, "tokens"),
                                             (2, 2500, 7, "tokens"), (4, 3000, 20, "features")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sequences(darb, dtype, H, T, batch, order):
    """Time cut into slabs in every layout, a matrix of odd width, and what a replay finds in its workspace."""
    for form in ("gate", "linear"):
        z, x, h0, starts, r = data(H, T, batch, form, True, T, dtype)
        starts[:] = r.random(T * batch) < 0.002
        want, last, bound, lbound = forward(z, x, h0, starts, batch, form)
        say(dtype, H, T, batch, order, form)
        for again in range(2):
            args = dict(batch=batch, h0=state(h0, order), resets=on(starts), form=form)
            h, hl = darb.gated_recurrence(place(z, order, dtype), place(x, order, dtype), **args)
            check(wide(h), want, bound + rounding(np.abs(want) + bound, dtype), "h")
            check(wide(hl), last, lbound + 2.0 ** -24 * np.abs(last), "last")
        hr = torch.from_numpy(want).to(TYPES[dtype]).double().numpy()
        dh = torch.from_numpy(r.normal(size=z.shape)).to(TYPES[dtype]).double().numpy()
        dl = r.normal(size=h0.shape).astype(np.float32)
        dz, dx, d0, bz, bx, b0 = backward(dh, z, x, hr, h0, dl, starts, batch, form)
        got = darb.gated_recurrence_grad(place(dh, order, dtype), place(z, order, dtype), place(x, order, dtype),
                                         place(hr, order, dtype), dh_last=state(dl, order), **args)
        for g, w, b, name in zip(got, (dz, dx, d0), (bz, bx, b0), ("dgate", "dx", "dh0")):
            check(wide(g), w, b + rounding(np.abs(w) + b, dtype if name != "dh0" else "f32"), name)


def test_offsets_past_32_bits(darb):
    """Columns of one buffer 2^32 bytes and more apart."""
    far = (1 << 30) + 16                    # fp32 elements between steps
    H, T = 64, 3
    room = torch.empty((T - 1) * far + 3 * H, device="cuda")
    z, x, h = (room[k * H:].as_strided((H, T), (1, far)) for k in range(3))
    r = np.random.default_rng(0)
    a, b = r.normal(size=(2, H, T)).astype(np.float32)
    z.copy_(torch.from_numpy(a))
    x.copy_(torch.from_numpy(b))
    z0 = np.zeros((H, 1), np.float32)
    want, want_last, bound, lbound = forward(a, b, z0, None, 1, "gate")
    got, last = darb.gated_recurrence(z, x, h=h)
    assert got is h
    check(wide(h), want, bound + 2.0 ** -24 * np.abs(want), "h")
    check(wide(last), want_last, lbound + 2.0 ** -24 * np.abs(want_last), "last")
    assert torch.equal(z.cpu(), torch.from_numpy(a)) and torch.equal(x.cpu(), torch.from_numpy(b))
    dz, dx, d0, bz, bx, b0 = backward(b, a, b, wide(h), z0, z0, None, 1, "gate")
    got = darb.gated_recurrence_grad(x, z, x, h, dgate=z, dx=x)
    assert got[0] is z and got[1] is x
    for g, w, e, name in zip(got, (dz, dx, d0), (bz, bx, b0), ("dgate", "dx", "dh0")):
        check(wide(g), w, e + 2.0 ** -24 * np.abs(w), name)


@pytest.mark.parametrize("form", ["gate", "linear"])
def test_gradients_against_differences(darb, form):
    """Central differences of the definition in 64 bits: off by about the step squared."""
    H, T, batch, d = 3, 9, 2, 1e-4
    z, x, h0, starts, r = data(H, T, batch, form, True, 7, "f32", 0.7)
    wh, wl = r.normal(size=z.shape), r.normal(size=h0.shape).astype(np.float32).astype(np.float64)
    wh = torch.from_numpy(wh).float().double().numpy()

    def loss(z, x, h0):
        h, last, _, _ = forward(z, x, h0, starts, batch, form)
        return (h * wh).sum() + (last * wl).sum()
    h = forward(z, x, h0, starts, batch, form)[0]
    f = lambda a: torch.from_numpy(np.asarray(a)).float().cuda()                     # noqa: E731
    got = darb.gated_recurrence_grad(f(wh), f(z), f(x), f(h), batch=batch, h0=f(h0), resets=on(starts),
                                     dh_last=f(wl), form=form)
    args = [z, x, h0.astype(np.float64)]
    for k, g in enumerate(got):
        want = np.empty_like(args[k])
        for i in np.ndindex(want.shape):
            ends = []
            for s in (d, -d):
                moved = [a.copy() for a in args]
                moved[k][i] += s
                ends.append(loss(*moved))
            want[i] = (ends[0] - ends[1]) / (2 * d)
        # third derivatives here are below 100; h was rounded to fp32, values are below 30
        check(wide(g), want, 100 * d * d + 1e-4 * 2.0 ** -10, f"{form} {k}")


@pytest.mark.parametrize("order", ["features", "tokens"])
def test_states_and_outputs_in_place(darb, order):
    for H, T, batch in ((40, 1, 6), (7, 2500, 1), (130, 1100, 1), (64, 9, 20)):
        z, x, h0, starts, r = data(H, T, batch, "gate", True, 3, "f32")
        a, b = place(z, order, "f32"), place(x, order, "f32")
        s = state(h0, order)
        want, last = darb.gated_recurrence(a, b, batch=batch, h0=s, resets=on(starts))
        into, both = b.clone(), s.clone()
        h, hl = darb.gated_recurrence(a, into, batch=batch, h0=both, resets=on(starts), h=into, h_last=both)
        assert h is into and hl is both and torch.equal(h, want) and torch.equal(hl, last)
        into = a.clone()
        assert torch.equal(darb.gated_recurrence(into, b, batch=batch, h0=s, resets=on(starts), h=into)[0], want)
        dh, dl = place(r.normal(size=z.shape), order, "f32"), state(r.normal(size=h0.shape), order)
        want = darb.gated_recurrence_grad(dh, a, b, h, batch=batch, h0=s, resets=on(starts), dh_last=dl)
        g, za, d0 = dh.clone(), a.clone(), dl.clone()
        got = darb.gated_recurrence_grad(g, za, b, h, batch=batch, h0=s, resets=on(starts), dh_last=d0, dgate=za,
                                         dx=g, dh0=d0)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        xa = b.clone()
        got = darb.gated_recurrence_grad(dh, a, xa, h, batch=batch, h0=s, resets=on(starts), dh_last=dl, dx=xa)
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_no_states_given(darb):
    z, x, h0, _, r = data(12, 40, 4, "gate", False, 5, "f32")
    a, b = place(z, "features", "f32"), place(x, "features", "f32")
    zero = torch.zeros(12, 4, device="cuda")
    h, last = darb.gated_recurrence(a, b, batch=4)
    w, wl = darb.gated_recurrence(a, b, batch=4, h0=zero)
    assert torch.equal(h, w) and torch.equal(last, wl)
    got = darb.gated_recurrence_grad(b, a, b, h, batch=4)
    want = darb.gated_recurrence_grad(b, a, b, h, batch=4, h0=zero, dh_last=zero)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    # the linear form's gradients do not read x
    got = darb.gated_recurrence_grad(b, a, None, h, batch=4, form="linear")
    want = darb.gated_recurrence_grad(b, a, b, h, batch=4, form="linear")
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    # one state for all sequences: strides of 0 are read
    one = torch.randn(12, 1, device="cuda")
    assert torch.equal(darb.gated_recurrence(a, b, batch=4, h0=one.expand(12, 4))[0],
                       darb.gated_recurrence(a, b, batch=4, h0=one.repeat(1, 4))[0])


@pytest.mark.parametrize("order,H,T,batch", [("features", 6, 2600, 1), ("tokens", 70, 1500, 1), ("features", 4, 40, 32),
                                             ("tokens", 40, 12, 3)])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_nothing_passes_a_start(darb, order, H, T, batch, bad):
    """What stands before a restart does not reach what comes after it, in either direction."""
    z, x, h0, _, r = data(H, T, batch, "gate", False, 11, "f32")
    starts = np.zeros((T, batch), np.uint8)
    starts[T // 2] = 1
    dh = r.normal(size=z.shape)
    args = dict(batch=batch, resets=on(starts.reshape(-1)))
    put = lambda a: place(a, order, "f32")                                           # noqa: E731
    clean, last = darb.gated_recurrence(put(z), put(x), h0=state(h0, order), **args)
    xb, zb = x.copy(), z.copy()
    xb[:, :batch] = bad
    zb[:, batch:2 * batch] = np.nan
    h, hl = darb.gated_recurrence(put(zb), put(xb), h0=state(h0, order), **args)
    half = T // 2 * batch
    assert torch.equal(h[:, half:], clean[:, half:]) and torch.equal(hl, last)
    assert not torch.isfinite(h[:, batch:half]).any()
    want = darb.gated_recurrence_grad(put(dh), put(z), put(x), clean, **args)
    db = dh.copy()
    db[:, -batch:] = bad
    got = darb.gated_recurrence_grad(put(db), put(z), put(x), clean, **args)
    for p, q in zip(got[:2], want[:2]):
        assert torch.equal(p[:, :half], q[:, :half])
        assert not torch.isfinite(p[:, half:]).any()
    assert torch.equal(got[2], want[2])
    # the state before a start on the first step is not used
    starts[0] = 1
    args["resets"] = on(starts.reshape(-1))
    h, _ = darb.gated_recurrence(put(z), put(x), h0=state(h0 * np.float32(bad), order), **args)
    assert torch.isfinite(h).all()
    assert not darb.gated_recurrence_grad(put(dh), put(z), put(x), h, h0=state(h0, order), **args)[2].any()


def test_extreme_gates(darb):
    z = torch.tensor([[-np.inf, -200.0, -30.0, 0.0, -0.0, 30.0, 200.0, np.inf]], device="cuda", dtype=torch.float32)
    x, one = torch.full_like(z, 3.0), torch.ones(1, 8, device="cuda")
    h, last = darb.gated_recurrence(z, x, batch=8, h0=one)
    want, _, bound, _ = forward(z.double().cpu().numpy(), x.double().cpu().numpy(), one.cpu().numpy(), None, 8, "gate")
    check(wide(h), want, bound, "gates")
    dz, dx, d0 = darb.gated_recurrence_grad(one, z, x, h, batch=8, h0=one)
    wz, wx, w0, bz, bx, b0 = backward(np.ones((1, 8)), z.double().cpu().numpy(), 3 * np.ones((1, 8)),
                                      wide(h), np.ones((1, 8)), np.zeros((1, 8)), None, 8, "gate")
    # fp32 ends at 2^-149
    for g, w, b in ((dz, wz, bz), (dx, wx, bx), (d0, w0, b0)):
        check(wide(g), w, b + 2.0 ** -126, "gradients of gates")


def test_streams_and_graphs(darb):
    from _streams import Busy, copies, same
    busy = Busy()
    z, x, h0, starts, r = data(130, 1100, 1, "gate", True, 21, "f32")
    a, b, s = place(z, "tokens", "f32"), place(x, "tokens", "f32"), state(h0, "tokens")
    dh, sr = place(r.normal(size=z.shape), "tokens", "f32"), on(starts)

    def both(stream=None):
        h = darb.gated_recurrence(a, b, h0=s, resets=sr, stream=stream)
        return h, darb.gated_recurrence_grad(dh, a, b, h[0], h0=s, resets=sr, dh_last=s, stream=stream)
    want = copies(both())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy.queue()
    got = both(side)
    side.synchronize()
    assert same(copies(got), want)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = both()
    for k in range(3):
        for t in copies(out):
            t.zero_()
        b.mul_(1.0)
        g.replay()
        torch.cuda.synchronize()
        assert same(copies(out), want), k
        both()
    b.mul_(0.5)
    g.replay()
    assert same(copies(out), copies(both()))
