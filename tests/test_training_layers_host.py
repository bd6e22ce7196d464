"""The recurrence, the losses and the orthogonalised update on the host: what must be refused before any
GPU work."""
import ctypes
import math

import pytest

import paper_1911_08020_amd as darb

L = darb.lib()
P = ctypes.c_void_p
BUF, WS = P(0x1000), P(0x100000)
BIG = 1 << 50
M = darb._Matrix


def ref(m):
    return None if m is None else ctypes.byref(m)


def recurrence(dtype=0, form=0, H=10, T=3, batch=4, gate=M(0x1000, 12, 1), x=M(0x2000, 12, 1), resets=None,
               h0=M(0x3000, 4, 1), h=M(0x4000, 12, 1), last=M(0x5000, 4, 1), ws=WS, n=BIG):
    return L.darb_gated_recurrence(dtype, form, H, T, batch, ref(gate), ref(x), resets, ref(h0), ref(h), ref(last), ws, n,
                                   None)


def recurrence_grad(dtype=0, form=0, H=10, T=3, batch=4, dh=M(0x1000, 12, 1), gate=M(0x2000, 12, 1), x=M(0x3000, 12, 1),
                    h=M(0x4000, 12, 1), h0=None, dl=None, dz=M(0x5000, 12, 1), dx=M(0x6000, 12, 1), d0=None, ws=WS, n=BIG):
    return L.darb_gated_recurrence_grad(dtype, form, H, T, batch, ref(dh), ref(gate), ref(x), ref(h), None, ref(h0),
                                        ref(dl), ref(dz), ref(dx), ref(d0), ws, n, None)


SIZES = [(dict(dtype=3), darb.E_DTYPE), (dict(dtype=-1), darb.E_DTYPE), (dict(form=2), darb.E_INVALID),
         (dict(form=-1), darb.E_INVALID), (dict(H=0), darb.E_INVALID), (dict(T=0), darb.E_INVALID),
         (dict(batch=0), darb.E_INVALID), (dict(H=1 << 31), darb.E_INVALID), (dict(T=1 << 30), darb.E_INVALID),
         (dict(T=1 << 62, batch=4), darb.E_INVALID), (dict(batch=-4, T=-3), darb.E_INVALID)]


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(gate=None), darb.E_INVALID), (dict(x=None), darb.E_INVALID), (dict(h=None), darb.E_INVALID),
    (dict(x=M(None, 12, 1)), darb.E_INVALID), (dict(gate=M(0x1002, 12, 1)), darb.E_INVALID),
    (dict(gate=M(0x1000, 11, 1)), darb.E_INVALID), (dict(gate=M(0x1000, 1, 10)), darb.E_INVALID),
    (dict(h=M(0x1000, 24, 2)), darb.E_INVALID), (dict(h=M(0x1000, 0, 1)), darb.E_INVALID),
    (dict(h0=M(0x3001, 4, 1)), darb.E_INVALID), (dict(h0=M(0x3000, -4, 1)), darb.E_INVALID),
    (dict(last=M(0x3000, 0, 1)), darb.E_INVALID), (dict(last=M(0x3000, 8, 2)), darb.E_INVALID)])
def test_recurrence_refuses(kw, code):
    assert recurrence(**kw) == code
    assert L.darb_last_error() != b""


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(dh=None), darb.E_INVALID), (dict(x=None), darb.E_INVALID), (dict(h=None), darb.E_INVALID),
    (dict(dz=None), darb.E_INVALID), (dict(dx=None), darb.E_INVALID), (dict(dh=M(0x1000, 1, 10)), darb.E_INVALID),
    (dict(dz=M(0x4000, 12, 1)), darb.E_INVALID), (dict(dx=M(0x4000, 12, 1)), darb.E_INVALID),
    (dict(dx=M(0x5000, 12, 1)), darb.E_INVALID), (dict(dl=M(0x3001, 4, 1)), darb.E_INVALID),
    (dict(h0=M(0x3002, 4, 1)), darb.E_INVALID), (dict(d0=M(0x3000, 0, 0)), darb.E_INVALID)])
def test_recurrence_grad_refuses(kw, code):
    assert recurrence_grad(**kw) == code


def test_recurrence_workspace():
    n = ctypes.c_int64()
    call = L.darb_gated_recurrence_workspace
    assert call(0, 0, 1024, 1, 32, ctypes.byref(n)) == 0 and n.value == 0
    assert call(1, 1, 1024, 65536, 1, ctypes.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    assert recurrence(H=16, T=65536, batch=1, gate=M(0x1000, 65536, 1), x=M(0x1000, 65536, 1), h=M(0x1000, 65536, 1),
                      h0=None, last=None, ws=None) == darb.E_INVALID
    assert recurrence(H=16, T=65536, batch=1, gate=M(0x1000, 65536, 1), x=M(0x1000, 65536, 1), h=M(0x1000, 65536, 1),
                      h0=None, last=None, n=16) == darb.E_WORKSPACE
    assert call(0, 0, 1024, 1, 32, None) == darb.E_INVALID and call(7, 0, 4, 1, 1, ctypes.byref(n)) == darb.E_DTYPE
    assert call(0, 0, 0, 1, 1, ctypes.byref(n)) == darb.E_INVALID


def policy(B=10, lp=BUF, old=BUF, adv=BUF, w=None, rf=None, ent=None, low=0.2, high=0.2, kl=0.0, ec=0.0, stats=BUF,
           g=P(0x2000), ge=None, ws=WS, n=BIG):
    return L.darb_policy_loss(B, lp, old, adv, w, rf, ent, low, high, kl, ec, stats, g, ge, ws, n, None)


@pytest.mark.parametrize("kw", [
    dict(B=0), dict(B=1 << 31), dict(lp=None), dict(old=None), dict(adv=None), dict(stats=None), dict(g=None),
    dict(low=-0.1), dict(high=-1e-9), dict(low=math.nan), dict(high=math.inf), dict(kl=0.1), dict(kl=-0.1, rf=BUF),
    dict(kl=math.nan, rf=BUF), dict(ec=0.1), dict(ent=BUF), dict(ge=BUF), dict(ec=math.inf, ent=BUF, ge=P(0x3000)),
    dict(ent=BUF, ge=P(0x2000)), dict(lp=P(0x1002)), dict(w=P(0x1001)), dict(B=1 << 20, ws=None),
    dict(B=1 << 20, ws=P(0x1010))])
def test_policy_refuses(kw):
    assert policy(**kw) == darb.E_INVALID


def test_policy_workspace():
    n = ctypes.c_int64()
    assert L.darb_policy_loss_workspace(700, ctypes.byref(n)) == 0 and n.value == 0
    assert L.darb_policy_loss_workspace(1 << 20, ctypes.byref(n)) == 0 and n.value > 0
    assert policy(B=1 << 20, n=n.value - 1) == darb.E_WORKSPACE
    assert L.darb_policy_loss_workspace(0, ctypes.byref(n)) == darb.E_INVALID
    assert L.darb_policy_loss_workspace(1, None) == darb.E_INVALID


@pytest.mark.parametrize("kw", [
    dict(pairs=0), dict(pairs=1 << 30), dict(B=0), dict(B=1 << 31), dict(B=13), dict(lp=None), dict(loss=None),
    dict(margin=None), dict(g=None), dict(beta=-0.1), dict(beta=math.inf), dict(beta=math.nan), dict(e=-0.1), dict(e=1.0),
    dict(e=math.nan), dict(lp=P(0x1001)), dict(starts=P(0x1004)), dict(w=P(0x1002))])
def test_preference_refuses(kw):
    a = dict(pairs=2, B=12, lp=BUF, rf=None, starts=None, w=None, beta=0.1, e=0.0, loss=BUF, margin=BUF, g=P(0x2000))
    a.update(kw)
    assert L.darb_preference_loss(a["pairs"], a["B"], a["lp"], a["rf"], a["starts"], a["w"], a["beta"], a["e"], a["loss"],
                                  a["margin"], a["g"], None) == darb.E_INVALID


def entry(**kw):
    t = dict(param=0x1000, master=None, grad=0x2000, momentum=0x3000, rows=10, cols=20, ld_param=20, ld_grad=20,
             scale=1.0, decay=0.0, dtype=0, gdtype=0)
    t.update(kw)
    return darb._MuonTensor(**t)


BAD = [(dict(rows=0), darb.E_INVALID), (dict(cols=1 << 20), darb.E_INVALID), (dict(rows=-1), darb.E_INVALID),
       (dict(dtype=3), darb.E_DTYPE), (dict(gdtype=9), darb.E_DTYPE), (dict(param=None), darb.E_INVALID),
       (dict(ld_param=19), darb.E_INVALID), (dict(ld_grad=19), darb.E_INVALID), (dict(param=0x1002), darb.E_INVALID),
       (dict(grad=0x2001), darb.E_INVALID)]


@pytest.mark.parametrize("kw,code", BAD + [
    (dict(momentum=None), darb.E_INVALID), (dict(momentum=0x3002), darb.E_INVALID), (dict(master=0x3001), darb.E_INVALID),
    (dict(scale=math.nan), darb.E_INVALID), (dict(decay=-1.0), darb.E_INVALID), (dict(decay=math.inf), darb.E_INVALID)])
def test_muon_refuses_tensors(kw, code):
    t = (darb._MuonTensor * 2)(entry(), entry(**kw))
    assert L.darb_muon_step(t, 2, 0.1, 0.9, 1, 5, 1e-7, None, WS, BIG, None) == code


@pytest.mark.parametrize("kw,code", BAD + [(dict(grad=None), darb.E_INVALID)])
def test_orthogonalize_refuses_tensors(kw, code):
    t = (darb._MuonTensor * 2)(entry(momentum=None), entry(momentum=None, **kw))
    assert L.darb_orthogonalize(t, 2, 5, 1e-7, WS, BIG, None) == code


def test_muon_refuses():
    t = (darb._MuonTensor * 1)(entry())

    def step(t=t, count=1, lr=0.1, mu=0.9, steps=5, eps=1e-7, gs=None, ws=WS, n=BIG):
        return L.darb_muon_step(t, count, lr, mu, 1, steps, eps, gs, ws, n, None)
    for kw in (dict(t=None), dict(count=0), dict(lr=-1.0), dict(lr=math.nan), dict(mu=1.0), dict(mu=-0.1), dict(steps=0),
               dict(steps=17), dict(eps=0.0), dict(eps=math.inf), dict(gs=P(0x1001)), dict(ws=None), dict(ws=P(0x1010))):
        assert step(**kw) == darb.E_INVALID, kw
    assert step(n=64) == darb.E_WORKSPACE
    n = ctypes.c_int64()
    assert L.darb_muon_workspace(t, 1, ctypes.byref(n)) == 0 and n.value % 256 == 0 and step(n=n.value - 1) == darb.E_WORKSPACE
    assert L.darb_muon_workspace(None, 1, ctypes.byref(n)) == darb.E_INVALID
    assert L.darb_muon_workspace(t, 1, None) == darb.E_INVALID
    assert L.darb_orthogonalize(t, 1, 0, 1e-7, WS, BIG, None) == darb.E_INVALID


def test_muon_workspace_is_that_of_the_largest_group():
    def need(*shapes, **kw):
        n = ctypes.c_int64()
        t = (darb._MuonTensor * len(shapes))(*(entry(rows=a, cols=b, ld_param=b, ld_grad=b, **kw) for a, b in shapes))
        assert L.darb_muon_workspace(t, len(shapes), ctypes.byref(n)) == 0
        return n.value
    one = need((1000, 1000))
    assert need((1000, 1000), (1000, 1000)) > 1.5 * one
    assert need(*[(1000, 1000)] * 200) <= 30 * one
    # tensors past 2^28 elements go one by one
    assert need((1 << 15, 1 << 14), (1 << 15, 1 << 14)) == need((1 << 15, 1 << 14))
    # a momentum's workspace does not depend on which gradients there are
    assert need((1000, 1000), (64, 64), grad=None) == need((1000, 1000), (64, 64))


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 6)
    v = torch.zeros(6)
    for call in (lambda: darb.gated_recurrence(x, x), lambda: darb.gated_recurrence_grad(x, x, x, x),
                 lambda: darb.policy_loss(v, v, v), lambda: darb.preference_loss(v, batch=2),
                 lambda: darb.orthogonalize(x), lambda: darb.Muon([x]), lambda: darb.Muon([])):
        with pytest.raises(ValueError):
            call()
