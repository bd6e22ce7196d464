"""The evaluation and retraining calls on the host: what must be refused before any GPU work."""
import ctypes
import math

import numpy as np
import pytest

import paper_1911_08020_amd as darb

L = darb.lib()
P = ctypes.c_void_p
BUF, WS = P(0x1000), P(0x100000)
BIG = 1 << 40


def logprobs(zdtype=0, V=10, B=4, z=BUF, fs=4, bs=1, t=None, top=2, lp=BUF, h=BUF, lse=BUF, tl=BUF, ti=BUF, ws=WS,
             n=BIG):
    return L.darb_token_logprobs(zdtype, V, B, z, fs, bs, t, top, lp, h, lse, tl, ti, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(zdtype=3), darb.E_DTYPE), (dict(zdtype=-1), darb.E_DTYPE), (dict(V=0), darb.E_INVALID),
    (dict(V=1 << 31), darb.E_INVALID), (dict(B=0), darb.E_INVALID), (dict(B=1 << 31), darb.E_INVALID),
    (dict(z=None), darb.E_INVALID), (dict(lp=None), darb.E_INVALID), (dict(lse=None), darb.E_INVALID),
    (dict(tl=None), darb.E_INVALID), (dict(ti=None), darb.E_INVALID), (dict(top=-1), darb.E_INVALID),
    (dict(top=11), darb.E_INVALID), (dict(V=100, top=65), darb.E_INVALID), (dict(z=P(0x1002)), darb.E_INVALID),
    (dict(t=P(0x1004)), darb.E_INVALID), (dict(fs=3), darb.E_INVALID), (dict(fs=2, bs=2), darb.E_INVALID),
    (dict(fs=1, bs=9), darb.E_INVALID), (dict(bs=0), darb.E_INVALID), (dict(ws=None), darb.E_INVALID),
    (dict(ws=P(0x1010)), darb.E_INVALID), (dict(n=16), darb.E_WORKSPACE)])
def test_logprobs_refuses(kw, code):
    assert logprobs(**kw) == code
    assert L.darb_last_error() != b""


def test_logprobs_workspace():
    n, plain = ctypes.c_int64(), ctypes.c_int64()

    def ws(out, zdtype=0, V=10000, B=700, fs=700, bs=1, top=20):
        return L.darb_token_logprobs_workspace(zdtype, V, B, fs, bs, top, out)
    assert ws(ctypes.byref(n)) == 0 and n.value % 256 == 0 and n.value > 0
    assert ws(ctypes.byref(plain), top=0) == 0 and 0 < plain.value < n.value
    assert ws(ctypes.byref(n), fs=1, bs=10000) == 0 and n.value == 0         # rows finished where they are read
    assert ws(ctypes.byref(n), V=1 << 24, B=1, fs=1, bs=1) == 0 and n.value > 0
    assert ws(None) == darb.E_INVALID and ws(ctypes.byref(n), V=0) == darb.E_INVALID
    assert ws(ctypes.byref(n), V=10, top=11) == darb.E_INVALID and ws(ctypes.byref(n), zdtype=5) == darb.E_DTYPE
    assert ws(ctypes.byref(n), fs=3, bs=3) == darb.E_INVALID


def test_logprobs_grad_refuses():
    def grad(zdtype=0, V=10, B=4, z=BUF, fs=4, bs=1, lse=BUF, g=BUF, h=None, gh=None, dz=BUF, dfs=4, dbs=1):
        return L.darb_token_logprobs_grad(zdtype, V, B, z, fs, bs, None, lse, g, h, gh, dz, dfs, dbs, None)
    for kw, code in [(dict(zdtype=7), darb.E_DTYPE), (dict(lse=None), darb.E_INVALID),
                     (dict(dz=None), darb.E_INVALID), (dict(g=None), darb.E_INVALID),
                     (dict(h=BUF), darb.E_INVALID), (dict(gh=BUF), darb.E_INVALID),
                     (dict(dfs=1, dbs=10), darb.E_INVALID), (dict(dfs=3), darb.E_INVALID),
                     (dict(V=0), darb.E_INVALID)]:
        assert grad(**kw) == code, kw


def test_layer_norm_refuses():
    def norm(xd=0, wd=0, H=10, B=4, x=BUF, fs=4, bs=1, w=None, b=None, eps=1e-5, y=BUF, yfs=4, ybs=1):
        return L.darb_layer_norm(xd, wd, H, B, x, fs, bs, w, b, eps, y, yfs, ybs, None, None, None)
    for kw, code in [(dict(xd=5), darb.E_DTYPE), (dict(wd=1), darb.E_DTYPE), (dict(xd=1, wd=2), darb.E_DTYPE),
                     (dict(H=0), darb.E_INVALID), (dict(B=-1), darb.E_INVALID), (dict(x=None), darb.E_INVALID),
                     (dict(y=None), darb.E_INVALID), (dict(eps=-1e-9), darb.E_INVALID),
                     (dict(eps=math.inf), darb.E_INVALID), (dict(yfs=1, ybs=10), darb.E_INVALID),
                     (dict(w=P(0x1001)), darb.E_INVALID), (dict(x=P(0x1002)), darb.E_INVALID)]:
        assert norm(**kw) == code, kw

    def grad(xd=0, wd=0, H=10, B=4, dy=BUF, x=BUF, mean=BUF, rstd=BUF, dx=BUF, dw=BUF, db=BUF, dfs=4, dbs=1, ws=WS,
             n=BIG):
        return L.darb_layer_norm_grad(xd, wd, H, B, dy, 4, 1, x, 4, 1, mean, rstd, None, dx, dfs, dbs, dw, db, ws,
                                      n, None)
    for kw, code in [(dict(xd=9), darb.E_DTYPE), (dict(wd=2), darb.E_DTYPE), (dict(dy=None), darb.E_INVALID),
                     (dict(mean=None), darb.E_INVALID), (dict(dx=None, dw=None, db=None), darb.E_INVALID),
                     (dict(dfs=1, dbs=10), darb.E_INVALID), (dict(ws=None), darb.E_INVALID),
                     (dict(ws=P(0x1080)), darb.E_INVALID), (dict(n=100), darb.E_WORKSPACE)]:
        assert grad(**kw) == code, kw
    n = ctypes.c_int64()
    assert L.darb_layer_norm_workspace(1024, 32, ctypes.byref(n)) == 0 and n.value > 0
    assert L.darb_layer_norm_workspace(0, 32, ctypes.byref(n)) == darb.E_INVALID


def test_transpose_and_grad_refuse():
    p = darb.Plan(4, 64, np.full(4, 0.25), 0.25, 0, 1, 16)
    n = ctypes.c_int64()
    assert L.darb_transpose_bytes(p.handle, ctypes.byref(n)) == 0 and n.value > 8 * p.nnz
    assert L.darb_transpose_bytes(None, ctypes.byref(n)) == darb.E_INVALID
    assert L.darb_transpose(p.handle, BUF, WS, BIG, None) == darb.E_NOT_UPLOADED
    assert L.darb_spmm_grad(p.handle, WS, 0, BUF, 0, 4, BUF, 4, BUF, 4, BUF, BUF, 4, WS, BIG,
                            None) == darb.E_NOT_UPLOADED
    assert L.darb_spmm_grad(None, WS, 0, BUF, 0, 4, BUF, 4, BUF, 4, BUF, BUF, 4, WS, BIG, None) == darb.E_INVALID
    assert L.darb_spmm_grad_workspace(p.handle, 4, ctypes.byref(n)) == 0 and n.value == 0
    assert L.darb_spmm_grad_workspace(p.handle, 1 << 20, ctypes.byref(n)) == 0 and 0 < n.value <= 72 * p.nnz + 4096 * p.M + 768
    assert L.darb_spmm_grad_workspace(p.handle, 0, ctypes.byref(n)) == darb.E_INVALID
    # fewer than 2^31 weights: 2^25 rows of 64
    big = darb.Plan(1 << 25, 64, np.full(1 << 25, 1.0), 1.0, 0, 1, 1)
    assert L.darb_transpose_bytes(big.handle, ctypes.byref(n)) == darb.E_INVALID


def _tensor(**kw):
    t = dict(param=0x1000, master=None, m=0x1000, v=0x1000, m_scale=0x1000, v_scale=0x1000, n=10, decay=0.0,
             dtype=0, reserved=0)
    t.update(kw)
    return darb._AdamTensor(**t)


def test_adamw_refuses():
    h = ctypes.c_void_p(1)

    def create(t, count=1, bits=8, ws=WS, n=BIG):
        return L.darb_adamw_create(ctypes.byref(t) if t else None, count, bits, ws, n, None, ctypes.byref(h))
    for t, code in [(_tensor(dtype=3), darb.E_DTYPE), (_tensor(n=-1), darb.E_INVALID),
                    (_tensor(n=1 << 39), darb.E_INVALID), (_tensor(decay=-1.0), darb.E_INVALID),
                    (_tensor(decay=math.nan), darb.E_INVALID), (_tensor(param=None), darb.E_INVALID),
                    (_tensor(m=None), darb.E_INVALID), (_tensor(v_scale=None), darb.E_INVALID),
                    (_tensor(param=0x1002), darb.E_INVALID), (_tensor(master=0x1002), darb.E_INVALID),
                    (None, darb.E_INVALID)]:
        assert create(t) == code
        assert h.value is None
    assert create(_tensor(m=0x1001), bits=32) == darb.E_INVALID
    assert create(_tensor(), bits=16) == darb.E_INVALID and create(_tensor(), count=0) == darb.E_INVALID
    assert create(_tensor(), ws=None) == darb.E_INVALID and create(_tensor(), ws=P(0x1010)) == darb.E_INVALID
    assert create(_tensor(), n=64) == darb.E_WORKSPACE
    n = ctypes.c_int64()
    t = _tensor()
    assert L.darb_adamw_workspace(ctypes.byref(t), 1, ctypes.byref(n)) == 0 and n.value >= 512
    assert L.darb_adamw_workspace(None, 1, ctypes.byref(n)) == darb.E_INVALID
    g = (ctypes.c_void_p * 1)(0x1000)
    ty = (ctypes.c_int * 1)(0)
    assert L.darb_adamw_step(None, g, ty, 1, 0.1, 0.9, 0.999, 1e-8, 1, None, 0, None) == darb.E_INVALID
    assert L.darb_adamw_moments(None, None, None, 1, None) == darb.E_INVALID
    L.darb_adamw_destroy(None)                       # ignored


def test_old_calls_do_not_take_bf16():
    n = ctypes.c_int64()
    assert L.darb_prune_workspace(64, 300, darb.BF16, ctypes.byref(n)) == darb.E_DTYPE


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 5)
    for call in (lambda: darb.token_logprobs(x), lambda: darb.layer_norm(x), lambda: darb.AdamW([x]),
                 lambda: darb.layer_norm_grad(x, x, x[0], x[0])):
        with pytest.raises(ValueError):
            call()
