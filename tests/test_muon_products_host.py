"""The choice of fp16 products on the host: what must be refused before any GPU work."""
import ctypes

import pytest

import paper_1911_08020_amd as darb

L = darb.lib()
WS, BIG = ctypes.c_void_p(0x100000), 1 << 50


@pytest.mark.parametrize("kw", [dict(fp16_products=2), dict(fp16_products=-1), dict(reserved=1)])
def test_refuses(kw):
    t = dict(param=0x1000, grad=0x2000, momentum=0x3000, rows=10, cols=20, ld_param=20, ld_grad=20, scale=1.0, dtype=1,
             gdtype=1)
    t.update(kw)
    table = (darb._MuonTensor * 1)(darb._MuonTensor(**t))
    assert L.darb_muon_step(table, 1, 0.1, 0.9, 1, 5, 1e-7, None, WS, BIG, None) == darb.E_INVALID
    assert L.darb_muon_workspace(table, 1, ctypes.byref(ctypes.c_int64())) == darb.E_INVALID
    assert L.darb_last_error() != b""
