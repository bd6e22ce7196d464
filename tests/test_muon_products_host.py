"""The orthogonalised update on the host: the choice of fp16 products, and the size of the workspace."""
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


def need(*shapes):
    n = ctypes.c_int64()
    t = (darb._MuonTensor * len(shapes))(*(darb._MuonTensor(rows=a, cols=b) for a, b in shapes))
    assert L.darb_muon_workspace(t, len(shapes), ctypes.byref(n)) == 0
    return n.value


def buffers(rows, cols):
    """What a matrix takes: X and X^T twice, A and b A + c A A, each in two parts of 16 bits, sides padded."""
    m, n = sorted((-(-rows // 32) * 32, -(-cols // 32) * 32))
    return 16 * m * n + 8 * m * m


@pytest.mark.parametrize("shape", [(1, (1 << 20) - 1), ((1 << 20) - 1, 1), (8, 1 << 19), (33, 300_000), (4096, 9216),
                                   (8192, 8192), (100, 100)])
def test_a_group_is_bounded_by_its_padded_buffers(shape):
    """Thin matrices count with the rows that they are padded to."""
    one, head = buffers(*shape), 1 << 20    # of the call and the norms
    assert one <= need(shape) <= one + head
    most = max(one, 1 << 32) + head
    for count in (2, 28, 60):
        assert need(*[shape] * count) <= most
    # as many as fit go together
    assert need(*[shape] * 28) >= min(28, max(1, (1 << 32) // one)) * one
    assert need(*[shape] * 5 + [(64, 64)] * 3) <= most
