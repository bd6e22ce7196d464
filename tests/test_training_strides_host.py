"""Strides that no operand may have, where one axis has a single element and the other's stride is
the only one in use: refused before any GPU work."""
import ctypes

import pytest

import paper_1911_08020_amd as darb

L = darb.lib()
P = ctypes.c_void_p
BUF, WS = P(0x1000), P(0x100000)
BIG = 1 << 40
#: (F, B, the good strides, index of the stride in use)
ONE = [(10, 1, (1, 1), 0), (1, 10, (1, 1), 1)]


def bad(good, at, value):
    s = list(good)
    s[at] = value
    return s


@pytest.mark.parametrize("F,B,good,at", ONE)
def test_workspace_takes_zero_but_nothing_below(F, B, good, at):
    n = ctypes.c_int64()

    def query(strides):
        return L.darb_token_logprobs_workspace(0, F, B, *strides, 0, ctypes.byref(n))
    assert query(good) == 0 and query(bad(good, at, 7)) == 0 and query(bad(good, at, 0)) == 0
    assert query(bad(good, 1 - at, -3)) == 0                 # not in use
    assert query(bad(good, at, -1)) == darb.E_INVALID


@pytest.mark.parametrize("F,B,good,at", ONE)
def test_written_operands_need_a_stride(F, B, good, at):
    for value in (0, -1):
        s = bad(good, at, value)
        assert L.darb_token_logprobs_grad(0, F, B, BUF, *good, None, BUF, BUF, None, None, BUF, *s,
                                          None) == darb.E_INVALID
        assert L.darb_layer_norm(0, 0, F, B, BUF, *good, None, None, 1e-5, BUF, *s, None, None,
                                 None) == darb.E_INVALID
        assert L.darb_layer_norm_grad(0, 0, F, B, BUF, *good, BUF, *good, BUF, BUF, None, BUF, *s, None, None, WS,
                                      BIG, None) == darb.E_INVALID


@pytest.mark.parametrize("F,B,good,at", ONE)
def test_read_operands_do_not_go_backwards(F, B, good, at):
    s = bad(good, at, -1)
    assert L.darb_token_logprobs(0, F, B, BUF, *s, None, 0, BUF, BUF, BUF, None, None, WS, BIG,
                                 None) == darb.E_INVALID
    assert L.darb_token_logprobs_grad(0, F, B, BUF, *s, None, BUF, BUF, None, None, BUF, *good,
                                      None) == darb.E_INVALID
    assert L.darb_layer_norm(0, 0, F, B, BUF, *s, None, None, 1e-5, BUF, *good, None, None, None) == darb.E_INVALID
    for x, dy in ((s, good), (good, s)):
        assert L.darb_layer_norm_grad(0, 0, F, B, BUF, *dy, BUF, *x, BUF, BUF, None, BUF, *good, None, None, WS,
                                      BIG, None) == darb.E_INVALID
