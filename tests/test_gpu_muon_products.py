"""The orthogonalised update of 16-bit matrices: as accurate as fp32 and rounded once, or, where the
caller asks for it, with products of fp16 operands."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb, say  # noqa: E402,F401
from _train import ROUND, TYPES, wide  # noqa: E402
from test_gpu_muon import SHAPES, bound, exact, matrix  # noqa: E402

pytestmark = pytest.mark.gpu

HALVES = ["f16", "bf16"]
TILED = [(64, 64), (70, 900), (290, 300), (520, 270), (400, 590), (333, 1100)]


def given(shape, kind, seed, dtype):
    return torch.from_numpy(matrix(*shape, kind, seed)).to(TYPES[dtype]).cuda()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("kind", ["flat", "low"])
def test_a_16_bit_result_is_the_fp32_one_rounded(darb, dtype, kind):
    """The same products in the same order: not a bit more is lost than the result's own rounding."""
    for n, shape in enumerate(SHAPES + TILED + [(256, 1024)]):
        g = given(shape, kind, 200 + n, dtype)
        say(dtype, kind, shape)
        assert torch.equal(darb.orthogonalize(g), darb.orthogonalize(g.float()).to(g.dtype)), shape
    many = torch.stack([given((256, 1024), kind, 300 + i, dtype) for i in range(8)])
    assert torch.equal(darb.orthogonalize(many), darb.orthogonalize(many.float()).to(many.dtype))


@pytest.mark.parametrize("dtype", HALVES)
def test_a_16_bit_parameter_is_the_step_of_its_fp32_copy_rounded(darb, dtype):
    shapes = [(64, 200), (300, 130), (96, 96), (3, 70)]
    params = [given(s, "flat", 20 + i, dtype) * 0.1 for i, s in enumerate(shapes)]
    grads = [given(s, "low", 30 + i, dtype) * 1e-3 for i, s in enumerate(shapes)]
    kw = dict(lr=0.03, weight_decay=0.1)
    plain = darb.Muon([p.clone() for p in params], **kw)
    kept = darb.Muon([p.clone() for p in params], masters=True, **kw)
    for opt in (plain, kept):
        opt.step(grads)
    for a, b, m in zip(plain.params, kept.params, kept.masters):
        assert torch.equal(a, b) and torch.equal(a, m.to(a.dtype))


@pytest.mark.parametrize("dtype", HALVES)
def test_fp16_products(darb, dtype):
    """Within the bound of operands rounded to 11 bits; fp32 results and small matrices as without."""
    for n, shape in enumerate(SHAPES):
        G = given(shape, "flat", n, dtype)
        g = wide(G)
        want = exact(g, 5, 1e-7)
        got = darb.orthogonalize(G, fp16_products=True)
        off = np.linalg.norm(wide(got) - want)
        rounded = ROUND[dtype][0] * np.linalg.norm(want) + ROUND[dtype][1] * math.sqrt(want.size)
        say(dtype, shape, off / np.linalg.norm(want))
        assert off <= bound(g, 5, 1e-7, False) + rounded, shape
        if min(shape) < 64:
            assert torch.equal(got, darb.orthogonalize(G))
        assert torch.equal(darb.orthogonalize(G.float(), fp16_products=True), darb.orthogonalize(G.float()))
    # of a parameter: 0.1 of the update's
    p, g = given((130, 300), "flat", 1, dtype), given((130, 300), "low", 2, dtype)
    opt = darb.Muon([p.clone()], lr=0.1, fp16_products=True)
    opt.step([g])
    u = wide(opt.momenta[0]) * 0.95 + 0.05 * wide(g)
    want = wide(p) - 0.1 * exact(u, 5, 1e-7)
    # the momentum is read back, so that u's own rounding (3 units of 2^-24) is below the bound's room
    limit = 0.1 * bound(u, 5, 1e-7, False) + (ROUND[dtype][0] + 4 * 2.0 ** -24) * np.linalg.norm(want) + \
        ROUND[dtype][1] * math.sqrt(want.size)
    assert np.linalg.norm(wide(opt.params[0]) - want) <= limit


@pytest.mark.parametrize("dtype", HALVES)
def test_every_tile_of_fp16_products(darb, dtype):
    """Each kind of tile, where tiles hang over, and where the sums are shorter than the stages ahead."""
    P, I64, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    call = darb.lib().darb_test_orthogonalize
    call.argtypes, call.restype = [P, I64, I, ctypes.c_double, P, I64, I, I, I, P], I
    code = {"f16": 1, "bf16": 2}[dtype]
    mats = [given(s, "flat", 70 + i, dtype) for i, s in enumerate(TILED)]
    want = [exact(wide(g), 5, 1e-7) for g in mats]
    limit = [bound(wide(g), 5, 1e-7, False) for g in mats]
    for kinds in ((0, 0, 0), (2, 2, 1), (2, 2, 2), (3, 3, 3), (4, 4, 4), (4, 0, 1)):
        for only in (None, 3):
            table = (darb._MuonTensor * len(mats))()
            out = [torch.empty_like(g) for g in mats]
            chosen = [i for i in range(len(mats)) if only in (None, i)]
            for j, i in enumerate(chosen):
                r, c = TILED[i]
                table[j] = darb._MuonTensor(out[i].data_ptr(), None, mats[i].data_ptr(), None, r, c, c, c, 1.0, 0.0,
                                            code, code, 1)
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
                    assert off <= limit[i] + rounded, (kinds, TILED[i], off, limit[i])
                    # no element is off by itself: a product's error is spread over a row and a column
                    worst = np.abs(got - want[i]).max()
                    assert worst <= 0.02 + ROUND[dtype][0] * np.abs(want[i]).max(), (kinds, TILED[i], worst)


def test_lists_of_unlike_accuracy(darb):
    """Tensors of both accuracies in one call: each group's results as if it were alone."""
    shapes = [(64, 130), (100, 70), (64, 130)]
    mats = [given(s, "flat", 40 + i, t) for i, (s, t) in enumerate(zip(shapes, ("bf16", "bf16", "f32")))]
    code = {torch.float32: 0, torch.bfloat16: 2}
    lib = darb.lib()

    def call(which, fp16):
        table = (darb._MuonTensor * len(which))()
        out = [torch.empty_like(mats[i]) for i in which]
        for j, i in enumerate(which):
            (r, c), t = shapes[i], code[mats[i].dtype]
            table[j] = darb._MuonTensor(out[j].data_ptr(), None, mats[i].data_ptr(), None, r, c, c, c, 1.0, 0.0, t, t,
                                        fp16[j])
        n = ctypes.c_int64()
        assert lib.darb_muon_workspace(table, len(which), ctypes.byref(n)) == 0
        ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
        assert lib.darb_orthogonalize(table, len(which), 5, 1e-7, ws.data_ptr(), n.value,
                                      torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        return out
    a, b, c = call([0, 1, 2], [1, 0, 1])
    assert torch.equal(a, call([0], [1])[0])
    assert all(torch.equal(x, y) for x, y in zip((b, c), call([1, 2], [0, 0])))
