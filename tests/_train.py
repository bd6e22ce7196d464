"""What the tests of the evaluation and retraining calls share: operands in every memory order,
types, and the bound of one rounding to a type."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
#: half a unit in the last place, and half the smallest step near zero
ROUND = {"f32": (2.0 ** -24, 0.0), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -134)}

#: features (contiguous along the batch), tokens (along the features), each also inside a wider
#: buffer that starts at an odd element
ORDERS = ["features", "tokens", "features+", "tokens+"]


def place(a, order, dtype):
    """Host array [F, B] as a device tensor of that order and type."""
    t = torch.from_numpy(np.ascontiguousarray(a)).to(TYPES[dtype])
    F, B = t.shape
    if not order.startswith("features"):
        t = t.t()
    if order.endswith("+"):
        rows, cols = t.shape
        wide = torch.full((rows * (cols + 5) + 3,), 7.0, dtype=t.dtype, device="cuda")
        view = wide[3:].view(rows, cols + 5)[:, :cols]
        view.copy_(t)
        t = view
    else:
        t = t.contiguous().cuda()
    return t if order.startswith("features") else t.t()


def wide(t):
    """The values as fp64 on the host."""
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def rounding(want, dtype):
    rel, small = ROUND[dtype]
    return rel * np.abs(want) + small


def check(got, want, bound, label):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, label
    bound = np.broadcast_to(bound, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), label
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), label
    off, bound = np.abs(got[fine] - want[fine]), bound[fine]
    worst = float((off / np.maximum(bound, 1e-300)).max()) if fine.any() else 0.0
    assert not (off > bound).any(), f"{label}: {worst:.3g} times the bound"
    return worst
