"""Long sequences cut into slabs of time, with and without restarts, in a workspace that holds nothing
to go on from."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from _gpu import darb, say  # noqa: E402,F401
from _recurrence import backward, forward  # noqa: E402
from _train import TYPES, check, place, rounding, wide  # noqa: E402
from test_gpu_recurrence import data, on, state  # noqa: E402

pytestmark = pytest.mark.gpu

#: rows along time, rows through LDS, and both orders read directly, of odd sizes
SIZES = [(3, 20000, 1, "features"), (1, 8193, 1, "features"), (2, 9001, 3, "features"), (5, 3001, 1, "tokens"),
         (2, 2500, 7, "tokens"), (4, 3000, 20, "features")]


def room(darb, code, back, H, T, batch):
    """A workspace that is NaN to its end."""
    n = ctypes.c_int64()
    assert darb.lib().darb_gated_recurrence_workspace(code, back, H, T, batch, ctypes.byref(n)) == 0
    assert n.value > 0, "not cut into slabs"
    return torch.full((n.value // 4,), float("nan"), device="cuda").view(torch.uint8)


@pytest.mark.parametrize("H,T,batch,order", SIZES)
@pytest.mark.parametrize("form", ["gate", "linear"])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_slabs(darb, dtype, form, H, T, batch, order):
    code = {"f32": 0, "f16": 1, "bf16": 2}[dtype]
    for resets in (False, True):
        say(dtype, form, H, T, batch, order, resets)
        z, x, h0, starts, r = data(H, T, batch, form, resets, T + 1, dtype)
        if resets:
            starts[:] = r.random(T * batch) < 0.002
        want, last, bound, lbound = forward(z, x, h0, starts, batch, form)
        hr = torch.from_numpy(want).to(TYPES[dtype]).double().numpy()
        dh = torch.from_numpy(r.normal(size=z.shape)).to(TYPES[dtype]).double().numpy()
        dl = r.normal(size=h0.shape).astype(np.float32)
        grads = backward(dh, z, x, hr, h0, dl, starts, batch, form)
        args = dict(batch=batch, h0=state(h0, order), resets=on(starts), form=form)
        put = lambda a: place(a, order, dtype)                                       # noqa: E731
        for again in range(2):
            h, hl = darb.gated_recurrence(put(z), put(x), workspace=room(darb, code, 0, H, T, batch), **args)
            check(wide(h), want, bound + rounding(np.abs(want) + bound, dtype), "h")
            check(wide(hl), last, lbound + 2.0 ** -24 * np.abs(last), "last")
            got = darb.gated_recurrence_grad(put(dh), put(z), put(x), put(hr), dh_last=state(dl, order),
                                             workspace=room(darb, code, 1, H, T, batch), **args)
            for g, w, b, name in zip(got, grads[:3], grads[3:], ("dgate", "dx", "dh0")):
                check(wide(g), w, b + rounding(np.abs(w) + b, dtype if name != "dh0" else "f32"), name)
