"""Through the C ABI, whatever the type beside a NULL gradient says, the other tensors' gradients
are read as what they are."""
import ctypes

import pytest

from tests._gpu import darb, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("junk", [-1, 3, 0x55555555])
def test_types_beside_null_gradients(darb, junk):  # noqa: F811
    say(f"adamw: type {junk} beside NULL gradients")
    count = 40
    start = [torch.randn(100 + i, device="cuda") for i in range(count)]
    kinds = [torch.float32, torch.float16, torch.bfloat16]
    grads = [None if i % 5 == 2 else torch.randn(100 + i, device="cuda").to(kinds[i % 3]) for i in range(count)]
    want, got = [t.clone() for t in start], [t.clone() for t in start]
    darb.AdamW(want).step(grads)
    opt = darb.AdamW(got)
    codes = {torch.float32: darb.F32, torch.float16: darb.F16, torch.bfloat16: darb.BF16}
    ptrs = (ctypes.c_void_p * count)(*[None if g is None else g.data_ptr() for g in grads])
    types = (ctypes.c_int * count)(*[junk if g is None else codes[g.dtype] for g in grads])
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    rc = darb.lib().darb_adamw_step(opt._h, ptrs, types, count, opt.lr, *opt.betas, opt.eps, 1, None, 0, stream)
    assert rc == 0, darb.lib().darb_last_error()
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), i
        assert torch.equal(a, start[i]) == (grads[i] is None)
