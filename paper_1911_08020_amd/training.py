"""Evaluating and retraining a DARB layer: token log probabilities, layer norm, AdamW.

Argument marshalling for the calls of include/darb.h.  Activations are [features, batch] in
either memory order: contiguous along the batch, as the products' X and Y are, or along the
features, as the transposed view of a [batch, features] tensor is.  Results that have the
shape of an input come in its order.

A call on a given stream takes its results and workspace from that stream's memory.  Its inputs
are the caller's to have ready for that stream, and to keep until it is done with them.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

from . import (BF16, F16, F32, _AdamTensor, _after_current, _as_stream, _check, _check_format,
               _lib, _memory_of, _native, _ptr, _stream_ptr, _torch, _used_on)


class TokenLogprobs(NamedTuple):
    logprob: object                     # fp32 [B]
    entropy: object                     # fp32 [B]
    lse: object                         # fp32 [B]
    top_logprob: Optional[object]       # fp32 [B, top], greatest first
    top_index: Optional[object]         # int64 [B, top]


def _require_cuda(*ts):
    torch = _torch()
    for t in ts:
        if not t.is_cuda:
            raise ValueError("device tensors required (torch cuda tensors)")
        if t.device.index != torch.cuda.current_device():
            raise ValueError(f"a tensor is on {t.device}, the current device is "
                             f"cuda:{torch.cuda.current_device()}")


def _float_code(t, name: str) -> int:
    torch = _torch()
    code = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: unsupported dtype {t.dtype} (fp32, fp16 or bf16)")
    return code


def _matrix(t, name: str, like=None):
    """Checks an operand [F, B] and returns its strides."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be 2-D, got {tuple(t.shape)}")
    if like is not None:
        if t.shape != like.shape:
            raise ValueError(f"{name} must be {tuple(like.shape)}, got {tuple(t.shape)}")
        if t.dtype != like.dtype:
            raise TypeError(f"{name} must be {like.dtype}, got {t.dtype}")
    if t.numel() == 0:
        raise ValueError(f"{name} is empty")
    fs, bs = t.stride()
    F, B = t.shape
    if not (F == 1 or B == 1 or (fs == 1 and bs >= F) or (bs == 1 and fs >= B)):
        raise ValueError(f"{name} must have one unit stride, got {(fs, bs)}")
    return fs, bs


def _empty_like(t):
    """A dense tensor in t's memory order (contiguous where one token or feature leaves it open)."""
    torch = _torch()
    F, B = t.shape
    if t.stride(0) == 1 and F > 1 and B > 1:
        return torch.empty((B, F), dtype=t.dtype, device=t.device).t()
    return torch.empty((F, B), dtype=t.dtype, device=t.device)


def _vector(t, n: int, name: str, dtype=None):
    torch = _torch()
    _require_cuda(t)
    _check_format(t, n, name, (dtype or torch.float32,))
    return _ptr(t)


def _optional(t, n: int, name: str, dtype=None):
    return None if t is None else _vector(t, n, name, dtype)


def _workspace(fn, where: str, device, workspace, *sizes):
    torch = _torch()
    need = ctypes.c_int64()
    _check(fn(*sizes, ctypes.byref(need)), where)
    if workspace is None:
        if need.value == 0:
            return None
        workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
    _require_cuda(workspace)
    _check_format(workspace, need.value, "workspace", (torch.uint8,))
    return workspace


def token_logprobs(logits, targets=None, top: int = 0, workspace=None, stream=None) -> TokenLogprobs:
    """Log probability of each column's target under logits [V, B] (fp32, fp16 or bf16), the
    column's entropy and log sum, and its ``top`` (at most 64) most likely alternatives, equal
    ones by the lower class.

    ``targets``: int64 [B]; a negative one means that the column has none (logprob 0).  See
    darb_token_logprobs in include/darb.h for masked logits (-inf), NaN and refused values.
    """
    if workspace is None:
        done = _native.token_logprobs(logits, targets, top, stream)
        if done is not None:
            return TokenLogprobs(*done)
    torch = _torch()
    _require_cuda(logits)
    code = _float_code(logits, "logits")
    fs, bs = _matrix(logits, "logits")
    V, B = logits.shape
    top = int(top)
    dev = logits.device
    tp = _optional(targets, B, "targets", torch.int64)
    with _memory_of(stream):
        workspace = _workspace(_lib.darb_token_logprobs_workspace, "darb_token_logprobs_workspace",
                               dev, workspace, code, V, B, fs, bs, top)
        out = torch.empty((3, B), dtype=torch.float32, device=dev)
        tl = torch.empty((B, top), dtype=torch.float32, device=dev) if top else None
        ti = torch.empty((B, top), dtype=torch.int64, device=dev) if top else None
    base = out.data_ptr()
    _check(_lib.darb_token_logprobs(code, V, B, _ptr(logits), fs, bs, tp, top,
                                    ctypes.c_void_p(base), ctypes.c_void_p(base + 4 * B),
                                    ctypes.c_void_p(base + 8 * B), _ptr(tl) if top else None,
                                    _ptr(ti) if top else None,
                                    None if workspace is None else _ptr(workspace),
                                    0 if workspace is None else workspace.numel(),
                                    _stream_ptr(stream)),
           "darb_token_logprobs")
    _used_on(stream, out, tl, ti, workspace)
    return TokenLogprobs(out[0], out[1], out[2], tl, ti)


def token_logprobs_grad(logits, targets, lse, grad_logprob=None, entropy=None, grad_entropy=None,
                        out=None, stream=None):
    """The gradient by the logits of sum(grad_logprob * logprob + grad_entropy * entropy), from
    ``token_logprobs``' lse (and entropy).  ``out`` may be ``logits`` itself."""
    done = _native.token_logprobs_grad(logits, targets, lse, grad_logprob, entropy, grad_entropy,
                                       out, stream)
    if done is not None:
        return done
    torch = _torch()
    _require_cuda(logits)
    code = _float_code(logits, "logits")
    fs, bs = _matrix(logits, "logits")
    V, B = logits.shape
    if out is None:
        with _memory_of(stream):
            out = _empty_like(logits)
    _require_cuda(out)
    ofs, obs = _matrix(out, "out", logits)
    _check(_lib.darb_token_logprobs_grad(
        code, V, B, _ptr(logits), fs, bs, _optional(targets, B, "targets", torch.int64),
        _vector(lse, B, "lse"), _optional(grad_logprob, B, "grad_logprob"),
        _optional(entropy, B, "entropy"), _optional(grad_entropy, B, "grad_entropy"), _ptr(out),
        ofs, obs, _stream_ptr(stream)), "darb_token_logprobs_grad")
    _used_on(stream, out)
    return out


def _norm_weight(t, x, H: int, name: str):
    if t is None:
        return None, None
    torch = _torch()
    _require_cuda(t)
    _check_format(t, H, name, (torch.float32, x.dtype))
    return _ptr(t), t.dtype


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, y=None, mean=None, rstd=None,
               stream=None):
    """(y, mean, rstd): layer norm over the features of x [H, B] (fp32, fp16 or bf16), with
    weight and bias [H] in fp32 or x's type; mean and rstd fp32 [B].  ``y`` may be x."""
    done = _native.layer_norm(x, weight, bias, eps, y, mean, rstd, stream)
    if done is not None:
        return done
    torch = _torch()
    _require_cuda(x)
    code = _float_code(x, "x")
    fs, bs = _matrix(x, "x")
    H, B = x.shape
    wp, wt = _norm_weight(weight, x, H, "weight")
    bp, bt = _norm_weight(bias, x, H, "bias")
    if wt is not None and bt is not None and wt != bt:
        raise TypeError("weight and bias must have one dtype")
    wdtype = wt or bt or torch.float32
    with _memory_of(stream):
        if y is None:
            y = _empty_like(x)
        if mean is None:
            mean = torch.empty(B, dtype=torch.float32, device=x.device)
        if rstd is None:
            rstd = torch.empty(B, dtype=torch.float32, device=x.device)
    _require_cuda(y)
    yfs, ybs = _matrix(y, "y", x)
    _check(_lib.darb_layer_norm(code, F32 if wdtype == torch.float32 else code, H, B, _ptr(x), fs,
                                bs, wp, bp, float(eps), _ptr(y), yfs, ybs,
                                _vector(mean, B, "mean"), _vector(rstd, B, "rstd"),
                                _stream_ptr(stream)), "darb_layer_norm")
    _used_on(stream, y, mean, rstd)
    return y, mean, rstd


def layer_norm_grad(dy, x, mean, rstd, weight=None, dx=None, dweight=None, dbias=None,
                    need_x: bool = True, need_params: bool = True, workspace=None, stream=None):
    """(dx, dweight, dbias) of ``layer_norm`` from dy and x [H, B] and its mean and rstd; dweight
    and dbias are fp32 [H].  None in the place of what is not needed.  ``dx`` may be dy or x."""
    if need_x and need_params and dx is dweight is dbias is workspace is None:
        done = _native.layer_norm_grad(dy, x, mean, rstd, weight, stream)
        if done is not None:
            return done
    torch = _torch()
    _require_cuda(dy, x)
    code = _float_code(x, "x")
    fs, bs = _matrix(x, "x")
    gfs, gbs = _matrix(dy, "dy", x)
    H, B = x.shape
    wp, wt = _norm_weight(weight, x, H, "weight")
    dfs = dbs = 0
    with _memory_of(stream):
        if need_x and dx is None:
            dx = _empty_like(x)
        if need_params and dweight is None:
            dweight = torch.empty(H, dtype=torch.float32, device=x.device)
        if need_params and dbias is None:
            dbias = torch.empty(H, dtype=torch.float32, device=x.device)
        workspace = _workspace(_lib.darb_layer_norm_workspace, "darb_layer_norm_workspace",
                               x.device, workspace, H, B)
    if need_x:
        _require_cuda(dx)
        dfs, dbs = _matrix(dx, "dx", x)
    _check(_lib.darb_layer_norm_grad(
        code, F32 if wt in (None, torch.float32) else code, H, B, _ptr(dy), gfs, gbs, _ptr(x), fs,
        bs, _vector(mean, B, "mean"), _vector(rstd, B, "rstd"), wp, _ptr(dx) if need_x else None,
        dfs, dbs, _vector(dweight, H, "dweight") if need_params else None,
        _vector(dbias, H, "dbias") if need_params else None, _ptr(workspace), workspace.numel(),
        _stream_ptr(stream)), "darb_layer_norm_grad")
    _used_on(stream, workspace, *([dx] if need_x else []), *([dweight, dbias] if need_params else []))
    return (dx if need_x else None, dweight if need_params else None,
            dbias if need_params else None)


class AdamW:
    """AdamW with decoupled weight decay over many tensors in one launch (darb_adamw_step).

    ``params``: contiguous device tensors, fp32, fp16 or bf16, of any shapes; updated in place.
    ``masters``: True keeps fp32 copies of the 16-bit ones, which the step updates and rounds
    into the parameters; or a list of fp32 tensors (or None) to use.  ``state_bits``: 32, or 8
    for moments in 8-bit codes with a scale per 256 elements, rounded at random.
    ``weight_decay``: one number, or one per tensor.  ``state``: moments to go on from, for each
    tensor (m, v) fp32, or (m codes, v codes, m scales, v scales) (``state_tensors`` gives them);
    ``steps``: the steps already taken.  Bits of the rounding come from ``seed`` and the step's
    number: the same run gives the same bits.

    The tensors must not overlap.  The optimizer keeps references to them; a step reads the
    gradients at their addresses of that call.
    """

    BLOCK = 256

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.01, state_bits: int = 32, masters=None, state=None,
                 steps: int = 0, seed: int = 0, stream=None):
        torch = _torch()
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        self.lr, self.betas, self.eps = float(lr), (float(betas[0]), float(betas[1])), float(eps)
        self.state_bits, self.steps, self.seed = int(state_bits), int(steps), int(seed)
        if self.state_bits not in (8, 32):
            raise ValueError("state_bits must be 32 or 8")
        count = len(self.params)
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * count
        for what, given in (("weight_decay", decay), ("state", state)):
            if given is not None and len(given) != count:
                raise ValueError(f"{what} must have one entry per tensor ({count})")
        dev = self.params[0].device
        for i, p in enumerate(self.params):
            _require_cuda(p)
            _float_code(p, f"parameter {i}")
            if p.device != dev:
                raise ValueError("the parameters must be on one device")
            if not p.is_contiguous():
                raise ValueError(f"parameter {i} must be contiguous")
        if masters is True:
            masters = [p.detach().float() if p.dtype != torch.float32 else None
                       for p in self.params]
        elif masters is None or masters is False:
            masters = [None] * count
        self.masters = list(masters)
        if len(self.masters) != count:
            raise ValueError(f"masters must have one entry per tensor ({count})")
        if state is None:
            state = [self._zeros(p) for p in self.params]
        self.state_tensors = [tuple(s) for s in state]
        table = (_AdamTensor * count)()
        for i, (p, t, s) in enumerate(zip(self.params, self.masters, self.state_tensors)):
            table[i] = self._entry(i, p, t, s, float(decay[i]))
        self.workspace = _workspace(_lib.darb_adamw_workspace, "darb_adamw_workspace", dev, None,
                                    table, count)
        _after_current(stream)              # the masters and zeros above
        h = ctypes.c_void_p()
        with torch.cuda.device(dev):
            _check(_lib.darb_adamw_create(table, count, self.state_bits, _ptr(self.workspace),
                                          self.workspace.numel(), _stream_ptr(stream),
                                          ctypes.byref(h)), "darb_adamw_create")
        self._h = h
        self._streams = set()               # that _hold_on was told of

    def _hold_on(self, stream):
        """The table, states, masters and parameters are in use on this stream (None: the current
        one): dropping the optimizer does not hand them out before its work there is done."""
        at = _native.current_stream() if stream is None else stream.cuda_stream
        if at not in self._streams:
            torch = _torch()
            s = torch.cuda.current_stream() if stream is None else _as_stream(stream)
            for t in [self.workspace, *self.params, *self.masters,
                      *(t for state in self.state_tensors for t in state)]:
                if t is not None:
                    t.record_stream(s)
            self._streams.add(at)

    def __del__(self, _destroy=_lib.darb_adamw_destroy):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            _destroy(h)
            self._h = None

    def _zeros(self, p):
        torch = _torch()
        n = p.numel()
        kind = dict(device=p.device)
        if self.state_bits == 32:
            return tuple(torch.zeros(n, dtype=torch.float32, **kind) for _ in range(2))
        blocks = -(-n // self.BLOCK)
        return (torch.zeros(n, dtype=torch.uint8, **kind),
                torch.zeros(n, dtype=torch.uint8, **kind),
                torch.zeros(blocks, dtype=torch.float32, **kind),
                torch.zeros(blocks, dtype=torch.float32, **kind))

    def _entry(self, i, p, master, state, decay):
        torch = _torch()
        n = p.numel()
        blocks = -(-n // self.BLOCK)
        kinds = [(n, torch.float32)] * 2 if self.state_bits == 32 else \
            [(n, torch.uint8)] * 2 + [(blocks, torch.float32)] * 2
        if len(state) != len(kinds):
            raise ValueError(f"state {i} must have {len(kinds)} tensors")
        ptrs = [_vector(t, k, f"state {i}", dtype) for t, (k, dtype) in zip(state, kinds)]
        ptrs += [None] * (4 - len(ptrs))
        return _AdamTensor(p.data_ptr(), None if master is None else
                           _vector(master, n, f"master {i}"), *ptrs, n, decay,
                           _float_code(p, f"parameter {i}"), 0)

    def step(self, grads, lr: Optional[float] = None, grad_scale=None, stream=None):
        """One step with the gradients (contiguous, fp32, fp16 or bf16, each of its parameter's
        size; None leaves a tensor as it is).  ``grad_scale``: a device fp32 tensor whose first
        element multiplies every gradient (a clipping or loss scale computed on the device)."""
        t = self.steps + 1
        seed = (self.seed + t * 0x6A09E667) & 0xFFFFFFFF
        lr = self.lr if lr is None else float(lr)
        self._hold_on(stream)
        if _native.adamw_step(self._h.value, self.params, grads, lr, *self.betas, self.eps, t,
                              grad_scale, seed, stream):
            self.steps = t
            return
        count = len(self.params)
        if len(grads) != count:
            raise ValueError(f"one gradient per tensor ({count}), got {len(grads)}")
        ptrs, types = (ctypes.c_void_p * count)(), (ctypes.c_int * count)()
        for i, (g, p) in enumerate(zip(grads, self.params)):
            if g is None:
                continue
            _require_cuda(g)
            types[i] = _float_code(g, f"gradient {i}")
            if not g.is_contiguous() or g.numel() != p.numel():
                raise ValueError(f"gradient {i} must be contiguous with {p.numel()} elements")
            ptrs[i] = g.data_ptr() or None
        _check(_lib.darb_adamw_step(self._h, ptrs, types, count, lr, *self.betas, self.eps, t,
                                    _optional(grad_scale, 1, "grad_scale"), seed,
                                    _stream_ptr(stream)), "darb_adamw_step")
        self.steps = t

    def moments(self, out=None, stream=None):
        """(list of m, list of v): the values that the states stand for, fp32, flat."""
        torch = _torch()
        self._hold_on(stream)
        if out is None:
            with _memory_of(stream):
                out = tuple([torch.empty(p.numel(), dtype=torch.float32, device=p.device)
                             for p in self.params] for _ in range(2))
        if _native.adamw_moments(self._h.value, self.params, out[0], out[1], stream):
            _used_on(stream, *out[0], *out[1])
            return out
        count = len(self.params)
        arrays = []
        for name, ts in zip("mv", out):
            if len(ts) != count:
                raise ValueError(f"out must have {count} tensors of {name}")
            a = (ctypes.c_void_p * count)()
            for i, (t, p) in enumerate(zip(ts, self.params)):
                a[i] = _vector(t, p.numel(), f"out {i}").value or None
            arrays.append(a)
        _check(_lib.darb_adamw_moments(self._h, *arrays, count, _stream_ptr(stream)),
               "darb_adamw_moments")
        _used_on(stream, *out[0], *out[1])
        return out
