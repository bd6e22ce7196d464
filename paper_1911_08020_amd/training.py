"""Evaluating and retraining a DARB layer: token log probabilities and the losses over them, layer
norm, a gated recurrence, AdamW and the orthogonalised update.

Argument marshalling for the calls of include/darb.h.  Activations are [features, batch] in
either memory order: contiguous along the batch, as the products' X and Y are, or along the
features, as the transposed view of a [batch, features] tensor is.  Results that have the
shape of an input come in its order.

A call on a given stream takes its results and workspace from that stream's memory.  Its inputs
are the caller's to have ready for that stream, and to keep until it is done with them.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional

from . import (BF16, F16, F32, _AdamTensor, _Matrix, _MuonTensor, _after_current, _as_stream,
               _check, _check_format, _lib, _memory_of, _native, _ptr, _stream_ptr, _torch,
               _used_on)


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


# ---- gated recurrence ------------------------------------------------------------------

FORMS = {"gate": 0, "linear": 1}


def _as_matrix(t, name: str, like=None):
    _require_cuda(t)
    fs, bs = _matrix(t, name, like)
    return _Matrix(t.data_ptr(), fs, bs)


def _as_state(t, H: int, batch: int, name: str):
    if t is None:
        return None
    torch = _torch()
    _require_cuda(t)
    if t.dtype != torch.float32 or tuple(t.shape) != (H, batch):
        raise ValueError(f"{name} must be fp32 [{H}, {batch}], got {t.dtype} {tuple(t.shape)}")
    return ctypes.byref(_Matrix(t.data_ptr(), *t.stride()))


def _sequences(x, batch, form, resets):
    """Checks what both directions share; returns (dtype code, form, H, T, batch, resets)."""
    torch = _torch()
    code = _float_code(x, "x")
    if form not in FORMS:
        raise ValueError(f"form must be one of {tuple(FORMS)}, got {form!r}")
    batch = int(batch)
    H, columns = x.shape
    if batch < 1 or columns % batch:
        raise ValueError(f"{columns} columns are not a multiple of the batch ({batch})")
    if resets is None:
        return code, FORMS[form], H, columns // batch, batch, None
    _require_cuda(resets)
    if resets.dim() != 1 or resets.shape[0] != columns:
        raise ValueError(f"resets must be [{columns}], got {tuple(resets.shape)}")
    _check_format(resets, columns, "resets", (torch.bool, torch.uint8))
    return code, FORMS[form], H, columns // batch, batch, _ptr(resets)


def _state_like(x, H: int, batch: int):
    """A new fp32 state [H, batch] in x's memory order."""
    torch = _torch()
    if x.stride(0) == 1 and H > 1 and x.shape[1] > 1:
        return torch.empty((batch, H), dtype=torch.float32, device=x.device).t()
    return torch.empty((H, batch), dtype=torch.float32, device=x.device)


def gated_recurrence(gate, x, batch: int = 1, h0=None, resets=None, form: str = "gate", h=None,
                     h_last=None, workspace=None, stream=None):
    """(h, h_last): h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(gate) (``form`` "gate"), or
    h_t = gate_t h_{t-1} + x_t ("linear"), over the sequences of gate and x [H, T * batch] (fp32,
    fp16 or bf16; column t * batch + n is step t of sequence n).

    ``h0``, ``h_last``: fp32 [H, batch], the states before and after; they may be one tensor.
    ``resets``: bool or uint8 [T * batch], where a new sequence starts.  ``h`` may be gate or x.
    T = 1 is the step of a program that generates.  See darb_gated_recurrence."""
    if workspace is None:
        done = _native.gated_recurrence(gate, x, batch, h0, resets, FORMS.get(form, -1), h, h_last, stream)
        if done is not None:
            return done
    _require_cuda(gate, x)
    xm = _as_matrix(x, "x")
    gm = _as_matrix(gate, "gate", x)
    code, kind, H, T, batch, rp = _sequences(x, batch, form, resets)
    with _memory_of(stream):
        workspace = _workspace(_lib.darb_gated_recurrence_workspace, "darb_gated_recurrence_workspace",
                               x.device, workspace, code, 0, H, T, batch)
        if h is None:
            h = _empty_like(x)
        if h_last is None:
            h_last = _state_like(x, H, batch)
    hm = _as_matrix(h, "h", x)
    _check(_lib.darb_gated_recurrence(
        code, kind, H, T, batch, ctypes.byref(gm), ctypes.byref(xm), rp,
        _as_state(h0, H, batch, "h0"), ctypes.byref(hm), _as_state(h_last, H, batch, "h_last"),
        None if workspace is None else _ptr(workspace),
        0 if workspace is None else workspace.numel(), _stream_ptr(stream)), "darb_gated_recurrence")
    _used_on(stream, h, h_last, workspace)
    return h, h_last


def gated_recurrence_grad(dh, gate, x, h, batch: int = 1, h0=None, resets=None, dh_last=None,
                          form: str = "gate", dgate=None, dx=None, dh0=None, workspace=None,
                          stream=None):
    """(dgate, dx, dh0) of ``gated_recurrence`` from dh, by every state, and dh_last (fp32
    [H, batch] or None), by the last one; ``h`` as it was returned.  ``x`` may be None in the linear
    form.  ``dgate`` and ``dx`` may be dh, gate or x, not h; ``dh0`` (fp32 [H, batch]) may be
    dh_last."""
    if workspace is None:
        done = _native.gated_recurrence_grad(dh, gate, x, h, batch, h0, resets, dh_last, FORMS.get(form, -1),
                                             dgate, dx, dh0, stream)
        if done is not None:
            return done
    _require_cuda(dh, gate, h)
    gm = _as_matrix(gate, "gate")
    dm, hm = _as_matrix(dh, "dh", gate), _as_matrix(h, "h", gate)
    if x is None and form != "linear":
        raise ValueError("x is needed in this form")
    xm = None if x is None else ctypes.byref(_as_matrix(x, "x", gate))
    code, kind, H, T, batch, rp = _sequences(gate, batch, form, resets)
    with _memory_of(stream):
        workspace = _workspace(_lib.darb_gated_recurrence_workspace, "darb_gated_recurrence_workspace",
                               gate.device, workspace, code, 1, H, T, batch)
        if dgate is None:
            dgate = _empty_like(gate)
        if dx is None:
            dx = _empty_like(gate)
        if dh0 is None:
            dh0 = _state_like(gate, H, batch)
    ggm, dxm = _as_matrix(dgate, "dgate", gate), _as_matrix(dx, "dx", gate)
    _check(_lib.darb_gated_recurrence_grad(
        code, kind, H, T, batch, ctypes.byref(dm), ctypes.byref(gm), xm, ctypes.byref(hm), rp,
        _as_state(h0, H, batch, "h0"), _as_state(dh_last, H, batch, "dh_last"), ctypes.byref(ggm),
        ctypes.byref(dxm), _as_state(dh0, H, batch, "dh0"),
        None if workspace is None else _ptr(workspace),
        0 if workspace is None else workspace.numel(), _stream_ptr(stream)),
        "darb_gated_recurrence_grad")
    _used_on(stream, dgate, dx, dh0, workspace)
    return dgate, dx, dh0


# ---- losses over token log probabilities -----------------------------------------------

class PolicyLoss(NamedTuple):
    loss: object                        # fp32 [], as kl and clipped
    kl: object
    clipped: object
    grad_logprob: object                # fp32 [B]
    grad_entropy: Optional[object]      # fp32 [B]


class PreferenceLoss(NamedTuple):
    loss: object                        # fp32 []
    margin: object                      # fp32 [P]
    grad_logprob: object                # fp32 [B]


def _tokens(t, n: int, name: str):
    if t is None:
        return None
    if t.dim() != 1 or t.shape[0] != n:
        raise ValueError(f"{name} must be [{n}], got {tuple(t.shape)}")
    return _vector(t, n, name)


def policy_loss(logprob, old_logprob, advantage, weight=None, clip=0.2, ref_logprob=None,
                kl_coef: float = 0.0, entropy=None, entropy_coef: float = 0.0, grad_logprob=None,
                grad_entropy=None, workspace=None, stream=None) -> PolicyLoss:
    """The clipped policy loss of tokens with log probabilities ``logprob`` (fp32 [B],
    ``token_logprobs``'), sampled at ``old_logprob``, and its gradients, which
    ``token_logprobs_grad`` takes: sum of weight * (-min(r A, clip(r) A) + kl_coef (e^q - 1 - q)
    - entropy_coef entropy) with r = e^(logprob - old), q = ref_logprob - logprob.

    ``weight``: fp32 [B], 0 for tokens that do not count (None: 1 / B each).  ``clip``: one bound, or
    (below, above).  See darb_policy_loss."""
    low, high = clip if hasattr(clip, "__len__") else (clip, clip)
    low, high, kl_coef, entropy_coef = float(low), float(high), float(kl_coef), float(entropy_coef)
    if workspace is None:
        done = _native.policy_loss(logprob, old_logprob, advantage, weight, low, high, ref_logprob,
                                   kl_coef, entropy, entropy_coef, grad_logprob, grad_entropy, stream)
        if done is not None:
            return PolicyLoss(*done)
    torch = _torch()
    _require_cuda(logprob)
    B = logprob.numel()
    lp = _tokens(logprob, B, "logprob")
    old, adv = _tokens(old_logprob, B, "old_logprob"), _tokens(advantage, B, "advantage")
    if old is None or adv is None:
        raise ValueError("old_logprob and advantage are needed")
    w, ref = _tokens(weight, B, "weight"), _tokens(ref_logprob, B, "ref_logprob")
    ent = _tokens(entropy, B, "entropy")
    kind = dict(dtype=torch.float32, device=logprob.device)
    with _memory_of(stream):
        workspace = _workspace(_lib.darb_policy_loss_workspace, "darb_policy_loss_workspace",
                               logprob.device, workspace, B)
        stats = torch.empty(3, **kind)
        if grad_logprob is None:
            grad_logprob = torch.empty(B, **kind)
        if entropy is None:
            grad_entropy = None
        elif grad_entropy is None:
            grad_entropy = torch.empty(B, **kind)
    _check(_lib.darb_policy_loss(B, lp, old, adv, w, ref, ent, low, high, kl_coef, entropy_coef,
                                 _ptr(stats), _tokens(grad_logprob, B, "grad_logprob"),
                                 _tokens(grad_entropy, B, "grad_entropy"),
                                 None if workspace is None else _ptr(workspace),
                                 0 if workspace is None else workspace.numel(),
                                 _stream_ptr(stream)), "darb_policy_loss")
    _used_on(stream, stats, grad_logprob, grad_entropy, workspace)
    return PolicyLoss(stats[0], stats[1], stats[2], grad_logprob, grad_entropy)


def preference_loss(logprob, ref_logprob=None, batch: Optional[int] = None, starts=None,
                    beta: float = 0.1, label_smoothing: float = 0.0, weight=None,
                    grad_logprob=None, stream=None) -> PreferenceLoss:
    """The preference loss of pairs of sequences over token log probabilities (fp32 [B],
    ``token_logprobs``'), and its gradient, which ``token_logprobs_grad`` takes.  The first half of the
    sequences are the preferred ones, the second half the others of the same pairs.  With a
    sequence's s = sum(logprob - ref_logprob) and m = beta (s_preferred - s_other):
    sum of weight * (-(1 - label_smoothing) log sigmoid(m) - label_smoothing log sigmoid(-m)).

    Either ``batch``, the number of sequences, token t of sequence s being at t * batch + s; or
    ``starts``, int64 [sequences + 1], for packed ones.  ``weight``: fp32 [pairs] (None: 1 / pairs
    each).  See darb_preference_loss."""
    beta, smoothing = float(beta), float(label_smoothing)
    done = _native.preference_loss(logprob, ref_logprob, batch, starts, beta, smoothing, weight, grad_logprob, stream)
    if done is not None:
        return PreferenceLoss(*done)
    torch = _torch()
    _require_cuda(logprob)
    B = logprob.numel()
    lp, ref = _tokens(logprob, B, "logprob"), _tokens(ref_logprob, B, "ref_logprob")
    if (batch is None) == (starts is None):
        raise ValueError("pass batch or starts")
    sp = None
    if starts is not None:
        if starts.dim() != 1:
            raise ValueError("starts must be 1-D")
        sequences = starts.shape[0] - 1
        sp = _vector(starts, sequences + 1, "starts", torch.int64)
    else:
        sequences = int(batch)
    if sequences < 2 or sequences % 2:
        raise ValueError(f"the sequences must be pairs, got {sequences}")
    P = sequences // 2
    if starts is None and B % sequences:
        raise ValueError(f"{B} tokens are not a multiple of the batch ({sequences})")
    kind = dict(dtype=torch.float32, device=logprob.device)
    with _memory_of(stream):
        out = torch.empty(1 + P, **kind)
        if grad_logprob is None:
            grad_logprob = torch.empty(B, **kind)
    _check(_lib.darb_preference_loss(P, B, lp, ref, sp, _tokens(weight, P, "weight"), beta, smoothing,
                                     _ptr(out), ctypes.c_void_p(out.data_ptr() + 4),
                                     _tokens(grad_logprob, B, "grad_logprob"), _stream_ptr(stream)),
           "darb_preference_loss")
    _used_on(stream, out, grad_logprob)
    return PreferenceLoss(out[0], out[1:], grad_logprob)


# ---- the orthogonalised update ---------------------------------------------------------

def _unit_columns(t, name: str) -> int:
    """The leading dimension of a non-empty matrix with unit column stride."""
    if t.dim() != 2 or t.numel() == 0:
        raise ValueError(f"{name} must be a matrix that is not empty, got {tuple(t.shape)}")
    rows, cols = t.shape
    if (cols > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) < cols):
        raise ValueError(f"{name} must have unit column stride")
    return t.stride(0) if rows > 1 else cols


def _muon_workspace(table, count: int, device, workspace):
    return _workspace(_lib.darb_muon_workspace, "darb_muon_workspace", device, workspace, table, count)


def orthogonalize(G, steps: int = 5, eps: float = 1e-7, out=None, workspace=None, stream=None,
                  fp16_products: bool = False):
    """G [m, n], or each matrix of G [k, m, n] (fp32, fp16 or bf16; one of the last two strides 1),
    with its singular values taken towards 1: G / (|G| + eps) through ``steps`` steps of a quintic
    (darb_orthogonalize).  ``out``, in G's memory order, may be G.  ``fp16_products``: a 16-bit result may be off by 1 to
    3 10^-3 of its norm beside its rounding, and takes less time."""
    torch = _torch()
    _require_cuda(G)
    code = _float_code(G, "G")
    if G.dim() not in (2, 3) or G.numel() == 0:
        raise ValueError(f"G must be [m, n] or [k, m, n] and not empty, got {tuple(G.shape)}")
    turned = G.stride(-1) != 1 and G.shape[-1] > 1      # its transpose has the transposed result
    with _memory_of(stream):
        if out is None:
            out = torch.empty(G.mT.shape, dtype=G.dtype, device=G.device).mT if turned else \
                torch.empty(G.shape, dtype=G.dtype, device=G.device)
    _require_cuda(out)
    if out.shape != G.shape or out.dtype != G.dtype:
        raise ValueError(f"out must be {G.dtype} {tuple(G.shape)}")
    a, b = (G.mT, out.mT) if turned else (G, out)
    a, b = (a, b) if G.dim() == 3 else (a[None], b[None])
    count, rows, cols = a.shape
    lda, ldb = _unit_columns(a[0], "G"), _unit_columns(b[0], "out")
    apart = b.stride(0)                     # of two matrices: one behind the other, or row by row in turn
    if count > 1 and apart < (rows - 1) * ldb + cols and not (apart >= cols and ldb >= (count - 1) * apart + cols):
        raise ValueError("the matrices of out must not overlap")
    table = (_MuonTensor * count)()
    size = G.element_size()
    for i in range(count):
        table[i] = _MuonTensor(b.data_ptr() + i * b.stride(0) * size, None,
                               a.data_ptr() + i * a.stride(0) * size, None, rows, cols, ldb, lda,
                               1.0, 0.0, code, code, int(bool(fp16_products)))
    with _memory_of(stream):
        workspace = _muon_workspace(table, count, G.device, workspace)
    _check(_lib.darb_orthogonalize(table, count, int(steps), float(eps), _ptr(workspace),
                                   workspace.numel(), _stream_ptr(stream)), "darb_orthogonalize")
    _used_on(stream, out, workspace)
    return out


class Muon:
    """An optimizer of weight matrices whose update is the momentum's, orthogonalised
    (darb_muon_step): m = momentum m + (1 - momentum) g, u = momentum m + (1 - momentum) g
    (``nesterov``, else m), p = p (1 - lr decay) - lr scale orthogonalize(u).

    ``params``: contiguous device matrices, fp32, fp16 or bf16; updated in place.  ``masters``: True
    keeps fp32 copies of the 16-bit ones, which the step updates and rounds into the parameters;
    or a list of fp32 tensors (or None) to use.  ``scale``: one number or one per matrix (None:
    sqrt(max(1, rows / cols))); ``weight_decay`` as well.  ``state``: momenta to go on from, fp32
    of the matrices' shapes (``momenta`` has them).  ``fp16_products``: the updates of 16-bit
    parameters without masters may be off by 1 to 3 10^-3 of their norm, and take less time.

    The tensors must not overlap.  The optimizer keeps references to them, and its workspace: 16 to
    24 bytes an element, square matrices the most, sides padded to multiples of 32, of the largest
    group of up to 28 matrices and 4 GiB (or a single one).  A step reads the gradients at their
    addresses of that call.  Steps on different streams share the workspace: the caller
    orders them, replays of captured ones among them."""

    def __init__(self, params, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True,
                 weight_decay=0.0, steps: int = 5, eps: float = 1e-7, scale=None, masters=None,
                 state=None, stream=None, fp16_products: bool = False):
        torch = _torch()
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        self.lr, self.momentum, self.nesterov = float(lr), float(momentum), bool(nesterov)
        self.ns_steps, self.eps = int(steps), float(eps)
        count, dev = len(self.params), self.params[0].device
        for i, p in enumerate(self.params):
            _require_cuda(p)
            _float_code(p, f"parameter {i}")
            if p.dim() != 2 or p.numel() == 0 or not p.is_contiguous():
                raise ValueError(f"parameter {i} must be a contiguous matrix that is not empty")
            if p.device != dev:
                raise ValueError("the parameters must be on one device")

        def each(given, what):
            given = list(given) if hasattr(given, "__len__") else [given] * count
            if len(given) != count:
                raise ValueError(f"{what} must have one entry per tensor ({count})")
            return given
        scales = each(scale, "scale")
        decays = each(weight_decay, "weight_decay")
        if masters is True:
            masters = [p.detach().float() if p.dtype != torch.float32 else None for p in self.params]
        self.masters = each(None if masters is False else masters, "masters")
        if state is None:
            state = [torch.zeros(p.shape, dtype=torch.float32, device=dev) for p in self.params]
        self.momenta = each(state, "state")
        self._table = (_MuonTensor * count)()
        for i, (p, t, m) in enumerate(zip(self.params, self.masters, self.momenta)):
            rows, cols = p.shape
            for name, s in (("master", t), ("state", m)):
                if s is not None and tuple(s.shape) != (rows, cols):
                    raise ValueError(f"{name} {i} must be [{rows}, {cols}]")
            self._table[i] = _MuonTensor(
                p.data_ptr(), None if t is None else _vector(t, p.numel(), f"master {i}").value, None,
                _vector(m, p.numel(), f"state {i}").value, rows, cols, cols, cols,
                math.sqrt(max(1.0, rows / cols)) if scales[i] is None else float(scales[i]),
                float(decays[i]), _float_code(p, f"parameter {i}"), 0, int(bool(fp16_products)))
        _after_current(stream)              # the masters and zeros above
        self.workspace = _muon_workspace(self._table, count, dev, None)
        self._streams = set()               # that _hold_on was told of
        self._hold_on(stream)

    def _hold_on(self, stream):
        """The workspace, momenta, masters and parameters are in use on this stream (None: the
        current one): dropping the optimizer does not hand them out before its work there is done."""
        at = _native.current_stream() if stream is None else stream.cuda_stream
        if at not in self._streams:
            s = _torch().cuda.current_stream() if stream is None else _as_stream(stream)
            for t in [self.workspace, *self.params, *self.masters, *self.momenta]:
                if t is not None:
                    t.record_stream(s)
            self._streams.add(at)

    def step(self, grads, lr: Optional[float] = None, grad_scale=None, stream=None):
        """One step with the gradients (fp32, fp16 or bf16 matrices of the parameters' shapes with
        unit column stride; None leaves a matrix and its momentum as they are).  ``grad_scale``: a
        device fp32 tensor whose first element multiplies every gradient."""
        count = len(self.params)
        if len(grads) != count:
            raise ValueError(f"one gradient per tensor ({count}), got {len(grads)}")
        _require_cuda(self.params[0])
        table = type(self._table).from_buffer_copy(self._table)
        for i, (g, p, row) in enumerate(zip(grads, self.params, table)):
            if g is None:
                continue
            _require_cuda(g)
            row.gdtype = _float_code(g, f"gradient {i}")
            if g.shape != p.shape:
                raise ValueError(f"gradient {i} must be {tuple(p.shape)}, got {tuple(g.shape)}")
            row.ld_grad = _unit_columns(g, f"gradient {i}")
            row.grad = g.data_ptr()
        self._hold_on(stream)
        _check(_lib.darb_muon_step(table, count, self.lr if lr is None else float(lr), self.momentum,
                                   int(self.nesterov), self.ns_steps, self.eps,
                                   _optional(grad_scale, 1, "grad_scale"), _ptr(self.workspace),
                                   self.workspace.numel(), _stream_ptr(stream)), "darb_muon_step")
