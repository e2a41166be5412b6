"""The operators of a residual gated block (include/enova_block.h) on torch tensors.

Each class owns one library handle; its methods check and marshal their arguments and call the C
entry points on torch's current stream (or the one given). All computation happens in the
library's HIP kernels. Matrices are two-dimensional, in the handle's type, with neighbouring
columns next to each other in memory; where a method says so, rows may be further apart.

A method that is given a stream works there as torch's own operations do under ``torch.cuda.stream``: what
it returns is allocated on that stream, and the caller orders the stream after the work that makes the
arguments, and keeps them until the work is done. Calls on one object share its workspace and must not
overlap: order their streams, or take an object a stream. An object whose calls were captured into a graph
has to outlive the graph, and a replay counts as such a call.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from .binding import (ENOVA_BF16, ENOVA_F32, _check, _on, enova_adamw_config, enova_gated_config, enova_i8_config,
                      enova_resnorm_config, lib)

__all__ = ["GatedBlock", "ResidualNorm", "AdamW", "Int8Linear", "quantize_weight"]

ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}
NORMS = {"rms": 0, "layer": 1}
_TYPES = {"f32": (ENOVA_F32, torch.float32), "bf16": (ENOVA_BF16, torch.bfloat16)}
_CODES = {torch.float32: ENOVA_F32, torch.bfloat16: ENOVA_BF16}


def _known(value, table, what):
    if value not in table:
        raise ValueError(f"{what} {value!r}: one of {', '.join(map(repr, table))}")
    return table[value]


class _Handle:
    """One library handle, on the device that was current when the object was made."""
    handle = None

    def __init__(self):
        self._device = torch.cuda.current_device()

    def _open(self, name, *args):
        h = ctypes.c_void_p()
        _check(getattr(lib(), f"enova_{name}_init")(*args, ctypes.byref(h)), f"enova_{name}_init")
        self.handle, self._name = h.value, name

    def _matrix(self, t, dtype, cols, what, rows=None):
        """(pointer, row pitch) of a matrix on the handle's device whose rows may be apart."""
        if (t.get_device() != self._device or t.dtype != dtype or t.dim() != 2 or t.shape[1] != cols
                or (rows is not None and t.shape[0] != rows)):
            raise ValueError(f"{what}: expected a matrix of {cols} columns{'' if rows is None else f' and {rows} rows'} "
                             f"in {dtype} on cuda:{self._device}, got {tuple(t.shape)} {t.dtype} on {t.device}")
        row, col = t.stride()
        if (col != 1 and cols > 1) or (row < cols and t.shape[0] > 1):
            raise ValueError(f"{what}: columns have to be next to each other, and rows must not overlap")
        return t.data_ptr(), max(row, cols)

    def _dense(self, t, dtype, shape, what):
        """Pointer of a contiguous tensor on the handle's device (None -> NULL)."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self._device or not t.is_contiguous():
            raise ValueError(f"{what}: expected a contiguous tensor of shape {shape} in {dtype} on cuda:{self._device}, "
                             f"got {tuple(t.shape)} {t.dtype} on {t.device}")
        return t.data_ptr()

    def _flat(self, tensors, dtypes, what, sizes):
        """Their pointers, after a check of a list of contiguous tensors on the handle's device."""
        if len(tensors) != len(sizes):
            raise ValueError(f"{what}: {len(tensors)} tensors for {len(sizes)} parameters")
        for i, t in enumerate(tensors):
            if t.dtype not in dtypes or t.numel() != sizes[i] or t.get_device() != self._device or not t.is_contiguous():
                raise ValueError(f"{what}[{i}]: expected a contiguous tensor of {sizes[i]} elements in "
                                 f"{' or '.join(map(str, dtypes))} on cuda:{self._device}")
        return [t.data_ptr() for t in tensors]

    def _queue(self, stream):
        """The stream given, or torch's current one on the handle's device."""
        return (torch.cuda.current_stream(self._device) if stream is None else stream).cuda_stream

    def close(self):
        if self.handle:
            _check(getattr(lib(), f"enova_{self._name}_destroy")(self.handle), f"enova_{self._name}_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GatedBlock(_Handle):
    """y = (act(x Wg^T) * (x Wu^T)) Wd^T and its gradients; wg, wu [hidden, model], wd [model, hidden]."""

    def __init__(self, model, hidden, dtype="bf16", act="silu"):
        code, self.dtype = _known(dtype, _TYPES, "dtype")
        super().__init__()
        self.model, self.hidden = model, hidden
        self._open("gated", ctypes.byref(enova_gated_config(model, hidden, code, _known(act, ACTIVATIONS, "activation"))))

    def _weights(self, wg, wu, wd):
        up = (self.hidden, self.model)
        return (self._dense(wg, self.dtype, up, "wg"), self._dense(wu, self.dtype, up, "wu"),
                self._dense(wd, self.dtype, (self.model, self.hidden), "wd"))

    def saved(self, rows, device="cuda", stream=None):
        """A buffer for what forward leaves for backward (g, u and h)."""
        with _on(stream):
            return torch.empty(self._saved_floats(rows), dtype=torch.float32, device=device)

    def _saved_floats(self, rows):
        n = ctypes.c_int64()
        _check(lib().enova_gated_saved_floats(self.handle, rows, ctypes.byref(n)), "enova_gated_saved_floats")
        return n.value

    def _kept(self, saved, rows):
        return None if saved is None else self._dense(saved, torch.float32, (self._saved_floats(rows),), "saved")

    def forward(self, x, wg, wu, wd, save=False, y=None, saved=None, stream=None):
        """y, or (y, saved) with ``save`` (or a buffer from ``saved(rows)`` to save in). Rows of x and y may be apart."""
        px, ldx = self._matrix(x, self.dtype, self.model, "x")
        rows = x.shape[0]
        if y is None:
            with _on(stream):
                y = torch.empty((rows, self.model), dtype=self.dtype, device=x.device)
        py, ldy = self._matrix(y, self.dtype, self.model, "y", rows)
        if save and saved is None:
            saved = self.saved(rows, x.device, stream)
        _check(lib().enova_gated_forward(self.handle, px, ldx, rows, *self._weights(wg, wu, wd), py, ldy,
                                         self._kept(saved, rows), self._queue(stream)), "enova_gated_forward")
        return y if saved is None else (y, saved)

    def backward(self, x, wg, wu, wd, dy, saved=None, input_grad=True, weight_grads=True, stream=None):
        """(dx, dwg, dwu, dwd); None for those not asked for. Without ``saved`` g and u are computed again."""
        px, ldx = self._matrix(x, self.dtype, self.model, "x")
        rows = x.shape[0]
        pdy, lddy = self._matrix(dy, self.dtype, self.model, "dy", rows)
        with _on(stream):
            dx = torch.empty((rows, self.model), dtype=self.dtype, device=x.device) if input_grad else None
            dw = [torch.empty_like(w) for w in (wg, wu, wd)] if weight_grads else [None] * 3
        _check(lib().enova_gated_backward(self.handle, px, ldx, rows, *self._weights(wg, wu, wd),
                                          self._kept(saved, rows), pdy, lddy,
                                          None if dx is None else dx.data_ptr(), self.model,
                                          *(None if d is None else d.data_ptr() for d in dw), self._queue(stream)),
               "enova_gated_backward")
        return (dx, *dw)


class ResidualNorm(_Handle):
    """res = keep * residual + scale * gate * N(branch; post), out = N(res; pre), and the gradients.

    norm: "rms" or "layer". post may be None (no norm before the gate), biases and gate too; row r takes
    gate row r // group."""

    def __init__(self, model, dtype="bf16", norm="rms", eps=1e-5, keep=1.0, scale=1.0, group=0):
        code, self.dtype = _known(dtype, _TYPES, "dtype")
        super().__init__()
        self.model, self.group = model, group
        self._open("resnorm", ctypes.byref(enova_resnorm_config(model, code, _known(norm, NORMS, "norm"), eps, keep,
                                                                scale, group)))

    def _vector(self, t, what):
        return self._dense(t, torch.float32, (self.model,), what)

    def _gate(self, gate, rows):
        if gate is not None and self.group < 1:
            raise ValueError("a gate needs a group of 1 row or more")
        return None if gate is None else self._dense(gate, torch.float32, (-(-rows // self.group), self.model), "gate")

    def forward(self, residual, branch, post, pre, post_bias=None, pre_bias=None, gate=None, stream=None):
        """(res, out, stats); stats is for backward."""
        shape = (residual.shape[0], self.model)
        rows = shape[0]
        with _on(stream):
            res, out = torch.empty_like(residual), torch.empty_like(residual)
            stats = torch.empty((rows, 4), dtype=torch.float32, device=residual.device)
        _check(lib().enova_resnorm_forward(
            self.handle, self._dense(residual, self.dtype, shape, "residual"),
            self._dense(branch, self.dtype, shape, "branch"), rows, self._vector(post, "post"), self._vector(post_bias, "post_bias"), self._vector(pre, "pre"),
            self._vector(pre_bias, "pre_bias"), self._gate(gate, rows), res.data_ptr(), out.data_ptr(),
            stats.data_ptr(), self._queue(stream)), "enova_resnorm_forward")
        return res, out, stats

    def backward(self, residual, branch, post, pre, post_bias, pre_bias, dres, dout, stats, gate=None, stream=None):
        """A dict of gradients: "dr" and "do" of residual and branch, "dpre", and "dpost", "dpost_bias",
        "dpre_bias", "dgate" of those that are there."""
        shape = (residual.shape[0], self.model)
        rows, dev = shape[0], residual.device
        self._vector(pre_bias, "pre_bias")     # its gradient's shape, and nothing else
        with _on(stream):
            g = {"dr": torch.empty_like(residual), "do": torch.empty_like(residual),
                 "dpre": torch.empty(self.model, dtype=torch.float32, device=dev)}
            for name, t in (("dpost", post), ("dpost_bias", post_bias), ("dpre_bias", pre_bias), ("dgate", gate)):
                if t is not None:
                    g[name] = torch.empty_like(t)
        p = {k: t.data_ptr() for k, t in g.items()}
        _check(lib().enova_resnorm_backward(
            self.handle, self._dense(residual, self.dtype, shape, "residual"),
            self._dense(branch, self.dtype, shape, "branch"), rows, self._vector(post, "post"), self._vector(post_bias, "post_bias"), self._vector(pre, "pre"),
            self._gate(gate, rows), self._dense(stats, torch.float32, (rows, 4), "stats"),
            self._dense(dres, self.dtype, shape, "dres"), self._dense(dout, self.dtype, shape, "dout"), p["dr"], p["do"],
            p.get("dpost"), p.get("dpost_bias"), p["dpre"], p.get("dpre_bias"), p.get("dgate"), self._queue(stream)),
            "enova_resnorm_backward")
        return g


class AdamW(_Handle):
    """AdamW over a list of tensors in one launch, states in 32 or 8 bits.

    params (all fp32 or all bf16) and grads are kept and updated where they are; copies: bf16 tensors that
    receive the rounded fp32 parameters. States are made as zeros, or given: m and v in fp32, or for 8 bits m in
    int8, v in uint8 and both scales in fp32, one for each 256 elements."""

    def __init__(self, params, grads, copies=None, bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, decay=0.01,
                 m=None, v=None, m_scale=None, v_scale=None):
        if not params:
            raise ValueError("no parameters")
        if bits not in (32, 8):
            raise ValueError(f"states of {bits} bits: 32 or 8")
        super().__init__()
        dev, sizes = params[0].device, [p.numel() for p in params]

        def made(given, dtype, per=1):
            return [torch.zeros(-(-n // per), dtype=dtype, device=dev) for n in sizes] if given is None else list(given)

        self.params, self.grads, self.copies, self.bits = list(params), list(grads), copies and list(copies), bits
        self.m = made(m, torch.int8 if bits == 8 else torch.float32)
        self.v = made(v, torch.uint8 if bits == 8 else torch.float32)
        self.m_scale = made(m_scale, torch.float32, 256) if bits == 8 else None
        self.v_scale = made(v_scale, torch.float32, 256) if bits == 8 else None
        self._sizes, self._grad_type = sizes, self.grads[0].dtype if self.grads else torch.float32
        blocks = [-(-n // 256) for n in sizes]
        lists = [self._flat(self.params, (torch.float32,) if params[0].dtype == torch.float32 else (torch.bfloat16,),
                       "params", sizes),
                 self._flat(self.grads, (self._grad_type,) if self._grad_type in _CODES else tuple(_CODES), "grads", sizes),
                 self._flat(self.copies, (torch.bfloat16,), "copies", sizes) if self.copies else [None] * len(sizes),
                 self._flat(self.m, (self.m[0].dtype if m is None else torch.int8 if bits == 8 else torch.float32,), "m", sizes),
                 self._flat(self.v, (torch.uint8 if bits == 8 else torch.float32,), "v", sizes)]
        lists += ([self._flat(self.m_scale, (torch.float32,), "m_scale", blocks),
                   self._flat(self.v_scale, (torch.float32,), "v_scale", blocks)]
                  if bits == 8 else [[None] * len(sizes)] * 2)
        # rows of enova_adamw_tensor: seven pointers and a length
        rows = np.array([[x or 0 for x in row] for row in zip(*lists, sizes)], dtype=np.int64)
        table = rows.ctypes.data_as(ctypes.c_void_p)
        self.lr, self.steps = lr, 0
        self._open("adamw", ctypes.byref(enova_adamw_config(bits, _CODES[params[0].dtype], _CODES[self._grad_type], b1,
                                                            b2, eps, decay)), table, len(sizes))

    def set_grads(self, grads, stream=None):
        """Other gradient tensors for the steps from here on."""
        p = self._flat(grads, (self._grad_type,), "grads", self._sizes)
        _check(lib().enova_adamw_set_grads(self.handle, (ctypes.c_void_p * len(p))(*p), self._queue(stream)),
               "enova_adamw_set_grads")
        if stream is not None:                 # steps queued there may still read the old ones
            for t in self.grads:
                t.record_stream(stream)
        self.grads = list(grads)

    def step(self, lr=None, grad_scale=1.0, stream=None):
        """The next step, with gradients times ``grad_scale``."""
        _check(lib().enova_adamw_step(self.handle, self.steps + 1, self.lr if lr is None else lr, grad_scale,
                                      self._queue(stream)), "enova_adamw_step")
        self.steps += 1

    def states(self, m=None, v=None, stream=None):
        """The values of m and v in fp32, into the lists given: for checkpoints, and to look at 8-bit states."""
        if self.bits == 32 and m is None and v is None:
            return self.m, self.v
        with _on(stream):
            m, v = ([torch.empty_like(p, dtype=torch.float32) for p in self.params] if t is None else t for t in (m, v))
        pm, pv = (self._flat(t, (torch.float32,), "states", self._sizes) for t in (m, v))
        n = len(pm)
        _check(lib().enova_adamw_states(self.handle, (ctypes.c_void_p * n)(*pm), (ctypes.c_void_p * n)(*pv),
                                        self._queue(stream)), "enova_adamw_states")
        return m, v


def quantize_weight(w):
    """(codes [outputs, inputs] int8 in rows of whole 16 bytes, scales [outputs]) of a weight matrix."""
    w = w.float()
    top = w.abs().amax(1)
    codes = torch.zeros(w.shape[0], -(-w.shape[1] // 16) * 16, dtype=torch.int8, device=w.device)[:, :w.shape[1]]
    codes.copy_(torch.round(w / torch.where(top > 0, top, 1.0)[:, None] * 127))
    return codes, top / 127


class Int8Linear(_Handle):
    """y = x W^T + bias with W as int8 codes and a scale for each output, x quantised row by row.

    codes and scales as ``quantize_weight`` gives them; they are kept, not copied. gate: the activation
    with which x's two halves [g | u] make act(g) * u first."""

    def __init__(self, codes, scales, bias=None, dtype="bf16", gate=None):
        code, self.dtype = _known(dtype, _TYPES, "dtype")
        super().__init__()
        self.outputs, self.inputs = codes.shape
        p, ld = self._matrix(codes, torch.int8, self.inputs, "codes")
        self.codes, self.scales, self.bias = codes, scales, bias
        self.columns = self.inputs * (1 if gate is None else 2)
        self._open("i8", ctypes.byref(enova_i8_config(self.inputs, self.outputs, code,
                                                      -1 if gate is None else _known(gate, ACTIVATIONS, "activation"))),
                   p, ld, self._dense(scales, torch.float32, (self.outputs,), "scales"),
                   self._dense(bias, torch.float32, (self.outputs,), "bias"))

    def __call__(self, x, y=None, stream=None):
        """y [rows, outputs]; rows of x and y may be apart."""
        px, ldx = self._matrix(x, self.dtype, self.columns, "x")
        if y is None:
            with _on(stream):
                y = torch.empty((x.shape[0], self.outputs), dtype=self.dtype, device=x.device)
        py, ldy = self._matrix(y, self.dtype, self.outputs, "y", x.shape[0])
        _check(lib().enova_i8_forward(self.handle, px, ldx, x.shape[0], py, ldy, self._queue(stream)), "enova_i8_forward")
        if stream is not None:                 # the handle may go before the product is done
            for t in (self.codes, self.scales, self.bias):
                if t is not None:
                    t.record_stream(stream)
        return y
