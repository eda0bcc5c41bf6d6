"""The two ends of a training step over libarctopk: ``TokenLogProbs`` (log
probabilities of given tokens, entropy, top alternatives and their gradient)
and ``AdamW`` (gradient norms and the AdamW step over many tensors).

Both own one context of the C library, bound to a torch stream: inputs must be
ready on that stream, and outputs are.  Where it is not the current stream,
making them so (an event, a synchronization) is the caller's part.  Tensors may
be dropped after a call all the same: the allocator keeps inputs until the
context's stream is done with them, and outputs until the stream is that was
current at the call.  Tensors are checked here for what the library cannot see
in a pointer (type, device, shape, strides).
"""
from __future__ import annotations

import ctypes
from collections import namedtuple

import numpy as np
import torch

from . import _lib
from ._lib import (ARC_DTYPE_BF16, ARC_DTYPE_F32, ARC_STATE_BLOCK, ARC_STATE_F32, ARC_STATE_F8,
                   arc_adamw_config, arc_optim_adamw, arc_optim_create, arc_optim_destroy,
                   arc_optim_norm, arc_optim_state_elems, arc_optim_state_offset,
                   arc_tokens_create, arc_tokens_destroy, arc_tokens_grad, arc_tokens_loss,
                   arc_tokens_score, make_optim_config, make_tokens_config)

_DTYPES = {"f32": (ARC_DTYPE_F32, torch.float32), "bf16": (ARC_DTYPE_BF16, torch.bfloat16)}

Scores = namedtuple("Scores", "logp entropy lse top_ids top_logp")
Loss = namedtuple("Loss", "logp entropy lse grad")
Norms = namedtuple("Norms", "total norms")


class _Bound:
    """A context's device and stream."""

    def _bind(self, device, stream):
        self.device = torch.device(device or "cuda")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self.stream = stream or torch.cuda.current_stream(self.device)
        self._raw_stream = self.stream.cuda_stream

    def _check(self, name, x, dtype, count=None):
        if x.dtype != dtype or x.get_device() != self._index:  # (half the time of devices)
            raise ValueError(f"{name}: need {dtype} on {self.device}, got {x.dtype} on {x.device}")
        if not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if count is not None and x.numel() != count:
            raise ValueError(f"{name}: need {count} elements, got {x.numel()}")
        return x

    def _elsewhere(self):
        # (the raw handles compare in 0.1 us, stream objects in 2)
        return torch._C._cuda_getCurrentRawStream(self._index) != self._raw_stream

    def _empty(self, *shape, dtype=torch.float32):
        # memory of the stream that writes it
        if not self._elsewhere():
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            out = torch.empty(shape, dtype=dtype, device=self.device)
        out.record_stream(torch.cuda.current_stream(self.device))
        return out

    def _keep(self, *tensors):
        """What a call on another stream than the current one reads or writes:
        tensors, lists of them, None."""
        for x in tensors:
            for y in x if isinstance(x, (list, tuple)) else (x,):
                if y is not None:
                    y.record_stream(self.stream)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class TokenLogProbs(_Bound):
    """Scores rows of logits [T, V] (T at most ``rows``; "bf16" or "f32"; rows
    may lie further apart than V) against given tokens [T] int64, negative for
    a row without one.  The logits are multiplied with ``scale``."""

    def __init__(self, *, V, rows, dtype="bf16", top=0, scale=1.0, device=None, stream=None):
        self._bind(device, stream)
        self.V, self.rows, self.top, self.scale = V, rows, top, scale
        code, self.dtype = _DTYPES[dtype]
        with torch.cuda.device(self.device):
            self.ctx = arc_tokens_create(
                make_tokens_config(vocab=V, max_rows=rows, dtype=code, top=top, scale=scale),
                self.stream)

    def _rows(self, x, name="logits"):
        if x.dtype != self.dtype or x.device != self.device:
            raise ValueError(f"{name}: need {self.dtype} on {self.device}, got {x.dtype} on "
                             f"{x.device}")
        if x.dim() != 2 or x.shape[1] != self.V:
            raise ValueError(f"{name}: need [T, {self.V}], got {tuple(x.shape)}")
        T = x.shape[0]
        step, last = x.stride()
        if (last != 1 and self.V > 1) or (step < self.V and T > 1):
            raise ValueError(f"{name}: the elements of a row must follow one another")
        return T, max(step, self.V)

    def _each(self, name, x, T, dtype=torch.float32):
        return None if x is None else self._check(name, x, dtype, T)

    def score(self, logits, targets):
        """(logp, entropy, lse [T], top_ids int32 and top_logp [T, top])."""
        T, stride = self._rows(logits)
        self._each("targets", targets, T, torch.int64)
        k = T * self.top
        out = self._empty(3 * T + 2 * k)  # one allocation: a call of one row is mostly host time
        at = out.data_ptr()
        arc_tokens_score(self.ctx, T, logits.data_ptr(), stride, targets.data_ptr(), at,
                         at + 4 * T, at + 8 * T, at + 12 * T if k else None,
                         at + 12 * T + 4 * k if k else None)
        if self._elsewhere():
            self._keep(logits, targets)
        logp, entropy, lse, ids, near = out.split_with_sizes((T, T, T, k, k))
        return Scores(logp, entropy, lse, ids.view(torch.int32).view(T, self.top),
                      near.view(T, self.top))

    def grad(self, logits, targets, lse, entropy=None, d_logp=None, d_entropy=None, d_lse=None,
             out=None):
        """The gradient of scored rows [T, V] for upstream gradients [T], None
        for zeros.  ``out``: where to write it (the logits themselves allowed)."""
        T, stride = self._rows(logits)
        out, out_stride = self._out(out, T)
        each = self._each
        arc_tokens_grad(self.ctx, T, logits, stride, each("targets", targets, T, torch.int64),
                        each("lse", lse, T), each("entropy", entropy, T),
                        each("d_logp", d_logp, T), each("d_entropy", d_entropy, T),
                        each("d_lse", d_lse, T), out, out_stride)
        if self._elsewhere():
            self._keep(logits, targets, lse, entropy, d_logp, d_entropy, d_lse, out)
        return out

    def loss(self, logits, targets, d_logp=None, d_entropy=None, d_lse=None, out=None):
        """(logp, entropy, lse [T], grad [T, V]) for upstream gradients known
        beforehand."""
        T, stride = self._rows(logits)
        out, out_stride = self._out(out, T)
        each = self._each
        row = self._empty(3 * T)
        at = row.data_ptr()
        arc_tokens_loss(self.ctx, T, logits, stride, each("targets", targets, T, torch.int64),
                        each("d_logp", d_logp, T), each("d_entropy", d_entropy, T),
                        each("d_lse", d_lse, T), at, at + 4 * T, at + 8 * T, out, out_stride)
        if self._elsewhere():
            self._keep(logits, targets, d_logp, d_entropy, d_lse, out)
        return Loss(*row.split(T) if T else (row,) * 3, out)

    def _out(self, out, T):
        if out is None:
            return self._empty(T, self.V, dtype=self.dtype), self.V
        rows, stride = self._rows(out, "out")
        if rows != T:
            raise ValueError(f"out: need {T} rows, got {rows}")
        return out, stride

    def close(self):
        if getattr(self, "ctx", None):
            arc_tokens_destroy(self.ctx)
            self.ctx = None


def _state(name):
    return property(lambda self: self._states[name],
                    lambda self, x: self._take_state(name, x),
                    doc=f"{name} of all tensors; a tensor assigned here is what later steps use.")


class AdamW(_Bound):
    """AdamW over tensors of the given ``sizes``, with their states ``m``, ``v``
    and, in 8 bits, ``m_scale``, ``v_scale``.

    Parameters, gradients and copies are passed to each call, as a list of one
    tensor each or as one flat tensor that holds them in order.  ``param_dtype``
    and ``grad_dtype`` ("f32", "bf16"), ``weight_decay`` and ``lr_scale`` are
    one value for all tensors or a list.  ``state``: "f32" (m, v) or "f8" (m and
    sqrt(v) in 8 bits, m_scale and v_scale).  ``states``: a dict of existing
    ones, used in place; those that it lacks start at zero.
    """

    def __init__(self, sizes, *, param_dtype="f32", grad_dtype="f32", state="f32",
                 weight_decay=0.01, lr_scale=1.0, stochastic=False, seed=0, states=None,
                 device=None, stream=None):
        self._bind(device, stream)
        self.sizes = [int(n) for n in sizes]
        num = len(self.sizes)

        def each(v):
            return list(v) if isinstance(v, (list, tuple)) else [v] * num

        params, grads = each(param_dtype), each(grad_dtype)
        self._param = [_DTYPES[d][1] for d in params]
        self._grad = [_DTYPES[d][1] for d in grads]
        self.state = state
        cfg, keep = make_optim_config(
            counts=self.sizes, param_dtypes=[_DTYPES[d][0] for d in params],
            grad_dtypes=[_DTYPES[d][0] for d in grads], weight_decays=each(weight_decay),
            lr_scales=each(lr_scale),
            state={"f32": ARC_STATE_F32, "f8": ARC_STATE_F8}[state], stochastic=stochastic,
            seed=seed)
        with torch.cuda.device(self.device):
            self.ctx = arc_optim_create(cfg, self.stream)
        del keep
        S = arc_optim_state_elems(self.ctx)
        self.offsets = [arc_optim_state_offset(self.ctx, i) for i in range(num)]
        kind = torch.float8_e4m3fn if state == "f8" else torch.float32
        self._want = {"m": (kind, S), "v": (kind, S)}
        if state == "f8":
            self._want.update(m_scale=(torch.float32, S // ARC_STATE_BLOCK),
                              v_scale=(torch.float32, S // ARC_STATE_BLOCK))
        self._states = dict.fromkeys(("m", "v", "m_scale", "v_scale"))
        self._checked = None  # the states' addresses and lengths that were looked at last
        for name, (dtype, n) in self._want.items():
            x = None if states is None else states.get(name)
            if x is None:
                with torch.cuda.stream(self.stream):
                    x = torch.zeros(n, dtype=torch.uint8 if dtype.itemsize == 1 else dtype,
                                    device=self.device).view(dtype)
            self._take_state(name, x)
        starts = np.cumsum([0] + self.sizes[:-1], dtype=np.uint64)
        self._starts = {2: starts * np.uint64(2), 4: starts * np.uint64(4)}  # in bytes
        self._copy = [torch.bfloat16] * num
        self._one = {k: d[0] if len(set(d)) == 1 else None for k, d in (
            ("param", self._param), ("grad", self._grad), ("copy", self._copy))}
        self._table = {k: np.zeros(num, dtype=np.uint64) for k in ("param", "grad", "copy")}
        self._args = {k: ctypes.c_void_p(v.ctypes.data) for k, v in self._table.items()}
        self._flat = sum(self.sizes)

    m, v, m_scale, v_scale = (_state(name) for name in ("m", "v", "m_scale", "v_scale"))

    def _take_state(self, name, x):
        if name not in self._want:
            raise ValueError(f"{name}: states in {self.state!r} have none")
        self._states[name] = self._check(name, x, *self._want[name])
        self._held = [x for x in self._states.values() if x is not None]
        x.record_stream(self.stream)

    def _state_pointers(self):
        held = self._held
        now = [*map(torch.Tensor.data_ptr, held), *map(torch.Tensor.numel, held)]
        if now != self._checked:  # other tensors, or another storage of the same ones
            for name, want in self._want.items():
                self._check(name, self._states[name], *want)
            self._checked = now
        return now[:4] if len(held) == 4 else (now[0], now[1], None, None)

    def _pointers(self, key, x, dtypes):
        """Fills the host table of device pointers of this call."""
        table = self._table[key]
        if isinstance(x, torch.Tensor):  # flat
            dtype = self._one[key]
            if dtype is None:
                raise ValueError(f"{key}: one flat tensor holds one dtype")
            self._check(key, x, dtype, self._flat)
            np.add(self._starts[dtype.itemsize], x.data_ptr(), table)
        else:
            if len(x) != len(table):
                raise ValueError(f"{key}: need {len(table)} tensors, got {len(x)}")
            for i, (t, n, dtype) in enumerate(zip(x, self.sizes, dtypes)):
                if t is None and (key == "copy" or n == 0):
                    table[i] = 0
                else:
                    table[i] = self._check(f"{key}[{i}]", t, dtype, n).data_ptr()
        return self._args[key]

    def norm(self, grads, *, max_norm=float("inf"), scale=1.0):
        """(total [2], norms [num]): scale * the norm of all gradients and the
        factor for ``step`` that also clips it to max_norm, and scale * the norm
        of each tensor's."""
        num = len(self.sizes)
        out = self._empty(2 + num)
        at = out.data_ptr()
        arc_optim_norm(self.ctx, self._pointers("grad", grads, self._grad), scale, max_norm,
                       at + 8, at)
        if self._elsewhere():
            self._keep(grads)
        return Norms(*out.split_with_sizes((2, num)))

    def step(self, t, params, grads, *, lr, beta1=0.9, beta2=0.999, eps=1e-8, factor=None,
             copies=None):
        """One step t >= 0, in place.  ``factor``: norm()'s total [2], whose
        second value multiplies the gradients.  (In a captured graph every
        replay is this step again, t, lr and random bits with it.)"""
        at = None
        if factor is not None:
            at = self._check("factor", factor, torch.float32, 2).data_ptr() + 4
        arc_optim_adamw(
            self.ctx, arc_adamw_config(lr, beta1, beta2, eps), t,
            self._pointers("param", params, self._param),
            self._pointers("grad", grads, self._grad),
            None if copies is None else self._pointers("copy", copies, self._copy),
            at, *self._state_pointers())
        if self._elsewhere():
            self._keep(params, grads, copies, factor)

    def close(self):
        if getattr(self, "ctx", None):
            arc_optim_destroy(self.ctx)
            self.ctx = None
