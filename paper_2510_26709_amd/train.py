"""The two ends of a training step over libarctopk: ``TokenLogProbs`` (log
probabilities of given tokens, entropy, top alternatives and their gradient,
and the policy and preference losses made of them), ``AdamW`` (gradient norms
and the AdamW step over many tensors) and ``Muon`` (orthogonalised steps of
matrices).

Each owns one context of the C library, bound to a torch stream: inputs must be
ready on that stream, and outputs are.  Where it is not the current stream,
making them so (an event, a synchronization) is the caller's part.  A context has
one workspace: graphs captured from it, and calls, must not overlap in time.  Tensors
may be dropped after a call all the same: the allocator keeps inputs until the
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
from ._lib import (ARC_DTYPE_BF16, ARC_DTYPE_F32, ARC_POLICY_TOTALS, ARC_PREFERENCE_TOTALS,
                   ARC_STATE_BLOCK, ARC_STATE_F32, ARC_STATE_F8, PREFERENCES, arc_adamw_config,
                   arc_muon_create, arc_muon_destroy, arc_muon_orthogonalize,
                   arc_muon_state_elems, arc_muon_state_offset, arc_muon_step,
                   arc_muon_step_config, arc_optim_adamw, arc_optim_create, arc_optim_destroy,
                   arc_optim_norm, arc_optim_state_elems, arc_optim_state_offset,
                   arc_policy_config, arc_preference_config, arc_tokens_create,
                   arc_tokens_destroy, arc_tokens_grad, arc_tokens_loss, arc_tokens_policy,
                   arc_tokens_policy_terms, arc_tokens_preference, arc_tokens_preference_terms,
                   arc_tokens_score, make_muon_config, make_optim_config, make_tokens_config)

_DTYPES = {"f32": (ARC_DTYPE_F32, torch.float32), "bf16": (ARC_DTYPE_BF16, torch.bfloat16)}

Scores = namedtuple("Scores", "logp entropy lse top_ids top_logp")
Loss = namedtuple("Loss", "logp entropy lse grad")
Policy = namedtuple("Policy", "totals loss ratio kl d_logp d_entropy")
PolicyLoss = namedtuple("PolicyLoss", "totals logp entropy lse loss ratio kl grad")
Preference = namedtuple("Preference", "totals loss rewards d_logp")
PreferenceLoss = namedtuple("PreferenceLoss", "totals logp entropy lse loss rewards grad")
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

    def _at(self, name, x, count, dtype=torch.float32):
        """The address of a checked tensor; None for None."""
        return None if x is None else self._check(name, x, dtype, count).data_ptr()

    def _policy_inputs(self, T, targets, advantages, old_logp, ref_logp, weights):
        at = self._at
        return (at("targets", targets, T, torch.int64), at("old_logp", old_logp, T),
                at("ref_logp", ref_logp, T), at("advantages", advantages, T),
                at("weights", weights, T))

    def policy_loss(self, logits, targets, advantages, *, old_logp=None, ref_logp=None,
                    weights=None, clip_low=0.2, clip_high=0.2, dual=0.0, kl_coef=0.0,
                    entropy_coef=0.0, scale=1.0, out=None):
        """The clipped policy loss with a KL term and an entropy bonus: (totals
        [5]: loss, ratio, KL, entropy and clipped share, weighted; logp, entropy,
        lse, loss, ratio, kl [T]; grad [T, V], of the first total).  ``weights``
        [T] times ``scale`` is each token's part (scale = 1 / tokens for a mean);
        without ``old_logp`` the ratio is 1.  ``out``: where to write the gradient
        (the logits themselves allowed)."""
        T, stride = self._rows(logits)
        out, out_stride = self._out(out, T)
        y, old, ref, A, w = self._policy_inputs(T, targets, advantages, old_logp, ref_logp,
                                                weights)
        row = self._empty(6 * T + ARC_POLICY_TOTALS)
        at = [row.data_ptr() + 4 * k * T for k in range(7)]
        arc_tokens_policy(self.ctx, arc_policy_config(clip_low, clip_high, dual, kl_coef,
                                                      entropy_coef, scale),
                          T, logits.data_ptr(), stride, y, old, ref, A, w, *at, out.data_ptr(),
                          out_stride)
        if self._elsewhere():
            self._keep(logits, targets, old_logp, ref_logp, advantages, weights, out)
        *rows, totals = row.split_with_sizes((T,) * 6 + (ARC_POLICY_TOTALS,))
        return PolicyLoss(totals, *rows, out)

    def policy(self, logp, targets, advantages, *, entropy=None, old_logp=None, ref_logp=None,
               weights=None, clip_low=0.2, clip_high=0.2, dual=0.0, kl_coef=0.0,
               entropy_coef=0.0, scale=1.0):
        """The same from scored rows: (totals [5], loss, ratio, kl, d_logp and, where
        entropy_coef is not 0, d_entropy [T]); d_logp and d_entropy are for ``grad``."""
        T = targets.numel()
        y, old, ref, A, w = self._policy_inputs(T, targets, advantages, old_logp, ref_logp,
                                                weights)
        scored, H = self._at("logp", logp, T), self._at("entropy", entropy, T)
        n = 5 if entropy_coef else 4
        row = self._empty(n * T + ARC_POLICY_TOTALS)
        at = [row.data_ptr() + 4 * k * T for k in range(n + 1)]
        loss, ratio, kl, d_logp, *d_entropy, totals = at
        arc_tokens_policy_terms(self.ctx, arc_policy_config(clip_low, clip_high, dual, kl_coef,
                                                            entropy_coef, scale),
                                T, scored, H, y, old, ref, A, w, loss, ratio, kl, totals,
                                d_logp, d_entropy[0] if d_entropy else None)
        if self._elsewhere():
            self._keep(logp, entropy, targets, old_logp, ref_logp, advantages, weights)
        *rows, totals = row.split_with_sizes((T,) * n + (ARC_POLICY_TOTALS,))
        return Policy(totals, *rows, *(() if entropy_coef else (None,)))

    def _pairs(self, T, targets, offsets, ref_logp, weights):
        P = (offsets.numel() - 1) // 2
        if offsets.numel() != 2 * P + 1:
            raise ValueError(f"offsets: need 2 * pairs + 1 elements, got {offsets.numel()}")
        at = self._at
        return (P, at("targets", targets, T, torch.int64),
                at("offsets", offsets, 2 * P + 1, torch.int64), at("ref_logp", ref_logp, T),
                at("weights", weights, P))

    def preference_loss(self, logits, targets, offsets, *, ref_logp=None, weights=None,
                        kind="sigmoid", beta=0.1, margin=0.0, smoothing=0.0, average=False,
                        scale=1.0, out=None):
        """The loss of preferred and rejected answers by their paired log ratios:
        (totals [3]: loss, margin of the rewards and share of pairs whose preferred
        answer has the larger one, weighted; logp, entropy, lse [T]; loss [P];
        rewards [2 P]; grad [T, V], of the first total).  The rows are 2 P sequences
        one after the other, the preferred ones first; ``offsets`` [2 P + 1] int64,
        ascending in 0 .. T, says where they begin and end.  ``weights`` [P] times
        ``scale`` is each pair's part.  ``out``: where to write the gradient (the
        logits themselves allowed)."""
        T, stride = self._rows(logits)
        P, y, o, ref, w = self._pairs(T, targets, offsets, ref_logp, weights)
        out, out_stride = self._out(out, T)
        row = self._empty(3 * T + 3 * P + ARC_PREFERENCE_TOTALS)
        at = row.data_ptr()
        arc_tokens_preference(
            self.ctx, arc_preference_config(PREFERENCES[kind], average, beta, margin, smoothing,
                                            scale),
            T, logits.data_ptr(), stride, y, P, o, ref, w, at, at + 4 * T, at + 8 * T,
            at + 12 * T, at + 4 * (3 * T + P), at + 12 * (T + P), out.data_ptr(), out_stride)
        if self._elsewhere():
            self._keep(logits, targets, offsets, ref_logp, weights, out)
        *rows, totals = row.split_with_sizes((T, T, T, P, 2 * P, ARC_PREFERENCE_TOTALS))
        return PreferenceLoss(totals, *rows, out)

    def preference(self, logp, targets, offsets, *, ref_logp=None, weights=None, kind="sigmoid",
                   beta=0.1, margin=0.0, smoothing=0.0, average=False, scale=1.0):
        """The same from scored rows: (totals [3], loss [P], rewards [2 P], d_logp
        [T]); d_logp is for ``grad``."""
        T = targets.numel()
        P, y, o, ref, w = self._pairs(T, targets, offsets, ref_logp, weights)
        scored = self._at("logp", logp, T)
        row = self._empty(T + 3 * P + ARC_PREFERENCE_TOTALS)
        at = row.data_ptr()
        arc_tokens_preference_terms(
            self.ctx, arc_preference_config(PREFERENCES[kind], average, beta, margin, smoothing,
                                            scale),
            T, scored, y, P, o, ref, w, at + 4 * T, at + 4 * (T + P), at + 4 * (T + 3 * P), at)
        if self._elsewhere():
            self._keep(logp, targets, offsets, ref_logp, weights)
        d_logp, loss, rewards, totals = row.split_with_sizes(
            (T, P, 2 * P, ARC_PREFERENCE_TOTALS))
        return Preference(totals, loss, rewards, d_logp)

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


class _Optimizer(_Bound):
    """Tensors of given sizes that each call gets, and the states kept for them."""

    def _start(self, states):
        """Takes the states of ``_want``: name -> (dtype, elements)."""
        self._states = dict.fromkeys(self._names)
        self._checked = None  # the states' addresses and lengths that were looked at last
        for name, (dtype, n) in self._want.items():
            x = None if states is None else states.get(name)
            if x is None:
                with torch.cuda.stream(self.stream):
                    x = torch.zeros(n, dtype=torch.uint8 if dtype.itemsize == 1 else dtype,
                                    device=self.device).view(dtype)
            self._take_state(name, x)
        num = len(self.sizes)
        starts = np.cumsum([0] + self.sizes[:-1], dtype=np.uint64)
        self._starts = {2: starts * np.uint64(2), 4: starts * np.uint64(4)}  # in bytes
        self._copy = [torch.bfloat16] * num
        self._one = {k: d[0] if len(set(d)) == 1 else None for k, d in (
            ("param", self._param), ("grad", self._grad), ("copy", self._copy))}
        self._table = {k: np.zeros(num, dtype=np.uint64) for k in ("param", "grad", "copy")}
        self._args = {k: ctypes.c_void_p(v.ctypes.data) for k, v in self._table.items()}
        self._flat = sum(self.sizes)

    def _take_state(self, name, x):
        if name not in self._want:
            raise ValueError(f"{name}: there is no such state here")
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
        return now[:len(held)]

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
                elif t is None:
                    raise ValueError(f"{key}[{i}] is missing")
                else:
                    table[i] = self._check(f"{key}[{i}]", t, dtype, n).data_ptr()
        return self._args[key]


class AdamW(_Optimizer):
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
        self._start(states)

    _names = ("m", "v", "m_scale", "v_scale")
    m, v, m_scale, v_scale = (_state(name) for name in _names)

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
            at, *(*self._state_pointers(), None, None)[:4])
        if self._elsewhere():
            self._keep(params, grads, copies, factor)

    def close(self):
        if getattr(self, "ctx", None):
            arc_optim_destroy(self.ctx)
            self.ctx = None


class Muon(_Optimizer):
    """Orthogonalised updates of matrices of the given ``shapes``, with their
    momenta ``m``.

    Parameters, gradients and copies are passed to each call as ``AdamW`` takes
    them, a list of one tensor each or one flat tensor; ``param_dtype``,
    ``grad_dtype``, ``weight_decay`` and ``lr_scale`` are one value for all
    matrices or a list.  A tensor of more than one dimension has a matrix's rows
    first (a convolution's weight is [out, in * height * width]).  ``lr_scale``
    None: sqrt(max(1, rows / cols)).
    ``coefficients``: a, b, c of one Newton-Schulz step, or of each of ``steps``.
    ``states``: a dict with existing momenta, used in place; else they start at
    zero.

    Steps are as exact as binary32 products make them where a parameter is "f32";
    where all are "bf16", O may be off by 1e-4 of its norm before it is rounded.
    Making one takes the host some milliseconds, which serve all later calls.
    """

    _names = ("m",)
    m = _state("m")

    def __init__(self, shapes, *, param_dtype="f32", grad_dtype="f32", weight_decay=0.0,
                 lr_scale=None, steps=5, coefficients=None, states=None, device=None,
                 stream=None):
        self._bind(device, stream)
        self.shapes = [(int(r), int(c)) for r, c in shapes]
        self.sizes = [r * c for r, c in self.shapes]
        num = len(self.shapes)

        def each(v):
            return list(v) if isinstance(v, (list, tuple)) else [v] * num

        if lr_scale is None:
            lr_scale = [max(1.0, r / max(c, 1)) ** 0.5 for r, c in self.shapes]
        params, grads = each(param_dtype), each(grad_dtype)
        self._param = [_DTYPES[d][1] for d in params]
        self._grad = [_DTYPES[d][1] for d in grads]
        cfg, keep = make_muon_config(
            shapes=self.shapes, param_dtypes=[_DTYPES[d][0] for d in params],
            grad_dtypes=[_DTYPES[d][0] for d in grads], weight_decays=each(weight_decay),
            lr_scales=each(lr_scale), steps=steps, coefficients=coefficients)
        with torch.cuda.device(self.device):
            self.ctx = arc_muon_create(cfg, self.stream)
        del keep
        self.offsets = [arc_muon_state_offset(self.ctx, i) for i in range(num)]
        self._want = {"m": (torch.float32, arc_muon_state_elems(self.ctx))}
        self._start(states)

    def _pointers(self, key, x, dtypes):
        if not isinstance(x, torch.Tensor):
            for i, (t, (rows, _)) in enumerate(zip(x, self.shapes)):
                if t is not None and t.dim() != 1 and (t.dim() == 0 or t.shape[0] != rows):
                    raise ValueError(f"{key}[{i}]: need {self.shapes[i]}, got {tuple(t.shape)}")
        return super()._pointers(key, x, dtypes)

    def orthogonalize(self, x, out=None):
        """The orthogonalised matrices, in the parameters' dtypes: one flat tensor
        for one, else a list.  ``out``: where to write them."""
        if out is None:
            if isinstance(x, torch.Tensor):
                if self._one["param"] is None:
                    raise ValueError("param: one flat tensor holds one dtype")
                out = self._empty(self._flat, dtype=self._one["param"])
            else:
                out = [self._empty(*s, dtype=d) for s, d in zip(self.shapes, self._param)]
        arc_muon_orthogonalize(self.ctx, self._pointers("grad", x, self._grad),
                               self._pointers("param", out, self._param))
        if self._elsewhere():
            self._keep(x, out)
        return out

    def step(self, params, grads, *, lr, momentum=0.95, nesterov=True, factor=None, copies=None):
        """One step, in place.  ``factor``: a total [2] of ``AdamW.norm``, whose
        second value multiplies the gradients."""
        at = None
        if factor is not None:
            at = self._check("factor", factor, torch.float32, 2).data_ptr() + 4
        arc_muon_step(self.ctx, arc_muon_step_config(lr, momentum, nesterov, 0),
                      self._pointers("param", params, self._param),
                      self._pointers("grad", grads, self._grad),
                      None if copies is None else self._pointers("copy", copies, self._copy),
                      at, *self._state_pointers())
        if self._elsewhere():
            self._keep(params, grads, copies, factor)

    def close(self):
        if getattr(self, "ctx", None):
            arc_muon_destroy(self.ctx)
            self.ctx = None
