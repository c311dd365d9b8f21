"""Operators of a Peri-LN training step next to the optimizer, on torch
tensors: AdamW over many tensors, the boundary of a Peri-LN block, linear
layers in 8-bit floating point, orthogonalised updates of matrices and their
optimizer, the embedding of tokens, the cross entropy over a vocabulary.

As in ``optimizer.py``, torch only allocates device memory and supplies the
current HIP stream; the work runs in the library's kernels through
``mtdao_ops.py`` (include/mtdao_ops.h has the formulas).  Outputs and
workspaces are allocated from torch's caching allocator on the current
stream; inputs that belong to another stream are the caller's to order, as
for any torch operation.  What ``AdamW``, ``Muon``, ``Matrix8`` and ``Weight8`` allocate for
themselves is kept from the allocator until the streams of their calls are done
with it.  There is no CPU path.

``peri_norm``, ``linear8``, ``embedding`` and ``cross_entropy`` take part in autograd
where an input (of ``linear8``: x, or the tensor that its weight was made from)
requires a gradient; their backward passes are the functions of the same names
and not differentiable themselves.  Derivatives in forward mode are not given: a
tensor with a tangent is refused by these, ``orthogonalize`` and ``Weight8``.
"""

from __future__ import annotations

import functools
import math
from typing import Dict, List, Optional, Sequence, Tuple, Union

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version

from . import mtdao as abi
from . import mtdao_ops as c_ops

_TYPES = {torch.float32: abi.MTDAO_F32, torch.bfloat16: abi.MTDAO_BF16}
_KINDS = {"rms": c_ops.MTDAO_NORM_RMS, "layer": c_ops.MTDAO_NORM_LAYER}
CODE, SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = c_ops.MTDAO_BLOCK8


def _stream(t: torch.Tensor) -> int:
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _type(t: torch.Tensor, what: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32 or bfloat16, not {t.dtype}")
    return code


def _no_tangent(**tensors: Optional[torch.Tensor]) -> None:
    """Refuses tensors that carry a derivative in forward mode: the results would be
    without it.  (Called where there is a level of such derivatives: to look at a tensor
    takes 0.6 us, at the level 0.1 us.)"""
    for name, t in tensors.items():
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError(f"{name} has a tangent: derivatives in forward mode are not given; call with its detach()")


def _on_device(first: torch.Tensor, *others: Optional[torch.Tensor]) -> torch.device:
    """The HIP device that all of the tensors are on (None is skipped) and
    that is the current one."""
    index = first.get_device()
    for t in (first, *others):
        if t is not None and t.get_device() != index or index < 0:
            raise ValueError(f"a tensor is on {first.device if index < 0 else t.device}: the operators run on the GPU only, "
                             "all tensors of a call on one")
    if index != torch.cuda.current_device():
        raise ValueError(f"the tensors are on {first.device}, the current device is {torch.cuda.current_device()}")
    return first.device


# -------------------------------------------------------------- optimizers


class _Stepper:
    """What the optimizers share: a C handle over device memory that steps on
    any stream read."""

    handle: Optional[int] = None
    workspace: torch.Tensor

    def _stream_here(self) -> int:
        """The current stream, of the tensors' device.  On another one than that of construction the
        allocator learns of it: freed earlier, the table of addresses in the
        workspace would be another tensor's while a step still reads it."""
        if torch.cuda.current_device() != self.workspace.get_device():
            raise ValueError(f"the tensors are on {self.workspace.device}, the current device is {torch.cuda.current_device()}")
        stream = _stream(self.workspace)
        if stream not in self._streams:
            current = torch.cuda.current_stream(self.workspace.device)
            for t in self._own:
                t.record_stream(current)
            self._streams.add(stream)
        return stream

    def _grads_ok(self, grads, dtype) -> None:
        if len(grads) != len(self.params):
            raise ValueError(f"{len(grads)} gradients for {len(self.params)} parameters")
        _on_device(self.params[0], *grads)
        for i, (p, g) in enumerate(zip(self.params, grads)):
            if g.dtype != dtype or g.numel() != p.numel() or not g.is_contiguous():
                raise ValueError(f"grads[{i}]: gradients are contiguous, of one type and as large as their parameters")

    def _keep(self, own: List[torch.Tensor]) -> int:
        """Tensors allocated on the current stream, whose handle it returns, that steps use."""
        self._own = own
        home = _stream(self.workspace)
        self._streams = {home}
        return home

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class AdamW(_Stepper):
    """AdamW over a list of tensors, one launch for all of them (three with
    clipping); states in 32 or 8 bits (``state_bits``).

    ``params`` and ``grads`` are lists of contiguous tensors, each list of one
    type (float32 or bfloat16); the gradients are read from these tensors at
    every step until ``set_grads`` names others.  ``weight_decay`` is one
    value or one per tensor; ``max_norm`` > 0 clips by the global norm.
    ``states`` takes states to go on from (lists "m", "v", with 8 bits also
    "m_scale", "v_scale", as in the attributes of the same names), zeros
    otherwise.  8-bit states are e4m3 codes with an e8m0 scale per 128
    elements; v holds sqrt(v).
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], *,
                 betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: Union[float, Sequence[float]] = 0.0, max_norm: float = 0.0, state_bits: int = 32,
                 start_step: int = 0, states: Optional[Dict[str, List[torch.Tensor]]] = None):
        self.handle = None
        self.params = list(params)
        n = len(self.params)
        if n == 0:
            raise ValueError("no parameters")
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [float(weight_decay)] * n
        if len(decay) != n:
            raise ValueError(f"{len(decay)} values of weight_decay for {n} tensors")
        device = _on_device(*self.params)
        for i, p in enumerate(self.params):
            if p.dtype != self.params[0].dtype or not p.is_contiguous():
                raise ValueError(f"params[{i}]: parameters are contiguous and of one type")
        self._grads_ok(grads, torch.float32 if len(grads) == 0 else grads[0].dtype)
        self.grads = list(grads)
        eight = state_bits == 8
        kinds = {"m": CODE if eight else torch.float32, "v": CODE if eight else torch.float32}
        if eight:
            kinds.update(m_scale=SCALE, v_scale=SCALE)
        for name, dtype in kinds.items():
            sizes = [-(-p.numel() // BLOCK) if name.endswith("scale") else p.numel() for p in self.params]
            if states is None:
                made = [torch.zeros(s, dtype=torch.uint8 if eight else dtype, device=device).view(dtype) for s in sizes]
            else:
                made = list(states[name])
                _on_device(self.params[0], *made)
                if len(made) != n or any(t.dtype != dtype or t.numel() != s or not t.is_contiguous()
                                         for t, s in zip(made, sizes)):
                    raise ValueError(f"states['{name}']: {n} contiguous tensors of {dtype}, as large as their parameters "
                                     "(scales: one per 128 elements)")
            setattr(self, name, made)
        if not eight:
            self.m_scale = self.v_scale = None
        rows = (c_ops.AdamwTensor * n)()
        for i, r in enumerate(rows):
            r.p, r.g, r.m, r.v = (t[i].data_ptr() for t in (self.params, self.grads, self.m, self.v))
            if eight:
                r.m_scale, r.v_scale = self.m_scale[i].data_ptr(), self.v_scale[i].data_ptr()
            r.numel, r.weight_decay = self.params[i].numel(), decay[i]
        cfg = c_ops.AdamwConfig(_type(self.params[0], "params"), _type(self.grads[0], "grads"), state_bits, n, betas[0],
                                betas[1], eps, max_norm, start_step)
        need = c_ops.mtdao_adamw_workspace_bytes(cfg, rows)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)
        self._followed = [p for p in self.params if not p.is_inference()]  # by autograd
        home = self._keep([self.workspace] + ([t for name in kinds for t in getattr(self, name)] if states is None else []))
        self.handle = c_ops.mtdao_adamw_init(cfg, rows, self.workspace.data_ptr(), need, home)

    def set_grads(self, grads: Sequence[torch.Tensor]) -> None:
        """Take the gradients from these tensors from here on."""
        self._grads_ok(grads, self.grads[0].dtype)
        c_ops.mtdao_adamw_set_grads(self.handle, [g.data_ptr() for g in grads], self._stream_here())
        self.grads = list(grads)

    def step(self, lr: float) -> None:
        """One step.  To autograd it is a change in place: a backward pass over
        parameters from before it is refused."""
        c_ops.mtdao_adamw_step(self.handle, lr, self._stream_here())
        increment_version(self._followed)

    @property
    def step_count(self) -> int:
        return c_ops.mtdao_adamw_step_count(self.handle)

    def close(self) -> None:
        if self.handle:
            c_ops.mtdao_adamw_destroy(self.handle)
            self.handle = None


def orthogonalize(x: torch.Tensor, *, steps: int = 5, eps: float = 1e-7, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """x [..., r, c] with the singular values of each matrix moved to about 1 by
    ``steps`` Newton-Schulz products (include/mtdao_ops.h), in x's type unless
    ``dtype`` is given.  It is not differentiable."""
    if x.dim() < 2:
        raise ValueError(f"matrices are wanted, not {tuple(x.shape)}")
    if torch.is_grad_enabled() and x.requires_grad:
        raise ValueError("x requires a gradient, which orthogonalize does not give: call it on x.detach() or under no_grad")
    if forward_ad._current_level >= 0:
        _no_tangent(x=x)
    _on_device(x)
    x = x.contiguous()
    r, c = x.shape[-2:]
    batch = math.prod(x.shape[:-2])
    out = _empty(x, dtype or x.dtype)
    need = _orthogonalize_workspace(batch, r, c)
    ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    c_ops.mtdao_orthogonalize(x.data_ptr(), _type(x, "x"), batch, r, c, out.data_ptr(), _type(out, "dtype"), steps, eps, _ptr(ws), need,
                              _stream(x))
    return out


@functools.lru_cache(maxsize=256)
def _orthogonalize_workspace(batch: int, r: int, c: int) -> int:
    return c_ops.mtdao_orthogonalize_workspace_bytes(batch, r, c)


class Muon(_Stepper):
    """Momentum steps with orthogonalised updates, over a list of matrices at
    once:  m = momentum m + g,  u = g + momentum m (``nesterov``) or m,
    p = p (1 - lr weight_decay) - lr factor orthogonalize(u).

    ``params`` and ``grads`` are lists of contiguous matrices (with more than two
    axes: one for each index of the first ones), each list of one type (float32 or
    bfloat16); the gradients are read from these tensors at every step until
    ``set_grads`` names others.  ``weight_decay`` is one value or one per tensor;
    ``factor`` likewise, or "shape", max(1, rows / cols)^(1/2), or "rms", 0.2
    max(rows, cols)^(1/2), with which the root mean square of an update is about
    AdamW's.  ``states`` takes momenta to go on from (the list "m", float32), zeros otherwise.
    Embeddings, norms and other vectors are ``AdamW``'s.
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], *, momentum: float = 0.95, nesterov: bool = True,
                 weight_decay: Union[float, Sequence[float]] = 0.0, factor: Union[str, float, Sequence[float]] = "shape", steps: int = 5,
                 eps: float = 1e-7, states: Optional[Dict[str, List[torch.Tensor]]] = None):
        self.handle = None
        self.params = list(params)
        n = len(self.params)
        if n == 0:
            raise ValueError("no parameters")
        device = _on_device(*self.params)
        for i, p in enumerate(self.params):
            if p.dtype != self.params[0].dtype or not p.is_contiguous() or p.dim() < 2:
                raise ValueError(f"params[{i}]: parameters are contiguous matrices and of one type")
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [float(weight_decay)] * n
        if isinstance(factor, str):
            if factor not in ("shape", "rms"):
                raise ValueError(f"factor {factor!r} is not 'shape' or 'rms'")
            each = [math.sqrt(max(1.0, p.shape[-2] / max(1, p.shape[-1]))) if factor == "shape" else 0.2 * math.sqrt(max(p.shape[-2:]))
                    for p in self.params]
        else:
            each = list(factor) if isinstance(factor, (list, tuple)) else [float(factor)] * n
        if len(decay) != n or len(each) != n:
            raise ValueError(f"{len(decay)} values of weight_decay and {len(each)} of factor for {n} tensors")
        self._grads_ok(grads, torch.float32 if len(grads) == 0 else grads[0].dtype)
        self.grads = list(grads)
        if states is None:
            self.m = [torch.zeros(p.shape, dtype=torch.float32, device=device) for p in self.params]
        else:
            self.m = list(states["m"])
            _on_device(self.params[0], *self.m)
            if len(self.m) != n or any(m.dtype != torch.float32 or m.numel() != p.numel() or not m.is_contiguous()
                                       for m, p in zip(self.m, self.params)):
                raise ValueError(f"states['m']: {n} contiguous tensors of float32, as large as their parameters")
        self._batch = [math.prod(p.shape[:-2]) for p in self.params]
        rows = (c_ops.MuonMatrix * max(1, sum(self._batch)))()
        at = 0
        for i, p in enumerate(self.params):
            r, c = p.shape[-2:]
            for k in range(self._batch[i]):
                a = rows[at]
                a.p, a.g, a.m = (t.data_ptr() + k * r * c * t.element_size() for t in (p, self.grads[i], self.m[i]))
                a.rows, a.cols, a.weight_decay, a.factor = r, c, decay[i], each[i]
                at += 1
        cfg = c_ops.MuonConfig(_type(self.params[0], "params"), _type(self.grads[0], "grads"), max(1, at), bool(nesterov), steps, 0, momentum,
                               eps)
        need = c_ops.mtdao_muon_workspace_bytes(cfg, rows)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)
        self._followed = [p for p in self.params if not p.is_inference()]  # by autograd
        home = self._keep([self.workspace] + (self.m if states is None else []))
        self.handle = c_ops.mtdao_muon_init(cfg, rows, self.workspace.data_ptr(), need, home)

    def set_grads(self, grads: Sequence[torch.Tensor]) -> None:
        """Take the gradients from these tensors from here on."""
        self._grads_ok(grads, self.grads[0].dtype)
        at = [g.data_ptr() + k * (g.numel() // b) * g.element_size() for g, b in zip(grads, self._batch) for k in range(b)]
        c_ops.mtdao_muon_set_grads(self.handle, at or [None], self._stream_here())
        self.grads = list(grads)

    def step(self, lr: float) -> None:
        """One step.  To autograd it is a change in place: a backward pass over
        parameters from before it is refused."""
        c_ops.mtdao_muon_step(self.handle, lr, self._stream_here())
        increment_version(self._followed)

    def close(self) -> None:
        if self.handle:
            c_ops.mtdao_muon_destroy(self.handle)
            self.handle = None


# -------------------------------------------------------- Peri-LN boundary


def _rows(t: Optional[torch.Tensor], shape, what: str):
    """t, its address and row stride as [rows, d] with contiguous rows."""
    if t is None:
        return None, 0, shape[-1]
    if t.shape != shape:
        raise ValueError(f"{what} is {tuple(t.shape)}, not {tuple(shape)}")
    d = shape[-1]
    if t.is_contiguous():
        return t, t.data_ptr(), d
    t = t.reshape(-1, d)
    if t.stride(1) != 1 and d > 1 or t.shape[0] > 1 and t.stride(0) < d:
        t = t.contiguous()
    return t, t.data_ptr(), t.stride(0) if t.shape[0] > 1 else d


def _empty(like: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
    """A new contiguous tensor of like's shape (the way through ``empty_like`` takes
    half the host time, 1.2 us)."""
    if like.is_contiguous():
        return torch.empty_like(like) if like.dtype is dtype else torch.empty_like(like, dtype=dtype)
    return torch.empty(like.shape, dtype=dtype, device=like.device)


def _sums(w: torch.Tensor) -> torch.Tensor:
    """For the gradient of w: float32 along one axis."""
    g = _empty(w, torch.float32)
    return g if g.dim() == 1 else g.view(-1)


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _peri_sizes(x, f, w_post, w_pre, gate, rows_per_gate, kind):
    """rows, d, weight type, rows per gate of a call whose weights fit."""
    if kind not in _KINDS:
        raise ValueError(f"kind {kind!r} is not 'rms' or 'layer'")
    if (f is None) != (w_post is None):
        raise ValueError("f and w_post come together")
    if f is None and w_pre is None:
        raise ValueError("neither f nor w_pre is given")
    d = x.shape[-1]
    rows = x.numel() // d if d else 0
    weight = (w_post if w_post is not None else w_pre).dtype
    for name, w in (("w_post", w_post), ("w_pre", w_pre), ("gate", gate)):
        if w is None:
            continue
        if w.dtype != weight or not w.is_contiguous():
            raise ValueError(f"{name}: w_post, w_pre and gate are contiguous and of one type")
        if w is not gate and w.numel() != d:
            raise ValueError(f"{name} has {w.numel()} elements, rows have {d}")
    if weight not in _TYPES:
        raise TypeError(f"weights must be float32 or bfloat16, not {weight}")
    if gate is None:
        return rows, d, weight, 1
    per = max(1, rows) if rows_per_gate <= 0 else min(rows_per_gate, max(1, rows))
    if gate.numel() != max(1, -(-rows // per)) * d:
        raise ValueError(f"gate is {tuple(gate.shape)}: one row of {d} per {per} rows of {rows}")
    return rows, d, weight, per


def peri_norm(x: torch.Tensor, f: Optional[torch.Tensor], w_post: Optional[torch.Tensor],
              w_pre: Optional[torch.Tensor], *, gate: Optional[torch.Tensor] = None, rows_per_gate: int = 0,
              scale: float = 1.0, eps: float = 1e-5, kind: str = "rms",
              branch_dtype: Optional[torch.dtype] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """x' = x + scale gate norm(f) w_post and n = norm(x') w_pre over the last
    axis; returns (x', n).

    ``f`` None: x' is x (the first norm of a model).  ``w_pre`` None: n is
    None.  ``gate`` has one row of D per ``rows_per_gate`` rows of x (0: one
    row for all).  n has f's type (``branch_dtype``, x's by default, without
    f)."""
    if forward_ad._current_level >= 0:
        _no_tangent(x=x, f=f, w_post=w_post, w_pre=w_pre, gate=gate)
    if torch.is_grad_enabled() and (x.requires_grad or f is not None and f.requires_grad or w_pre is not None and w_pre.requires_grad or
                                    w_post is not None and w_post.requires_grad or gate is not None and gate.requires_grad):
        out, n = _PeriNorm.apply(x, f, w_post, w_pre, gate, rows_per_gate, scale, eps, kind, branch_dtype)
        return x if f is None else out, n
    _on_device(x, f, w_post, w_pre, gate)
    branch = f.dtype if f is not None else branch_dtype or x.dtype
    if branch not in _TYPES:
        raise TypeError(f"f must be float32 or bfloat16, not {branch}")
    rows, d, weight, per = _peri_sizes(x, f, w_post, w_pre, gate, rows_per_gate, kind)
    stream = _type(x, "x")
    shape = x.shape
    x_in, px, ld_x = _rows(x, shape, "x")
    f_in, pf, ld_f = _rows(f, shape, "f")
    out = _empty(x, x.dtype) if f is not None else x
    n = _empty(f if f is not None else x, branch) if w_pre is not None else None
    if rows:
        c_ops.mtdao_peri_norm(
            c_ops.PACKED_ARGS.pack(rows, d, _KINDS[kind], stream, _TYPES[branch], _TYPES[weight], eps, scale, per, ld_x, ld_f, d, d,
                                   px, pf, _ptr(w_post), _ptr(w_pre), _ptr(gate), 0, 0, out.data_ptr() if f is not None else 0,
                                   _ptr(n), 0, 0, 0, 0), _stream(x))
    return out, n


@functools.lru_cache(maxsize=256)
def _peri_workspace(rows: int, d: int, per: int, gated: bool) -> int:
    """Bytes for these sizes (every part given: at least what any call needs)."""
    some = 256  # stands for an address; only whether there is one is looked at
    return c_ops.mtdao_peri_norm_backward_workspace_bytes(
        c_ops.PACKED_ARGS.pack(rows, d, 0, 0, 0, 0, 0.0, 1.0, per, d, d, d, d, some, some, some, some, some if gated else 0,
                               *(0,) * 8))


def peri_norm_backward(d_out: Optional[torch.Tensor], dn: Optional[torch.Tensor], x_out: torch.Tensor,
                       f: Optional[torch.Tensor], w_post: Optional[torch.Tensor], w_pre: Optional[torch.Tensor], *,
                       gate: Optional[torch.Tensor] = None, rows_per_gate: int = 0, scale: float = 1.0,
                       eps: float = 1e-5, kind: str = "rms"):
    """Gradients of ``peri_norm`` from those of its outputs (either may be
    None: zero), its output x' and its input f: (dx, df, d_w_post, d_w_pre,
    d_gate), those of weights in float32, None for what was not given."""
    _on_device(x_out, f, w_post, w_pre, gate, d_out, dn)
    branch = f.dtype if f is not None else dn.dtype if dn is not None else x_out.dtype
    if branch not in _TYPES:
        raise TypeError(f"f must be float32 or bfloat16, not {branch}")
    if d_out is not None and d_out.dtype != x_out.dtype or dn is not None and dn.dtype != branch:
        raise TypeError("d_out has the type of x_out, dn that of f")
    rows, d, weight, per = _peri_sizes(x_out, f, w_post, w_pre, gate, rows_per_gate, kind)
    stream = _type(x_out, "x_out")
    shape, f32 = x_out.shape, torch.float32
    x_in, px, ld_x = _rows(x_out, shape, "x_out")
    f_in, pf, ld_f = _rows(f, shape, "f")
    d_in, pd, ld_d = _rows(d_out, shape, "d_out")
    y_in, py, ld_y = _rows(dn, shape, "dn")
    dx = _empty(x_out, x_out.dtype)
    df = _empty(f, branch) if f is not None else None
    dw_post = _sums(w_post) if f is not None else None
    dw_pre = _sums(w_pre) if w_pre is not None else None
    dgate = _empty(gate, f32) if gate is not None else None
    if rows == 0:
        for t in (dw_post, dw_pre, dgate):
            if t is not None:
                t.zero_()
        return dx, df, dw_post, dw_pre, dgate
    if d > c_ops.MTDAO_PERI_MAX_D:
        raise ValueError(f"rows of {d}: at most {c_ops.MTDAO_PERI_MAX_D}")
    need = _peri_workspace(rows, d, per, gate is not None)
    ws = torch.empty(need, dtype=torch.uint8, device=x_out.device)
    c_ops.mtdao_peri_norm_backward(
        c_ops.PACKED_ARGS.pack(rows, d, _KINDS[kind], stream, _TYPES[branch], _TYPES[weight], eps, scale, per, ld_x, ld_f, ld_d, ld_y,
                               px, pf, _ptr(w_post), _ptr(w_pre), _ptr(gate), pd, py, dx.data_ptr(), 0, _ptr(df), _ptr(dw_post),
                               _ptr(dw_pre), _ptr(dgate)), ws.data_ptr(), need, _stream(x_out))
    return dx, df, dw_post, dw_pre, dgate


class _PeriNorm(torch.autograd.Function):
    """peri_norm for autograd (x' only where there is an f: else it is x itself).
    A function's ``forward`` runs without gradients."""

    @staticmethod
    def forward(ctx, x, f, w_post, w_pre, gate, rows_per_gate, scale, eps, kind, branch_dtype):
        ctx.set_materialize_grads(False)
        ctx.how = {"rows_per_gate": rows_per_gate, "scale": scale, "eps": eps, "kind": kind}
        out, n = peri_norm(x, f, w_post, w_pre, gate=gate, branch_dtype=branch_dtype, **ctx.how)
        ctx.save_for_backward(out, f, w_post, w_pre, gate)
        return out if f is not None else None, n

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out, dn):
        out, f, *weights = ctx.saved_tensors
        dx, df, *sums = peri_norm_backward(d_out, dn, out, f, weights[0], weights[1], gate=weights[2], **ctx.how)
        sums = [None if w is None else s.view(w.shape).to(w.dtype) for s, w in zip(sums, weights)]
        return (*(g if needed else None for g, needed in zip((dx, df, *sums), ctx.needs_input_grad)), *(None,) * 5)


# ------------------------------------------------------------ 8-bit blocks


class Matrix8:
    """A [rows, cols] matrix of 8-bit blocks: ``codes`` (e4m3, [rows, cols up
    to a multiple of 128]) and ``scales`` (e8m0, one row per ``scale_rows``
    rows, one column per 128 columns up to a multiple of 4; a copy: they are
    held four columns by four).  Rows of codes are an odd number of blocks
    apart, which spreads them over the L2."""

    def __init__(self, rows: int, cols: int, device, scale_rows: int = 1):
        self.rows, self.cols, self.scale_rows = rows, cols, scale_rows
        blocks = -(-cols // BLOCK)
        ld = (blocks | 1) * BLOCK
        scale_ld = 4 * -(-rows // scale_rows)
        buf = torch.empty(rows * ld + -(-blocks // 4) * scale_ld, dtype=torch.uint8, device=device)
        self._buf = buf
        self._streams = {_stream(buf)}
        self.args = c_ops.Matrix8(buf.data_ptr(), buf.data_ptr() + rows * ld, rows, cols, ld, scale_ld, scale_rows)

    def on(self, stream: int) -> "c_ops.Matrix8":
        """The C structure, for a call on the current stream, whose handle is
        ``stream``: on another one than that of construction the allocator learns
        of it."""
        if stream not in self._streams:
            self._buf.record_stream(torch.cuda.current_stream(self._buf.device))
            self._streams.add(stream)
        return self.args

    @property
    def codes(self) -> torch.Tensor:
        a = self.on(_stream(self._buf))
        return self._buf[:a.rows * a.ld].view(CODE).view(a.rows, a.ld)[:, :-(-a.cols // BLOCK) * BLOCK]

    @property
    def scales(self) -> torch.Tensor:
        a = self.on(_stream(self._buf))
        fours, rows = -(-a.cols // (4 * BLOCK)), a.scale_ld // 4
        held = self._buf[a.rows * a.ld:].view(fours, rows, 4)
        return held.permute(1, 0, 2).reshape(rows, 4 * fours).view(SCALE)

    def dequantize(self) -> torch.Tensor:
        """The values as float32 [rows, cols]."""
        codes = self.codes.float().contiguous()
        s = self.scales.float()[:, :codes.shape[1] // BLOCK]
        if self.scale_rows > 1:
            s = s.repeat_interleave(self.scale_rows, 0)[:self.rows]
        return (codes.view(self.rows, codes.shape[1] // BLOCK, BLOCK) * s[:, :, None]).view(codes.shape)[:, :self.cols]


def _matrix(x: torch.Tensor) -> torch.Tensor:
    if x.dim() != 2:
        raise ValueError(f"a matrix is wanted, not {tuple(x.shape)}")
    if x.stride(1) != 1 and x.shape[1] > 1 or x.shape[0] > 1 and x.stride(0) < x.shape[1]:
        x = x.contiguous()
    return x


def _flat(x: torch.Tensor) -> torch.Tensor:
    """x [..., k] as a matrix [tokens, k] (k may be 0)."""
    return _matrix(x if x.dim() == 2 else x.reshape(math.prod(x.shape[:-1]), x.shape[-1]))


def _ld(x: torch.Tensor) -> int:
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


@functools.lru_cache(maxsize=256)
def _product_workspace(m: int, n: int, k: int) -> int:
    return c_ops.mtdao_product8_workspace_bytes(m, n, k)


@functools.lru_cache(maxsize=256)
def _linear_workspace(m: int, n: int, k: int) -> Tuple[int, int]:
    return c_ops.mtdao_linear8_workspace_bytes(m, n, k)


def _quantize(x: torch.Tensor, q: Optional[Matrix8], qt: Optional[Matrix8]) -> None:
    st = _stream(x)
    c_ops.mtdao_quantize8(x.data_ptr(), _type(x, "x"), _ld(x), q.on(st) if q is not None else None,
                          qt.on(st) if qt is not None else None, st)


def quantize8(x: torch.Tensor, *, rows: bool = True, transposed: bool = False):
    """x [r, c] as 8-bit blocks of 1 x 128: along its rows (``rows``), and/or
    transposed, along its columns (``transposed``).  Returns the one asked
    for, or both in one pass over x."""
    _on_device(x)
    x = _matrix(x)
    q = Matrix8(x.shape[0], x.shape[1], x.device) if rows else None
    qt = Matrix8(x.shape[1], x.shape[0], x.device) if transposed else None
    if q is None and qt is None:
        raise ValueError("neither rows nor transposed is asked for")
    _quantize(x, q, qt)
    return (q, qt) if rows and transposed else q if rows else qt


def product8(a: Matrix8, b: Matrix8, *, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
             accumulate: bool = False) -> torch.Tensor:
    """a b^T [a.rows, b.rows].  float32 results are float32 sums of exact products;
    bfloat16 ones, at twice the rate, leave out what lies more than 13 bits below
    the largest of each eight products: up to 4e-5 of the result's norm, next to
    1.7e-3 for their rounding.  ``out``: written in place of a new tensor (contiguous
    rows); ``accumulate``: added to (float32)."""
    given = out is not None
    if not given:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((a.rows, b.rows), dtype=dtype, device=a._buf.device)
    elif tuple(out.shape) != (a.rows, b.rows) or out.shape[1] > 1 and out.stride(1) != 1:
        raise ValueError(f"out is {tuple(out.shape)} with strides {out.stride()}, not [{a.rows}, {b.rows}] with contiguous rows")
    _on_device(out, a._buf, b._buf)
    need = _product_workspace(a.rows, b.rows, a.cols)
    ws = torch.empty(need, dtype=torch.uint8, device=out.device) if need else None
    st = _stream(out)
    c_ops.mtdao_product8(a.on(st), b.on(st), out.data_ptr(), _type(out, "out"), _ld(out), accumulate, _ptr(ws), need, st)
    if given and not out.is_inference():
        increment_version(out)
    return out


class Weight8:
    """The weight [out, in] of a linear layer in 8-bit blocks of 128 x 128,
    with its transpose for the gradient of the input (the same values).
    ``update`` takes the weight again after an optimizer step, in place.  In
    autograd the weight's gradient goes to the last tensor taken that required
    one (``source``)."""

    source: Optional[torch.Tensor] = None
    version = 0

    def __init__(self, w: torch.Tensor):
        if forward_ad._current_level >= 0:
            _no_tangent(w=w)
        _on_device(w)
        if w.requires_grad:
            self.source = w
        w = _matrix(w)
        self.q = Matrix8(w.shape[0], w.shape[1], w.device, BLOCK)
        self.qt = Matrix8(w.shape[1], w.shape[0], w.device, BLOCK)
        _quantize(w, self.q, self.qt)

    def update(self, w: torch.Tensor) -> None:
        if forward_ad._current_level >= 0:
            _no_tangent(w=w)
        _on_device(w, self.q._buf)
        if tuple(w.shape) != (self.q.rows, self.q.cols):
            raise ValueError(f"the weight is [{self.q.rows}, {self.q.cols}], not {tuple(w.shape)}")
        if w.requires_grad:
            self.source = w
        self.version += 1
        _quantize(_matrix(w), self.q, self.qt)


def linear8(x: torch.Tensor, w: Weight8, *, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """x W^T over the last axis of x, x in 8-bit blocks along it; in x's type
    unless ``dtype`` is given, which also says how it is summed (``product8``)."""
    if forward_ad._current_level >= 0:
        _no_tangent(x=x)
    if torch.is_grad_enabled() and (x.requires_grad or w.source is not None and w.source.requires_grad):
        return _Linear8.apply(x, w.source, w, dtype)
    wq = w.q
    if x.shape[-1] != wq.cols:
        raise ValueError(f"x has {x.shape[-1]} columns, the weight {wq.cols}")
    dev = _on_device(x, wq._buf)
    x2 = _flat(x)
    m = x2.shape[0]
    y = torch.empty((*x.shape[:-1], wq.rows), dtype=dtype or x.dtype, device=dev)
    need = _linear_workspace(m, wq.rows, wq.cols)[0]
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    st = _stream(x)
    c_ops.mtdao_linear8(x2.data_ptr(), _type(x, "x"), m, _ld(x2), wq.on(st), y.data_ptr(), _type(y, "dtype"), wq.rows, _ptr(ws), need, st)
    return y


def linear8_backward(dy: torch.Tensor, x: torch.Tensor, w: Weight8, *, dw: Optional[torch.Tensor] = None,
                     accumulate: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dx, dw) of ``linear8``: dx = dy W in dy's type, with dy in 8-bit
    blocks along its rows; dw = dy^T x in float32, with dy and x in 8-bit
    blocks along the tokens.  ``dw``: written in place of a new tensor
    (float32, contiguous rows); ``accumulate``: added to.  Sums are those of
    ``product8`` for these types (its float32 sums for a bfloat16 dy:
    ``product8(quantize8(dy), w.qt, dtype=torch.float32)``)."""
    n, k = w.q.rows, w.q.cols
    if x.shape[-1] != k or dy.shape[-1] != n or x.shape[:-1] != dy.shape[:-1]:
        raise ValueError(f"dy is {tuple(dy.shape)}, x {tuple(x.shape)}, the weight [{n}, {k}]")
    if dy.dtype != x.dtype:
        raise TypeError(f"dy is {dy.dtype}, x {x.dtype}")
    given = dw is not None
    if not given:
        if accumulate:
            raise ValueError("accumulate needs dw")
        dw = torch.empty((n, k), dtype=torch.float32, device=x.device)
    elif tuple(dw.shape) != (n, k) or k > 1 and dw.stride(1) != 1 or dw.dtype != torch.float32:
        raise ValueError(f"dw is {tuple(dw.shape)}, {dw.dtype} with strides {dw.stride()}, not float32 [{n}, {k}] with contiguous rows")
    dev = _on_device(x, dy, dw, w.qt._buf)
    x2 = _flat(x)
    dy2 = _flat(dy)
    m = x2.shape[0]
    dx = _empty(x, dy.dtype)
    need = _linear_workspace(m, n, k)[1]
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    st = _stream(x)
    c_ops.mtdao_linear8_backward(dy2.data_ptr(), x2.data_ptr(), _type(dy, "dy"), m, _ld(dy2), _ld(x2), w.qt.on(st), dx.data_ptr(), k,
                                 dw.data_ptr(), _ld(dw), accumulate, ws.data_ptr(), need, st)
    if given and not dw.is_inference():
        increment_version(dw)
    return dx, dw


class _Linear8(torch.autograd.Function):
    """linear8 for autograd; ``source`` takes the weight's gradient."""

    @staticmethod
    def forward(ctx, x, source, w, dtype):
        ctx.save_for_backward(x)
        ctx.w, ctx.version, ctx.type = w, w.version, source.dtype if source is not None else torch.float32
        return linear8(x, w, dtype=dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, = ctx.saved_tensors
        if ctx.w.version != ctx.version:
            raise RuntimeError("the weight has been updated since the forward pass that this gradient belongs to")
        kind = x.dtype if x.dtype == dy.dtype else torch.float32
        dx, dw = linear8_backward(dy.to(kind), x.to(kind), ctx.w)
        return dx.to(x.dtype) if ctx.needs_input_grad[0] else None, dw.to(ctx.type) if ctx.needs_input_grad[1] else None, None, None


# -------------------------------------------------------------- embedding


_BITS = {torch.int32: 32, torch.int64: 64}


def _ids(t: torch.Tensor, what: str) -> Tuple[torch.Tensor, int]:
    """t contiguous, and its bits."""
    bits = _BITS.get(t.dtype)
    if bits is None:
        raise TypeError(f"{what} must be int32 or int64, not {t.dtype}")
    return t.contiguous(), bits


def embedding(tokens: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """scale table[tokens]: tokens (int32 or int64) of any shape, a table [rows, d];
    in the table's type unless ``dtype`` is given.  A token below 0 stands for none:
    its row is zero.  One that the table does not have makes its row NaN."""
    if forward_ad._current_level >= 0:
        _no_tangent(table=table)
    if torch.is_grad_enabled() and table.requires_grad:
        return _Embedding.apply(tokens, table, scale, dtype)
    dev = _on_device(tokens, table)
    ids, bits = _ids(tokens, "tokens")
    w = _matrix(table)
    rows, d = w.shape
    out = torch.empty((*tokens.shape, d), dtype=dtype or table.dtype, device=dev)
    if out.numel():
        c_ops.mtdao_embedding(ids.data_ptr(), bits, ids.numel(), w.data_ptr(), _type(w, "table"), rows, d, _ld(w), scale, out.data_ptr(),
                              _type(out, "dtype"), d, _stream(out))
    return out


@functools.lru_cache(maxsize=256)
def _embedding_workspace(n: int, rows: int, d: int) -> int:
    return c_ops.mtdao_embedding_backward_workspace_bytes(n, rows, d)


def embedding_backward(dy: torch.Tensor, tokens: torch.Tensor, rows: int, *, scale: float = 1.0, dw: Optional[torch.Tensor] = None,
                       accumulate: bool = False) -> torch.Tensor:
    """The gradient of ``embedding``'s table of ``rows`` rows, in float32, from that
    of its output: scale times the sum of each token's rows of dy, in their order.  ``dw``: written in place
    of a new tensor (contiguous rows); ``accumulate``: added to, and rows whose token does not come are not touched."""
    d = dy.shape[-1]
    if dy.shape[:-1] != tokens.shape:
        raise ValueError(f"dy is {tuple(dy.shape)}, tokens {tuple(tokens.shape)}")
    given = dw is not None
    if not given:
        if accumulate:
            raise ValueError("accumulate needs dw")
        dw = torch.empty((rows, d), dtype=torch.float32, device=dy.device)
    elif tuple(dw.shape) != (rows, d) or d > 1 and dw.stride(1) != 1 or dw.dtype != torch.float32:
        raise ValueError(f"dw is {tuple(dw.shape)}, {dw.dtype} with strides {dw.stride()}, not float32 [{rows}, {d}] with contiguous rows")
    dev = _on_device(dy, tokens, dw)
    ids, bits = _ids(tokens, "tokens")
    kind = _type(dy, "dy")
    dy2 = _flat(dy)
    if dw.numel():
        need = _embedding_workspace(ids.numel(), rows, d)
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        c_ops.mtdao_embedding_backward(dy2.data_ptr(), kind, _ld(dy2), ids.data_ptr(), bits, ids.numel(), scale, dw.data_ptr(), rows, d,
                                       _ld(dw), accumulate, ws.data_ptr(), need, _stream(dy))
    if given and not dw.is_inference():
        increment_version(dw)
    return dw


class _Embedding(torch.autograd.Function):
    """embedding for autograd."""

    @staticmethod
    def forward(ctx, tokens, table, scale, dtype):
        ctx.save_for_backward(tokens)
        ctx.rows, ctx.scale, ctx.type = table.shape[0], scale, table.dtype
        return embedding(tokens, table, scale=scale, dtype=dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        tokens, = ctx.saved_tensors
        return None, embedding_backward(dy, tokens, ctx.rows, scale=ctx.scale).to(ctx.type), None, None


# ---------------------------------------------------------- cross entropy

_REDUCTIONS = {"none": c_ops.MTDAO_LOSS_NONE, "sum": c_ops.MTDAO_LOSS_SUM, "mean": c_ops.MTDAO_LOSS_MEAN}


@functools.lru_cache(maxsize=256)
def _loss_workspace(rows: int, cols: int, reduction: int) -> int:
    return c_ops.mtdao_cross_entropy_workspace_bytes(c_ops.PACKED_LOSS.pack(rows, cols, cols, cols, 0, 32, reduction, 0.0, 1.0, 0, *(0,) * 6))


def _loss(logits, targets, z_loss, reduction, *, loss=False, gradient=False, d_loss=None, scale=1.0, in_place=False):
    """The loss and/or the gradient of the logits, None for what is not asked for."""
    if reduction not in _REDUCTIONS:
        raise ValueError(f"reduction {reduction!r} is not 'none', 'sum' or 'mean'")
    if logits.shape[:-1] != targets.shape or logits.shape[-1] == 0:
        raise ValueError(f"logits are {tuple(logits.shape)}, targets {tuple(targets.shape)}: a row of at least one logit for each target")
    dev = _on_device(logits, targets, d_loss)
    ids, bits = _ids(targets, "targets")
    kind = _type(logits, "logits")
    x = _flat(logits)
    rows, cols = x.shape
    each = reduction == "none"
    made = torch.empty(targets.shape if each else (), dtype=torch.float32, device=dev) if loss else None
    d = None
    if gradient:
        d = logits if in_place else _empty(logits, logits.dtype)
        if in_place and x.data_ptr() != logits.data_ptr():
            raise ValueError(f"logits with strides {logits.stride()} cannot be written in place")
    if rows or made is not None and not each:
        how = _REDUCTIONS[reduction]
        need = _loss_workspace(rows, cols, how)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        ld, at = _ld(x), _ptr(made)
        c_ops.mtdao_cross_entropy(
            c_ops.PACKED_LOSS.pack(rows, cols, ld, ld if in_place else cols, kind, bits, how, z_loss, scale, 0, x.data_ptr(), ids.data_ptr(),
                                   _ptr(d_loss), at if each else 0, 0 if each else at, _ptr(d)), _ptr(ws), need, _stream(logits))
    if in_place and not logits.is_inference():
        increment_version(logits)
    return made, d


def cross_entropy(logits: torch.Tensor, targets: torch.Tensor, *, z_loss: float = 0.0, reduction: str = "mean") -> torch.Tensor:
    """lse - x_target + z_loss lse^2 of every row x of the logits [..., vocabulary],
    lse = log sum exp x, in float32: for each ("none"), their sum or their mean over
    the rows with a target.  A target (int32 or int64) below 0 stands for none:
    no loss, no gradient.  One that the row does not have gives NaN."""
    if forward_ad._current_level >= 0:
        _no_tangent(logits=logits)
    if torch.is_grad_enabled() and logits.requires_grad:
        return _CrossEntropy.apply(logits, targets, z_loss, reduction)
    return _loss(logits, targets, z_loss, reduction, loss=True)[0]


def cross_entropy_backward(d_loss: Optional[torch.Tensor], logits: torch.Tensor, targets: torch.Tensor, *, z_loss: float = 0.0,
                           reduction: str = "mean") -> torch.Tensor:
    """The gradient of the logits, in their type, from that of ``cross_entropy``'s
    result (float32; None: 1)."""
    if d_loss is not None:
        if d_loss.dtype != torch.float32 or d_loss.shape != (targets.shape if reduction == "none" else ()):
            raise ValueError(f"d_loss is {tuple(d_loss.shape)}, {d_loss.dtype}, not float32 of the loss's shape")
        d_loss = d_loss.contiguous()
    return _loss(logits, targets, z_loss, reduction, gradient=True, d_loss=d_loss)[1]


def cross_entropy_step(logits: torch.Tensor, targets: torch.Tensor, *, z_loss: float = 0.0, reduction: str = "mean", scale: float = 1.0,
                       in_place: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """(loss, gradient of the logits) of ``cross_entropy`` in one pass over the
    logits; the gradient is that of ``scale`` times the loss, with ``in_place``
    written over the logits.  Neither takes part in autograd."""
    return _loss(logits.detach(), targets, z_loss, reduction, loss=True, gradient=True, scale=scale, in_place=in_place)


class _CrossEntropy(torch.autograd.Function):
    """cross_entropy for autograd."""

    @staticmethod
    def forward(ctx, logits, targets, z_loss, reduction):
        ctx.save_for_backward(logits, targets)
        ctx.how = {"z_loss": z_loss, "reduction": reduction}
        return cross_entropy(logits, targets, **ctx.how)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_loss):
        return cross_entropy_backward(d_loss, *ctx.saved_tensors, **ctx.how), None, None, None
