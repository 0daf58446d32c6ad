"""Training of the expert estimator (paper: Sec. 6, Appendix A) and of routers: torch tensors into the operators of
include/moe_spec_train.h.  Torch supplies memory and streams; the operators are the library's kernels.

Every function queues its kernels on the current stream of its tensors' device and returns tensors that are valid in that
stream's order; tensors of another stream are the caller's to order and to keep, as with torch's own operations.  Gradients are
results of explicit calls (a loss returns its own, `layernorm_backward` takes one): nothing here records or reads an autograd
graph, and results have none.  What is written in place (`out`, AdamW's parameters and copies) counts as changed for graphs that have
kept it: their backward pass raises torch's error, as after torch's own operations.  The functions and AdamW's calls can be captured into a graph."""
from __future__ import annotations

import ctypes as C
from array import array
from operator import attrgetter, index
from typing import List, Optional, Sequence

import torch
from torch.autograd.graph import increment_version

from . import moe_spec as M

# what is asked of every tensor of a list, by map
_NUMEL, _CONTIGUOUS, _DEVICE, _ADDRESS, _DTYPE = (torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.get_device, torch.Tensor.data_ptr,
                                                  attrgetter("dtype"))
_TYPES = {torch.float32: M.F32, torch.bfloat16: M.BF16}


def _queue(dev: torch.device, call, *args):
    """call(stream, *args) on the current stream of the tensors' device, with that device as the current one."""
    i = dev.index
    if torch._C._cuda_getDevice() == i:
        M._check_train(call(torch._C._cuda_getCurrentRawStream(i), *args))
    else:
        with torch.cuda.device(i):
            M._check_train(call(torch._C._cuda_getCurrentRawStream(i), *args))


def _rows(t: torch.Tensor, name: str, like: Optional[torch.Tensor] = None) -> int:
    """Type number of a matrix whose rows are contiguous."""
    dtype = _TYPES.get(t.dtype)
    if dtype is None or t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a two-dimensional float32 or bfloat16 tensor on a GPU")
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise ValueError(f"{name}: the values of a row must be contiguous")
    if like is not None and (t.shape != like.shape or t.device != like.device):
        raise ValueError(f"{name} must have the shape and the device of the other matrix")
    return dtype


def _vector(t: Optional[torch.Tensor], name: str, n: int, dev: torch.device, dtype=torch.float32):
    if t is None:
        return None
    if t.dtype != dtype or t.dim() != 1 or t.numel() != n or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{name} must be a contiguous {dtype} vector of {n} values on {dev}")
    return t.data_ptr()


def _mask(valid: Optional[torch.Tensor], rows: int, dev: torch.device):
    if valid is None:
        return None
    if valid.dtype not in (torch.bool, torch.uint8):
        raise ValueError("valid must be a bool or uint8 vector")
    return _vector(valid, "valid", rows, dev, valid.dtype)


def layernorm_forward(x: torch.Tensor, gain: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                      eps: float = 1e-5, *, out: Optional[torch.Tensor] = None):
    """LayerNorm over the last dimension of x [rows, cols] (rows may be strided) -> (y, mean [rows], rstd [rows]).  gain and
    bias: float32 [cols] or None.  out: where y goes, x itself included."""
    dtype = _rows(x, "x")
    rows, cols = x.shape
    dev = x.device
    given = out is not None
    if not given:
        out = x.new_empty((rows, cols))
    elif _rows(out, "out", x) != dtype:
        raise ValueError("out must have the type of x")
    elif out.requires_grad and torch.is_grad_enabled():
        raise ValueError("out requires a gradient, and what is written there would not be in its graph")
    mean, rstd = x.new_empty((2, rows), dtype=torch.float32).unbind(0)
    at = mean.data_ptr()
    _queue(dev, M.lib().moe_spec_layernorm_forward, dtype, x.data_ptr(), x.stride(0), rows, cols, _vector(gain, "gain", cols, dev),
           _vector(bias, "bias", cols, dev), eps, out.data_ptr(), out.stride(0), at, at + 4 * rows)
    if given:
        increment_version(out)
    return out, mean, rstd


def layernorm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                       gain: Optional[torch.Tensor] = None, *, input_grad: bool = True, weight_grads: bool = True):
    """Gradients of LayerNorm for dy [rows, cols], with x, mean and rstd of the forward pass -> (dx, dgain, dbias): dx in x's
    type, the weights' float32 [cols], summed over the rows in an order of their own (the same bits every time).  None in the
    place of what is not asked for."""
    dtype = _rows(x, "x")
    if _rows(dy, "dy", x) != dtype:
        raise ValueError("dy must have the type of x")
    rows, cols = x.shape
    dev = x.device
    lib = M.lib()
    dx = x.new_empty((rows, cols)) if input_grad else None
    dgain = dbias = space = at = None
    need = 0
    if weight_grads:
        dgain, dbias = x.new_empty((2, cols), dtype=torch.float32).unbind(0)
        at = dgain.data_ptr()
        need = lib.moe_spec_layernorm_backward_workspace_bytes(rows, cols)
        space = x.new_empty(need, dtype=torch.uint8) if need else None
    _queue(dev, lib.moe_spec_layernorm_backward, dtype, dy.data_ptr(), dy.stride(0), x.data_ptr(), x.stride(0), rows, cols,
           _vector(mean, "mean", rows, dev), _vector(rstd, "rstd", rows, dev), _vector(gain, "gain", cols, dev),
           dx.data_ptr() if input_grad else None, cols, at, at + 4 * cols if weight_grads else None,
           space.data_ptr() if need else None, need)
    return dx, dgain, dbias


def distill_loss(student: torch.Tensor, teacher: torch.Tensor, *, temperature: float = 1.0,
                 valid: Optional[torch.Tensor] = None, grad: bool = True):
    """Mean over the valid rows of KL(softmax(teacher / temperature) || softmax(student / temperature)) for logits
    [rows, experts] -> (loss, its gradient with respect to the student's logits, in their type, or None)."""
    ts, tt = _rows(student, "student"), _rows(teacher, "teacher", student)
    rows, experts = student.shape
    dev = student.device
    lib = M.lib()
    mask = _mask(valid, rows, dev)
    loss = student.new_empty((), dtype=torch.float32)
    dz = student.new_empty((rows, experts)) if grad else None
    need = lib.moe_spec_distill_loss_workspace_bytes(rows, experts)
    space = student.new_empty(need, dtype=torch.uint8) if need else None
    _queue(dev, lib.moe_spec_distill_loss, ts, student.data_ptr(), student.stride(0), tt, teacher.data_ptr(), teacher.stride(0),
           rows, experts, temperature, mask, loss.data_ptr(), dz.data_ptr() if grad else None, experts,
           space.data_ptr() if need else None, need)
    return loss, dz


def balance_loss(logits: torch.Tensor, ids: torch.Tensor, *, coef: float = 1.0, valid: Optional[torch.Tensor] = None,
                 grad: bool = True):
    """coef * experts * sum_e f_e P_e for logits [rows, experts] and the experts that each row chose, ids int32 [rows, k]
    -> (loss, counts int32 [experts], gradient with respect to the logits or None)."""
    dtype = _rows(logits, "logits")
    rows, experts = logits.shape
    dev = logits.device
    if ids.dtype != torch.int32 or ids.dim() != 2 or ids.shape[0] != rows or ids.device != dev:
        raise ValueError("ids must be an int32 tensor [rows, k] on the logits' device")
    k = ids.shape[1]
    if ids.stride(1) != 1 and k > 1:
        raise ValueError("ids: the values of a row must be contiguous")
    lib = M.lib()
    mask = _mask(valid, rows, dev)
    loss = logits.new_empty((), dtype=torch.float32)
    counts = logits.new_empty(experts, dtype=torch.int32)
    dz = logits.new_empty((rows, experts)) if grad else None
    need = lib.moe_spec_balance_loss_workspace_bytes(rows, experts, k)
    space = logits.new_empty(need, dtype=torch.uint8) if need else None
    _queue(dev, lib.moe_spec_balance_loss, dtype, logits.data_ptr(), logits.stride(0), rows, experts, ids.data_ptr(), ids.stride(0),
           k, coef, mask, loss.data_ptr(), counts.data_ptr(), dz.data_ptr() if grad else None, experts,
           space.data_ptr() if need else None, need)
    return loss, counts, dz


class AdamW:
    """AdamW over many float32 tensors in one call, moments in 32 ("f32") or 8 bits ("f8").  Holds the tensors and their
    moments; `lr`, `betas`, `eps` and `weight_decay` may be set between steps.  A captured step keeps those it was captured with;
    its number and grad_scale it reads anew where they are tensors.

    copies: bfloat16 tensors (or None in places) that get the updated parameters, rounded: what an Engine reads its weights
    from.  states: moments to go on with, as `states()` of another AdamW gave them; used in place."""

    def __init__(self, params: Sequence[torch.Tensor], *, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, state: str = "f32", copies: Optional[Sequence[Optional[torch.Tensor]]] = None,
                 seed: int = 0, states: Optional[dict] = None, steps: int = 0):
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        if state not in ("f32", "f8"):
            raise ValueError('state must be "f32" or "f8"')
        self.lr, self.betas, self.eps, self.weight_decay = lr, betas, eps, weight_decay
        self.state, self.seed, self.steps = state, int(seed) & 0xffffffff, int(steps)
        dev = self.device = self.params[0].device
        self._sizes = [p.numel() for p in self.params]
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        eight = state == "f8"
        if states is None:
            new = lambda n, t: torch.zeros(n, dtype=t, device=dev)  # noqa: E731
            states = {k: [new(n, torch.uint8 if eight else torch.float32) for n in self._sizes] for k in ("m", "v")}
            if eight:
                states.update({k: [new(-(-n // M.MOMENT_BLOCK), torch.uint8) for n in self._sizes] for k in ("m_exp", "v_exp")})
        self._states = {k: list(states[k]) for k in (("m", "v", "m_exp", "v_exp") if eight else ("m", "v"))}
        if any(len(t) != len(self.params) for t in (*self._states.values(), self.copies)):
            raise ValueError("as many moments and copies as parameters are needed")
        self._moments = [t for k in self._states.values() for t in k]
        self._written = [t for t in (*self.params, *self.copies) if t is not None]
        self._held = [*self._moments, *self._written]
        self._at = self._at_moments = None
        self._desc = (M.AdamWTensor * len(self.params))()
        self._entries = list(self._desc)                       # views of the table's entries
        self._whole = False                                    # whether each entry's n is its tensor's
        self._config = M.AdamWConfig(seed=self.seed, moments=M.MOMENTS_8BIT if eight else M.MOMENTS_32BIT)
        self._describe(self._held)

    def _tensor(self, t, name, dtype, n):
        if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.device != self.device or not t.is_cuda:
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} values on the parameters' GPU")

    def _tensors(self, tensors, name, dtype, sizes):
        """_tensor of each of them."""
        if not (list(map(_NUMEL, tensors)) == sizes and all(map(_CONTIGUOUS, tensors)) and set(map(_DTYPE, tensors)) == {dtype}
                and set(map(_DEVICE, tensors)) == {self.device.index}):
            for t, n in zip(tensors, sizes):
                self._tensor(t, name, dtype, n)

    def states(self) -> dict:
        """The moments: m and v, with 8 bits their codes and m_exp and v_exp."""
        return {k: list(t) for k, t in self._states.items()}

    def _describe(self, held):
        """The tensors' table for the library; made anew where one of those that a call needs has got other storage since."""
        if list(map(_ADDRESS, held)) == (self._at if held is self._held else self._at_moments):
            return
        s = self._states
        for i, (d, p) in enumerate(zip(self._entries, self.params)):
            d.p, d.m, d.v = p.data_ptr(), s["m"][i].data_ptr(), s["v"][i].data_ptr()
            if self.state == "f8":
                d.m_exp, d.v_exp = s["m_exp"][i].data_ptr(), s["v_exp"][i].data_ptr()
            d.copy = self.copies[i].data_ptr() if self.copies[i] is not None else None
        self._check()
        self._at, self._at_moments = list(map(_ADDRESS, self._held)), list(map(_ADDRESS, self._moments))

    def _check(self):
        eight = self.state == "f8"
        held = torch.uint8 if eight else torch.float32
        for i, p in enumerate(self.params):
            self._tensor(p, "a parameter", torch.float32, self._sizes[i])
            for k, t in self._states.items():
                self._tensor(t[i], k, held, -(-p.numel() // M.MOMENT_BLOCK) if k.endswith("exp") else p.numel())
            if self.copies[i] is not None:
                self._tensor(self.copies[i], "a copy", torch.bfloat16, p.numel())
        written = [t.data_ptr() for t in self._held if t.numel()]
        if len(set(written)) < len(written):
            raise ValueError("a tensor is named twice")

    def _all_whole(self):
        if not self._whole:
            for d, n in zip(self._entries, self._sizes):
                d.n = n
            self._whole = True

    def step(self, grads: Sequence[Optional[torch.Tensor]], *, step=None, grad_scale=1.0):
        """One step with a gradient for each parameter, all float32 or all bfloat16; a parameter whose gradient is None stays as
        it is.  step: the step's number, counted from 1 (by itself if left out), or an int64 tensor on the GPU that the kernels
        read it from, which a captured graph needs.  grad_scale: a factor of the gradients, a number or a float32 tensor on the GPU."""
        if len(grads) != len(self.params):
            raise ValueError("as many gradients as parameters are needed")
        given = [g for g in grads if g is not None]
        dtype = given[0].dtype if given else torch.float32
        if dtype not in _TYPES:
            raise ValueError("gradients must be float32 or bfloat16")
        all_given = len(given) == len(grads)
        self._tensors(given, "a gradient", dtype, self._sizes if all_given else [n for n, g in zip(self._sizes, grads) if g is not None])
        self._describe(self._held)
        self._all_whole()
        if all_given:
            for d, at in zip(self._entries, map(_ADDRESS, grads)):
                d.grad = at
        else:
            self._whole = False
            for d, g in zip(self._entries, grads):
                if g is None:
                    d.n = 0
                else:
                    d.grad = g.data_ptr()
        c = self._config
        c.lr, (c.beta1, c.beta2), c.eps, c.weight_decay, c.grad_dtype = self.lr, self.betas, self.eps, self.weight_decay, _TYPES[dtype]
        c.step_dev = c.grad_scale_dev = None
        c.grad_scale = 1.0
        if isinstance(grad_scale, torch.Tensor):
            self._tensor(grad_scale, "grad_scale", torch.float32, 1)
            c.grad_scale_dev = grad_scale.data_ptr()
        else:
            c.grad_scale = grad_scale
        if isinstance(step, torch.Tensor):
            self._tensor(step, "step", torch.int64, 1)
            c.step_dev = step.data_ptr()
        else:
            c.step = self.steps + 1 if step is None else step
        _queue(self.device, M.lib().moe_spec_adamw_step, self._desc, len(self._desc), C.byref(c))
        if not isinstance(step, torch.Tensor):
            self.steps = c.step
        increment_version(self._written if all_given else [t for i, g in enumerate(grads) if g is not None
                                                           for t in (self.params[i], self.copies[i]) if t is not None])

    def read_moments(self, m_out: Optional[List[torch.Tensor]] = None, v_out: Optional[List[torch.Tensor]] = None):
        """The values of 8-bit moments, into float32 or bfloat16 tensors (which hold all of them from 2^-120 on exactly) or new
        float32 ones -> (m, v)."""
        if self.state != "f8":
            raise ValueError("32-bit moments are tensors of their own: states()")
        if m_out is None and v_out is None:
            m_out, v_out = ([torch.empty_like(p) for p in self.params] for _ in range(2))
        n = len(self.params)
        if (m_out is not None and len(m_out) != n) or (v_out is not None and len(v_out) != n):
            raise ValueError("a tensor for each parameter is needed")
        outs = [*(m_out or ()), *(v_out or ())]
        dtype = outs[0].dtype
        if dtype not in _TYPES:
            raise ValueError("moments are read as float32 or bfloat16")
        self._tensors(outs, "an output", dtype, self._sizes * (len(outs) // n))
        self._describe(self._moments)
        self._all_whole()
        at = (C.c_void_p * n * (len(outs) // n)).from_buffer(array("Q", map(_ADDRESS, outs)))
        _queue(self.device, M.lib().moe_spec_adamw_read_moments, self._desc, n, _TYPES[dtype], at[0] if m_out is not None else None,
               at[-1] if v_out is not None else None)
        return m_out, v_out


def _out(out: Optional[torch.Tensor], name: str, shape, dtype: torch.dtype, like: torch.Tensor) -> torch.Tensor:
    """The tensor that a result goes to: a new one, or the given one."""
    if out is None:
        return like.new_empty(shape, dtype=dtype)
    if out.shape != shape or out.dtype != dtype or out.device != like.device or (out.stride(-1) != 1 and out.shape[-1] > 1):
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {like.device} whose rows are contiguous")
    if out.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, and what is written there would not be in its graph")
    return out


def _groups(ends: torch.Tensor, experts: int, dev: torch.device):
    if not 1 <= experts <= M.MAX_EXPERTS:
        raise ValueError(f"between 1 and {M.MAX_EXPERTS} experts are taken")
    return _vector(ends, "ends", experts, dev, torch.int32)


def grouped_product(x: torch.Tensor, w: torch.Tensor, ends: torch.Tensor, *, transpose: bool = False,
                    dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Products of rows that are sorted by expert with the experts' matrices w [experts, n, k]: w_e x_r for x [rows, k] -> [rows, n],
    or w_e^T x_r for x [rows, n] -> [rows, k] with transpose, the gradient with respect to the other form's x.  Expert e has the
    rows from ends[e - 1] (0 for the first) to ends[e], ends int32 [experts] on the GPU; rows behind the last become zero.
    x and w are both float32 or both bfloat16, rows and matrices may be strided (a part of larger expert blocks, one row for all);
    dtype: the result's type, x's own if left out."""
    t = _rows(x, "x")
    if w.dim() != 3 or w.dtype != x.dtype or w.device != x.device or (w.stride(2) != 1 and w.shape[2] > 1):
        raise ValueError("w must be a three-dimensional tensor of the type and on the device of x, whose rows are contiguous")
    experts, n, k = w.shape
    if x.shape[1] != (n if transpose else k):
        raise ValueError(f"x must have {n if transpose else k} columns")
    kind = x.dtype if dtype is None else dtype
    if kind not in _TYPES:
        raise ValueError("results are float32 or bfloat16")
    at = _groups(ends, experts, x.device)
    given = out is not None
    out = _out(out, "out", (x.shape[0], k if transpose else n), kind, x)
    _queue(x.device, M.lib().moe_spec_grouped_product, t, x.data_ptr(), x.stride(0), x.shape[0], w.data_ptr(), w.stride(1), w.stride(0),
           experts, n, k, at, bool(transpose), _TYPES[kind], out.data_ptr(), out.stride(0))
    if given:
        increment_version(out)
    return out


def grouped_weight_grad(dy: torch.Tensor, x: torch.Tensor, ends: torch.Tensor, *, dtype: Optional[torch.dtype] = None,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradients of the experts' matrices, [experts, n, k]: the sum of dy_r x_r^T over each expert's rows, for dy [rows, n] and
    x [rows, k] sorted by expert as for grouped_product; zeros for an expert without rows.  dtype: the result's type, x's own if left
    out.  out: where it goes, for instance a part of larger blocks."""
    t = _rows(x, "x")
    if _rows(dy, "dy") != t or dy.device != x.device or dy.shape[0] != x.shape[0]:
        raise ValueError("dy must have the type, the device and the rows of x")
    kind = x.dtype if dtype is None else dtype
    if kind not in _TYPES:
        raise ValueError("results are float32 or bfloat16")
    experts, n, k = ends.numel(), dy.shape[1], x.shape[1]
    at = _groups(ends, experts, x.device)
    given = out is not None
    out = _out(out, "out", (experts, n, k), kind, x)
    lib = M.lib()
    need = lib.moe_spec_grouped_weight_grad_workspace_bytes(t, x.shape[0], experts, n, k)
    space = x.new_empty(need, dtype=torch.uint8) if need else None
    _queue(x.device, lib.moe_spec_grouped_weight_grad, t, dy.data_ptr(), dy.stride(0), x.data_ptr(), x.stride(0), x.shape[0], experts,
           n, k, at, _TYPES[kind], out.data_ptr(), out.stride(1), out.stride(0), space.data_ptr() if need else None, need)
    if given:
        increment_version(out)
    return out


def _gate_up(a: torch.Tensor):
    t = _rows(a, "a")
    if a.shape[1] % 2 or a.shape[1] == 0:
        raise ValueError("a must hold as many columns of the gate as of the up projection")
    return t, a.shape[0], a.shape[1] // 2


def swiglu_forward(a: torch.Tensor, weight: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The experts' activation, silu(gate) * up for a [rows, 2 cols] = gate | up -> [rows, cols].  weight: float32 [rows] or None, a
    factor of each row: the mixing weights may be applied here, as the down projection is linear."""
    t, rows, cols = _gate_up(a)
    h = a.new_empty((rows, cols))
    _queue(a.device, M.lib().moe_spec_swiglu_forward, t, a.data_ptr(), a.stride(0), rows, cols, _vector(weight, "weight", rows, a.device),
           h.data_ptr(), cols)
    return h


def swiglu_backward(dh: torch.Tensor, a: torch.Tensor, weight: Optional[torch.Tensor] = None):
    """Gradients of swiglu_forward for dh [rows, cols] -> (da [rows, 2 cols], dweight float32 [rows], None without a weight)."""
    t, rows, cols = _gate_up(a)
    if _rows(dh, "dh") != t or dh.shape != (rows, cols) or dh.device != a.device:
        raise ValueError("dh must have the type, the device and the rows of a, and half its columns")
    da = a.new_empty((rows, 2 * cols))
    dweight = None if weight is None else a.new_empty(rows, dtype=torch.float32)
    _queue(a.device, M.lib().moe_spec_swiglu_backward, t, dh.data_ptr(), dh.stride(0), a.data_ptr(), a.stride(0), rows, cols,
           _vector(weight, "weight", rows, a.device), da.data_ptr(), 2 * cols, None if weight is None else dweight.data_ptr())
    return da, dweight


ORTHOGONALISE = (3.4445, -4.7750, 2.0315)          # coefficients of its iteration


def _three(coefficients):
    c = tuple(coefficients)
    if len(c) != 3:
        raise ValueError("the iteration has three coefficients")
    return (C.c_double * 3)(*c)


def orthogonalise(g: torch.Tensor, *, iterations: int = 5, coefficients=ORTHOGONALISE, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Matrices [rows, cols] or stacks of them [count, rows, cols], float32 or bfloat16, with their singular values pushed towards one
    -> bfloat16, of g's shape.  Formula and accuracy are in include/moe_spec_train.h."""
    dtype, c = _TYPES.get(g.dtype), _three(coefficients)
    if dtype is None or g.dim() not in (2, 3) or not g.is_cuda or (g.stride(-1) != 1 and g.shape[-1] > 1):
        raise ValueError("g must be a float32 or bfloat16 matrix on a GPU, or a stack of them, whose rows are contiguous")
    given = out is not None
    out = _out(out, "out", g.shape, torch.bfloat16, g)
    count, (rows, cols) = (g.shape[0] if g.dim() == 3 else 1), g.shape[-2:]
    lib = M.lib()
    need = lib.moe_spec_orthogonalise_workspace_bytes(count, rows, cols)
    space = g.new_empty(need, dtype=torch.uint8) if need else None
    _queue(g.device, lib.moe_spec_orthogonalise, dtype, g.data_ptr(), g.stride(0) if g.dim() == 3 else 0, g.stride(-2), count, rows, cols,
           c, iterations, out.data_ptr(), out.stride(0) if g.dim() == 3 else 0, out.stride(-2),
           space.data_ptr() if need else None, need)
    if given:
        increment_version(out)
    return out


class Muon:
    """Momentum with orthogonalised updates for float32 matrices [rows, cols] and stacks of them [count, rows, cols], such as experts'
    weights, in one call; embeddings, heads and vectors are AdamW's.  Holds the tensors and their momenta; the settings may be
    changed between steps.  A captured step keeps those it was captured with; grad_scale it reads anew where it is a tensor.

    update_rms: the root mean square of an update at lr = 1.  copies: bfloat16 tensors (or None in places) that get the updated
    parameters, rounded; a stack's may be a part of larger blocks, as an expert block holds gate, up and down.  states: momenta to go on with, as `states()` gave them; used in place."""

    def __init__(self, params: Sequence[torch.Tensor], *, lr: float, momentum: float = 0.95, nesterov: bool = True,
                 weight_decay: float = 0.01, update_rms: float = 0.2, iterations: int = 5, coefficients=ORTHOGONALISE,
                 copies: Optional[Sequence[Optional[torch.Tensor]]] = None, states: Optional[dict] = None):
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        self.lr, self.momentum, self.nesterov, self.weight_decay = lr, momentum, nesterov, weight_decay
        self.update_rms, self.iterations, self.coefficients = update_rms, iterations, tuple(coefficients)
        _three(self.coefficients)
        self.device = self.params[0].device
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        self._m = list(states["m"]) if states is not None else [torch.zeros_like(p, memory_format=torch.contiguous_format) for p in self.params]
        if len(self._m) != len(self.params) or len(self.copies) != len(self.params):
            raise ValueError("as many momenta and copies as parameters are needed")
        self._shapes = [tuple(p.shape) for p in self.params]
        if any(len(s) not in (2, 3) for s in self._shapes):
            raise ValueError("parameters must be matrices or stacks of matrices")
        self._held = [t for t in (*self.params, *self._m, *self.copies) if t is not None]
        self._at = None
        self._desc = (M.MuonTensor * len(self.params))()
        self._describe()

    def states(self) -> dict:
        """The momenta."""
        return {"m": list(self._m)}

    def _tensor(self, t, name, dtype, shape):
        if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != self.device or not t.is_cuda:
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on the parameters' GPU")

    def _describe(self):
        """The tensors' table for the library; made anew where one of them has got other storage since."""
        at = [*map(_ADDRESS, self._held), *(c.stride() for c in self.copies if c is not None)]
        if at == self._at:
            return
        for d, p, m, c, shape in zip(self._desc, self.params, self._m, self.copies, self._shapes):
            self._tensor(p, "a parameter", torch.float32, shape)
            self._tensor(m, "a momentum", torch.float32, shape)
            d.p, d.m, d.copy, d.copy_stride = p.data_ptr(), m.data_ptr(), None if c is None else c.data_ptr(), 0
            d.rows, d.cols = shape[-2:]
            if c is not None:
                if len(shape) == 3 and tuple(c.shape) == shape and shape[0] > 1 and c.stride(0) > shape[1] * shape[2]:
                    d.copy_stride, c = c.stride(0), c[0]                 # a part of larger blocks
                    self._tensor(c, "a copy's matrix", torch.bfloat16, shape[1:])
                else:
                    self._tensor(c, "a copy", torch.bfloat16, shape)
        written = [t.data_ptr() for t in self._held if t.numel()]
        if len(set(written)) < len(written):
            raise ValueError("a tensor is named twice")
        self._at = at

    def step(self, grads: Sequence[Optional[torch.Tensor]], *, grad_scale=1.0):
        """One step with a gradient for each parameter, all float32 or all bfloat16; a parameter whose gradient is None stays as it
        is.  grad_scale: a factor of the gradients, a number or a float32 tensor on the GPU."""
        if len(grads) != len(self.params):
            raise ValueError("as many gradients as parameters are needed")
        dtype = next((g.dtype for g in grads if g is not None), torch.float32)
        if dtype not in _TYPES:
            raise ValueError("gradients must be float32 or bfloat16")
        self._describe()
        for d, g, shape in zip(self._desc, grads, self._shapes):
            if g is None:
                d.count = 0
            else:
                self._tensor(g, "a gradient", dtype, shape)
                d.grad, d.count = g.data_ptr(), shape[0] if len(shape) == 3 else 1
        c = M.MuonConfig(lr=self.lr, momentum=self.momentum, weight_decay=self.weight_decay, update_rms=self.update_rms, grad_scale=1.0,
                         coefficients=_three(self.coefficients), iterations=self.iterations, nesterov=bool(self.nesterov), grad_dtype=_TYPES[dtype])
        if isinstance(grad_scale, torch.Tensor):
            if grad_scale.dtype != torch.float32 or grad_scale.numel() != 1 or grad_scale.device != self.device:
                raise ValueError("grad_scale must be a number or one float32 value on the parameters' GPU")
            c.grad_scale_dev = grad_scale.data_ptr()
        else:
            c.grad_scale = grad_scale
        lib = M.lib()
        need = lib.moe_spec_muon_workspace_bytes(self._desc, len(self._desc))
        space = self.params[0].new_empty(need, dtype=torch.uint8) if need else None
        _queue(self.device, lib.moe_spec_muon_step, self._desc, len(self._desc), C.byref(c), space.data_ptr() if need else None, need)
        increment_version([t for p, m, q, g in zip(self.params, self._m, self.copies, grads) if g is not None for t in (p, m, q) if t is not None])


def _choices(z: torch.Tensor, k: int) -> torch.Tensor:
    """The k largest of each row, among equals those of the lowest index: int32 [rows, k]."""
    return torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k].to(torch.int32)


class EstimatorTrainer:
    """Distils the expert estimator (paper: Appendix A) from the routers it stands in for.

    weights: the estimator's tables under the names that Engine and workload.make_estimator use (proj, layer_emb, ffn_in,
    ffn_out, ln_gain, ln_bias, head), as numpy arrays in storage format or as tensors on the GPU.  Tensors are trained in place:
    given an Engine's own (`engine.est`), its predictions follow the training, as its context reads the same memory; the caller
    keeps the engine's stream and the training stream apart in time.  bfloat16 tables have float32 masters here and are the
    copies that AdamW writes; products then take bfloat16 operands and add up in float32, in the library that torch
    calls for plain matrix products, and what lies between them is bfloat16 too: the feed-forward's values and all gradients that pass
    through it, each table's gradient (widened for AdamW, which takes one type a call), the two losses' gradients before and after they are
    added, and the logits, so that choices between nearly equal ones may differ from an engine's, which are float32.  LayerNorm, losses and
    AdamW are this library's.

    balance_coef: weight of a balance loss over the estimator's own predictions, against its collapse on a few experts.  top_k: how
    many experts it predicts for a token, which that loss counts.

    masters: the float32 tables of a training to go on with, as `masters()` gave them, to which weights are set; used in place where
    weights are bfloat16.  Together with the moments (states, steps and seed, as AdamW takes them) the steps go on as if they had
    never stopped; from bfloat16 weights alone they go on from rounded tables."""

    NAMES = ("proj", "layer_emb", "ffn_in", "ffn_out", "ln_gain", "ln_bias", "head")

    def __init__(self, weights: dict, *, lr: float = 1e-3, balance_coef: float = 0.0, top_k: Optional[int] = None, ln_eps: float = 1e-5,
                 masters: Optional[dict] = None, device="cuda:0", **adamw):
        from .engine import _np_to_torch_storage
        to = lambda v: v if isinstance(v, torch.Tensor) else _np_to_torch_storage(v).to(device)  # noqa: E731
        self.weights = {k: to(weights[k]) for k in self.NAMES}
        self.dtype = self.weights["proj"].dtype
        if masters is None:
            masters = {k: (v if v.dtype == torch.float32 else v.float()) for k, v in self.weights.items()}
        else:
            masters = {k: to(masters[k]) for k in self.NAMES}
            if any(m.dtype != torch.float32 or m.shape != self.weights[k].shape for k, m in masters.items()):
                raise ValueError("masters must be float32 tables of the weights' shapes")
            with torch.no_grad():
                for k, v in self.weights.items():
                    v.copy_(masters[k])
            masters = {k: (v if v.dtype == torch.float32 else masters[k]) for k, v in self.weights.items()}
        self.optimizer = AdamW([masters[k] for k in self.NAMES], lr=lr, copies=[
            self.weights[k] if self.weights[k] is not masters[k] else None for k in self.NAMES], **adamw)
        if top_k is not None and not 1 <= top_k <= self.weights["head"].shape[0]:
            raise ValueError("top_k must be between 1 and the number of experts")
        self.balance_coef, self.top_k, self.ln_eps = balance_coef, top_k, ln_eps

    @torch.no_grad()
    def gradients(self, layers: Sequence[int], signal: torch.Tensor, teacher: torch.Tensor, ids: Optional[torch.Tensor] = None,
                  valid: Optional[torch.Tensor] = None):
        """Losses and gradients for the predicting signals [n, T, H] of n different layers and the logits [n, T, E] that the
        next layers' routers gave -> (dict of loss, balance, counts; dict of gradients).  The balance loss and the counts are of
        the experts that the estimator chooses: the top_k largest of its logits, or ids, int32 [n, T, k], where the caller has its
        choices already.  (Not the routers' choices: against those the loss would push the estimator away from what it is
        to predict, and where they are balanced it would not push at all.)  valid: [n, T], 0 for padding, which counts for
        nothing whatever it holds."""
        n, tokens, _ = signal.shape
        w = self.weights
        layers = [index(l) for l in layers]     # a tensor's elements are no equal members of a set
        if len(set(layers)) != n or len(layers) != n or not all(0 <= l < w["layer_emb"].shape[0] for l in layers):
            raise ValueError("a layer of its own for each of the signals is needed")
        if ids is None and self.top_k is None and self.balance_coef != 0.0:
            raise ValueError("the balance term needs choices to count: top_k or ids, or a balance_coef of 0")
        if any(t is not None and t.shape[:2] != (n, tokens) for t in (teacher, ids, valid)):
            raise ValueError("teacher, ids and valid must have the layers and tokens of the signal")
        flat = lambda t: None if t is None else t.reshape(n * tokens, *t.shape[2:])  # noqa: E731
        at = torch.as_tensor(layers, dtype=torch.long, device=signal.device)
        x, mask = flat(signal).to(self.dtype), flat(valid)
        if mask is not None:                  # chosen, not multiplied: zero times what padding holds need not be zero in a product
            _mask(mask, n * tokens, x.device)
            x = torch.where(mask.bool()[:, None], x, 0.0)
        latent = w["proj"].shape[0]
        u = (torch.mm(x, w["proj"].T).view(n, tokens, latent) + w["layer_emb"][at][:, None]).view(n * tokens, latent)
        h = torch.mm(u, w["ffn_in"].T)
        gate = torch.sigmoid(h)
        act = h * gate
        v = u + torch.mm(act, w["ffn_out"].T)
        y, mean, rstd = layernorm_forward(v, w["ln_gain"], w["ln_bias"], self.ln_eps)
        z = torch.mm(y, w["head"].T)
        loss, dz = distill_loss(z, flat(teacher), valid=mask)
        out = {"loss": loss}
        if ids is not None or self.top_k is not None:
            chosen = flat(ids) if ids is not None else _choices(z, self.top_k)
            out["balance"], out["counts"], extra = balance_loss(z, chosen, coef=self.balance_coef, valid=mask,
                                                                grad=self.balance_coef != 0.0)
            if extra is not None:
                dz = dz + extra
        g = {"head": torch.mm(dz.T, y)}
        dv, g["ln_gain"], g["ln_bias"] = layernorm_backward(torch.mm(dz, w["head"]), v, mean, rstd, w["ln_gain"])
        g["ffn_out"] = torch.mm(dv.T, act)
        dh = torch.mm(dv, w["ffn_out"]) * (gate * (1.0 + h * (1.0 - gate)))
        g["ffn_in"] = torch.mm(dh.T, u)
        du = dv + torch.mm(dh, w["ffn_in"])
        g["proj"] = torch.mm(du.T, x)
        g["layer_emb"] = torch.zeros(w["layer_emb"].shape, device=signal.device)
        g["layer_emb"][at] = du.view(n, tokens, latent).sum(1, dtype=torch.float32)
        return out, g

    def step(self, layers, signal, teacher, ids=None, valid=None, *, grad_scale=1.0) -> dict:
        """One training step; returns the losses (and counts) from before it."""
        out, g = self.gradients(layers, signal, teacher, ids, valid)
        self.optimizer.step([g[k].float() for k in self.NAMES], grad_scale=grad_scale)
        return out

    def masters(self) -> dict:
        """The float32 tables that are trained: weights itself where those are float32."""
        return dict(zip(self.NAMES, self.optimizer.params))

    def numpy_weights(self) -> dict:
        """The weights in storage format, for a new Engine or a file (bfloat16 as uint16 bit patterns)."""
        return {k: (v.view(torch.int16).cpu().numpy().view("uint16") if v.dtype == torch.bfloat16 else v.cpu().numpy())
                for k, v in self.weights.items()}
