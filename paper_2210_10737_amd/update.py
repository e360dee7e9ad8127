"""The update phase of a training step on the library's kernels: the product
with a layer's weights and its epilogue, the class loss, the AdamW step.

Operands are fp32, bf16 or fp16 on the current device. A matrix whose rows do
not lie 16-byte aligned with unit stride (a contiguous [n, 41] tensor, an
expanded gradient) is copied into one that does before the call; outputs have
such rows, so chained calls copy nothing.

`linear` and `linear_cross_entropy` are differentiable once. Everything runs
on the current stream and can be captured into a HIP graph, a forward pass
together with its backward pass: the backward pass of one that ran outside the
capture cannot be captured, nor, by torch's own rule, a `backward()` while a result
of an eager pass over the same leaves is held (drop such losses before).
"""
from __future__ import annotations

import ctypes
from array import array

import torch
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version

from . import AdamwStruct, LinearStruct, XentStruct, _check, _device_index, _dp, _stream, _workspace, lib

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ACTS = {"none": 0, None: 0, "relu": 1, "gelu": 2, "silu": 3}
_REDUCTIONS = {"none": 0, "sum": 1, "mean": 2}


# ---------------------------------------------------------------- matrices
# (small calls are bound by the host's time for them, so each property is read
# from a tensor once)
def _new(rows: int, cols: int, dtype, device) -> torch.Tensor:
    """rows x cols, in rows that are whole 16-byte units. No view of a wider
    tensor: autograd refuses writes in place to views that a Function returns."""
    u = 16 // dtype.itemsize
    ld = (cols + u - 1) // u * u
    return torch.empty_strided((rows, cols), (ld, 1), dtype=dtype, device=device)


def _ld(t: torch.Tensor) -> int | None:
    """The leading dimension the library can use for a 2-D tensor, or None."""
    rows, cols = t.shape
    s0, s1 = t.stride()
    u = 16 // t.dtype.itemsize
    if (s1 != 1 and cols > 1) or t.data_ptr() % 16:
        return None
    if rows <= 1:
        return (cols + u - 1) // u * u
    return s0 if s0 >= cols and s0 % u == 0 else None


def _matrix(t: torch.Tensor) -> tuple[torch.Tensor, int]:
    """(t or an aligned copy of it, leading dimension)."""
    ld = _ld(t)
    if ld is not None:
        return t, ld
    c = _new(t.shape[0], t.shape[1], t.dtype, t.device)
    c.copy_(t)
    return c, _ld(c)


def _weights(w: torch.Tensor) -> tuple[torch.Tensor, int, int]:
    """(w or a copy, leading dimension, 1 if stored output-major)."""
    k, m = w.shape
    s0, s1 = w.stride()
    u = 16 // w.dtype.itemsize
    if w.data_ptr() % 16 == 0:
        if s1 == 1 and s0 >= m and s0 % u == 0:
            return w, s0, 0
        if s0 == 1 and s1 >= k and s1 % u == 0:
            return w, s1, 1
    if s0 == 1 and k > 1:   # keep the order it is stored in
        t, ld = _matrix(w.t())
        return t.t(), ld, 1
    c, ld = _matrix(w)
    return c, ld, 0


def _new_like_weights(w: torch.Tensor, out_major: int) -> tuple[torch.Tensor, int]:
    k, m = w.shape
    u = 16 // w.dtype.itemsize
    ld = ((k if out_major else m) + u - 1) // u * u
    return torch.empty_strided((k, m), (1, ld) if out_major else (ld, 1), dtype=w.dtype, device=w.device), ld


def _check_operand(t: torch.Tensor, name: str, shape, dtype=None) -> None:
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: {t.dtype}, {dtype} expected")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, {tuple(shape)} expected")
    if t.get_device() != _device_index():
        raise ValueError(f"{name} on {t.device}: the library runs on the current device cuda:{_device_index()}")


def _check_product(x: torch.Tensor, weight: torch.Tensor, bias) -> tuple[int, int, int]:
    """n, k, m of x @ weight (+ bias)."""
    dtype, xs, ws = x.dtype, x.shape, weight.shape
    if dtype not in _DTYPES:
        raise ValueError(f"x: {dtype}, one of float32, bfloat16, float16 expected")
    if len(xs) != 2 or len(ws) != 2:
        raise ValueError("x and weight must be 2-D")
    n, k = xs
    m = ws[1]
    if ws[0] != k or k < 1 or m < 1:
        raise ValueError(f"x of shape {tuple(xs)}, weight of shape {tuple(ws)}")
    if weight.dtype != dtype:
        raise ValueError(f"weight: {weight.dtype}, {dtype} expected")
    dev = _device_index()
    if x.get_device() != dev or weight.get_device() != dev:
        raise ValueError(f"x on {x.device}, weight on {weight.device}: the library runs on the current device "
                         f"cuda:{dev}")
    if bias is not None:
        if bias.dtype != dtype and bias.dtype != torch.float32:
            raise ValueError(f"bias: {bias.dtype}, {dtype} or float32 expected")
        _check_operand(bias, "bias", (m,))
    return n, k, m


def _bias_arg(bias):
    if bias is None:
        return None, None, 0
    b = bias if bias.is_contiguous() else bias.contiguous()
    return b, b.data_ptr(), _DTYPES[b.dtype]


# ------------------------------------------------------------------- layer
def _linear_forward(x, weight, bias, residual, act: int, alpha: float, beta: float, out, keep: bool):
    """(y, pre or None, the aligned x and weight)."""
    n, (k, m) = x.shape[0], weight.shape
    dtype, dev = x.dtype, x.device
    xa, ldx = _matrix(x)
    wa, ldw, out_major = _weights(weight)
    b, pb, b_dtype = _bias_arg(bias)
    p = LinearStruct(_DTYPES[dtype], act, n, k, m, out_major, alpha, beta, keep)
    y = _new(n, m, dtype, dev) if out is None else out
    ra, ldr = (None, 0) if residual is None else _matrix(residual)
    pre = _new(n, m, torch.float32, dev) if keep and act >= 2 else None
    L, ref = lib(), ctypes.byref(p)
    need = L.rsc_linear_workspace_bytes(ref)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    status = L.rsc_linear(ref, xa.data_ptr(), ldx, wa.data_ptr(), ldw, pb, b_dtype,
                          None if ra is None else ra.data_ptr(), ldr, y.data_ptr(), _ld(y),
                          None if pre is None else pre.data_ptr(), 0 if pre is None else _ld(pre),
                          None if ws is None else ws.data_ptr(), need, _stream())
    if status:
        _check(status)
    if out is not None:
        increment_version(out)
    return y, pre, xa, wa


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act, alpha, beta):
        y, pre, xa, wa = _linear_forward(x, weight, bias, residual, act, alpha, beta, None, True)
        ctx.layer = (act, alpha, beta, None if bias is None else bias.dtype)
        ctx.save_for_backward(xa, wa, y if act == 1 else pre)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        act, alpha, beta, bias_dtype = ctx.layer
        x, weight, saved = ctx.saved_tensors
        need_x, need_w, need_b, need_r = ctx.needs_input_grad[:4]
        n, (k, m) = x.shape[0], weight.shape
        dev, dtype = x.device, x.dtype
        _check_operand(dy, "the gradient", (n, m), dtype)
        dya, lddy = _matrix(dy)
        x, ldx = _matrix(x)
        weight, ldw, out_major = _weights(weight)
        p = LinearStruct(_DTYPES[dtype], act, n, k, m, out_major, alpha, beta)
        dx = _new(n, k, dtype, dev) if need_x else None
        dw, lddw = _new_like_weights(weight, out_major) if need_w else (None, 0)
        db = torch.empty(m, dtype=bias_dtype, device=dev) if need_b else None
        # without an activation the residual's gradient is dy times beta
        same = act == 0 and beta == 1.0
        dr = _new(n, m, dtype, dev) if need_r and not same else None
        if not (need_x or need_w or need_b or dr is not None):
            return None, None, None, dy if need_r else None, None, None, None
        need = lib().rsc_linear_backward_workspace_bytes(ctypes.byref(p), need_x, need_w, need_b)
        ws = _workspace(need, dev) if need else None
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        ld = lambda t: 0 if t is None else _ld(t)  # noqa: E731
        _check(lib().rsc_linear_backward(ctypes.byref(p), dya.data_ptr(), lddy, ptr(saved), ld(saved), x.data_ptr(), ldx,
                                         weight.data_ptr(), ldw, ptr(dx), ld(dx), ptr(dw), lddw, ptr(db),
                                         0 if db is None else _DTYPES[bias_dtype], ptr(dr), ld(dr), ptr(ws), need,
                                         _stream()))
        return dx, dw, db, (dy if same else dr) if need_r else None, None, None, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None,
           residual: torch.Tensor | None = None, act: str | None = "none", alpha: float = 1.0, beta: float = 1.0,
           out: torch.Tensor | None = None) -> torch.Tensor:
    """act(alpha x @ weight + bias + beta residual), act one of none, relu,
    gelu (exact), silu (rsc_linear).

    x [n, k], weight [k, m] in either storage order (a transposed view of an
    [m, k] tensor is used as it lies), residual [n, m], all of one type;
    bias [m] of that type or float32. The result's rows are whole 16-byte units
    apart, so with other m it is not contiguous (reshape, not view, flattens it).
    Differentiable once in all four; dW has weight's storage order. With gradients a ReLU's sign next to zero is decided
    in 64 bits (at most 32 times in some thousand results), and GELU and SiLU
    keep their argument, n x m float32. out (no gradients): [n, m] with aligned rows, may
    be the residual; the write counts as one in place to autograd."""
    if act not in _ACTS:
        raise ValueError(f"act {act!r}: none, relu, gelu or silu expected")
    n, _, m = _check_product(x, weight, bias)
    if residual is not None:
        _check_operand(residual, "residual", (n, m), x.dtype)
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or
                                    (bias is not None and bias.requires_grad) or
                                    (residual is not None and residual.requires_grad)):
        if out is not None:
            raise ValueError("out is for calls without gradients")
        return _Linear.apply(x, weight, bias, residual, _ACTS[act], float(alpha), float(beta))
    if out is not None:
        _check_operand(out, "out", (n, m), x.dtype)
        if out.requires_grad and torch.is_grad_enabled():
            raise ValueError("out requires gradients: a write to it is for no_grad")
        if _ld(out) is None:
            raise ValueError("out: rows of whole 16-byte units with unit column stride expected")
    return _linear_forward(x, weight, bias, residual, _ACTS[act], float(alpha), float(beta), out, False)[0]


# -------------------------------------------------------------- class loss
def _xent_struct(x, weight, out_major, targets, b_dtype, ignore_index, reduction):
    return XentStruct(_DTYPES[x.dtype], x.shape[0], weight.shape[0], weight.shape[1], out_major, reduction,
                      int(targets.dtype == torch.int32), b_dtype, ignore_index)


_KEPT_CLASSES = 64   # rsc_xent's bound for leaving the logits' gradient


def _xent_forward(x, weight, targets, bias, ignore_index: int, reduction: int, keep: bool = False):
    """(loss, lse and divisor, the logits' gradient or None, the aligned x and weight)."""
    n, dev = x.shape[0], x.device
    xa, ldx = _matrix(x)
    wa, ldw, out_major = _weights(weight)
    b, pb, b_dtype = _bias_arg(bias)
    p = _xent_struct(x, weight, out_major, targets, b_dtype, ignore_index, reduction)
    loss = torch.empty((n,) if reduction == 0 else (), dtype=torch.float32, device=dev)
    # lse of each row, behind it the divisor
    kept = torch.empty(n + 1, dtype=torch.float32, device=dev)
    grad = _new(n, p.v, x.dtype, dev) if keep and p.v <= _KEPT_CLASSES and reduction != 0 else None
    need = lib().rsc_xent_workspace_bytes(ctypes.byref(p))
    ws = _workspace(need, dev)
    _check(lib().rsc_xent(ctypes.byref(p), xa.data_ptr(), ldx, wa.data_ptr(), ldw, pb, targets.data_ptr(),
                          loss.data_ptr(), kept.data_ptr(), kept.data_ptr() + 4 * n,
                          None if grad is None else grad.data_ptr(), 0 if grad is None else _ld(grad), ws.data_ptr(),
                          need, _stream()))
    return loss, kept, grad, xa, wa


class _Xent(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, targets, bias, ignore_index, reduction):
        # (kept, G is in the operands' type: a float32 bias's gradient comes from before that rounding)
        keep = bias is None or bias.dtype == x.dtype or not ctx.needs_input_grad[3]
        loss, kept, grad, xa, wa = _xent_forward(x, weight, targets, bias, ignore_index, reduction, keep)
        ctx.save_for_backward(xa, wa, targets, bias, kept, grad)
        ctx.options = (ignore_index, reduction)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        x, weight, targets, bias, kept, grad = ctx.saved_tensors
        ignore_index, reduction = ctx.options
        need_x, need_w, _, need_b = ctx.needs_input_grad[:4]
        n, dev, dtype = x.shape[0], x.device, x.dtype
        x, ldx = _matrix(x)
        weight, ldw, out_major = _weights(weight)
        b, pb, b_dtype = _bias_arg(bias)
        p = _xent_struct(x, weight, out_major, targets, b_dtype, ignore_index, reduction)
        _check_operand(dloss, "the gradient", (n,) if reduction == 0 else (), torch.float32)
        dloss = dloss.contiguous()
        dx = _new(n, weight.shape[0], dtype, dev) if need_x else None
        dw, lddw = _new_like_weights(weight, out_major) if need_w else (None, 0)
        db = torch.empty(weight.shape[1], dtype=bias.dtype, device=dev) if need_b else None
        need = lib().rsc_xent_backward_workspace_bytes(ctypes.byref(p), need_x, need_w, grad is not None)
        ws = _workspace(need, dev)
        _check(lib().rsc_xent_backward(ctypes.byref(p), dloss.data_ptr(), x.data_ptr(), ldx, weight.data_ptr(), ldw,
                                       pb, targets.data_ptr(), kept.data_ptr(), kept.data_ptr() + 4 * n,
                                       None if grad is None else grad.data_ptr(), 0 if grad is None else _ld(grad),
                                       None if dx is None else dx.data_ptr(), 0 if dx is None else _ld(dx),
                                       None if dw is None else dw.data_ptr(), lddw,
                                       None if db is None else db.data_ptr(), ws.data_ptr(), need, _stream()))
        return dx, dw, None, db, None, None


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                         bias: torch.Tensor | None = None, ignore_index: int = -100,
                         reduction: str = "mean") -> torch.Tensor:
    """Softmax cross entropy (float32) of the logits x @ weight + bias against
    one class a row, without the logits in memory (rsc_xent): they are formed in
    tiles, and their gradient in pieces of the classes.

    x [n, k], weight [k, v] in either storage order, bias [v] as in `linear`;
    targets int64 or int32 [n]. Rows of ignore_index count for nothing; any
    other target outside 0 .. v-1 gives NaN. reduction: mean over the rows that
    count (0 if there is none), sum, or none (a loss per row). Differentiable
    once in x, weight and bias: the logits are then formed again, except that
    up to 64 classes the forward pass keeps their gradient (n x v values; not for
    16-bit operands with a float32 bias that requires gradients). The logits'
    gradient is rounded to x's type before dX and dW are formed from it.

    A bias of -inf or of the lowest finite value takes a class out; where it takes
    all of them out, gradients mean nothing. float16 with reduction none: dX's
    rows are held beside their own upstream gradient, what they add to dW beside the
    largest one (below 2^-34 of it, it is lost)."""
    if reduction not in _REDUCTIONS:
        raise ValueError(f"reduction {reduction!r}: none, sum or mean expected")
    if targets.dtype not in (torch.int64, torch.int32):
        raise ValueError(f"targets: {targets.dtype}, int64 or int32 expected")
    _check_product(x, weight, bias)
    _check_operand(targets, "targets", (x.shape[0],))
    targets = targets.contiguous()
    if not -(1 << 63) <= int(ignore_index) < 1 << 63:
        raise ValueError(f"ignore_index {ignore_index} is no int64")
    args = (x, weight, targets, bias, int(ignore_index), _REDUCTIONS[reduction])
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or
                                    (bias is not None and bias.requires_grad)):
        return _Xent.apply(*args)
    return _xent_forward(*args)[0]


# ----------------------------------------------------------------- optimizer
def _descriptors(count: int, columns) -> ctypes.Array:
    """rsc_adamw_tensor_t[count] from its eight columns of 64-bit values."""
    flat = array("Q", bytes(64 * count))
    for j, column in enumerate(columns):
        if column is not None:
            flat[j::8] = array("Q", column)
    return (ctypes.c_uint64 * (8 * count)).from_buffer(flat)


def _column(tensors, count: int, name: str, dtype, sizes) -> list[int]:
    """Addresses of contiguous tensors of the given sizes on the current device."""
    if len(tensors) != count:
        raise ValueError(f"{name}: {len(tensors)} tensors, {count} expected")
    dev = _device_index()
    # (one expression: with hundreds of small tensors this is most of a step's time)
    got = [t.data_ptr() for t, n in zip(tensors, sizes)
           if t.dtype is dtype and t.numel() == n and t.is_contiguous() and t.get_device() == dev]
    if len(got) != count:
        for t, n in zip(tensors, sizes):
            if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
                raise ValueError(f"{name}: {t.dtype}{list(t.shape)} on {t.device}, contiguous {dtype}[{n}] on the "
                                 f"current device cuda:{dev} expected")
    return got


def _moment_columns(exp_avgs, exp_avg_sqs, scales, scale_sqs, sizes):
    count = len(sizes)
    if scales is None:
        return (_column(exp_avgs, count, "exp_avgs", torch.float32, sizes),
                _column(exp_avg_sqs, count, "exp_avg_sqs", torch.float32, sizes), None, None)
    blocks = [(n + 255) // 256 for n in sizes]
    return (_column(exp_avgs, count, "exp_avgs", torch.int8, sizes),
            _column(exp_avg_sqs, count, "exp_avg_sqs", torch.uint8, sizes),
            _column(scales, count, "exp_avg_scales", torch.float32, blocks),
            _column(scale_sqs, count, "exp_avg_sq_scales", torch.float32, blocks))


def adamw_step(params, grads, exp_avgs, exp_avg_sqs, step: torch.Tensor, *, lr: float = 1e-3,
               betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2, masters=None,
               exp_avg_scales=None, exp_avg_sq_scales=None, seed: int = 0) -> None:
    """One AdamW step over lists of tensors, in place (rsc_adamw_step).

    params and grads: contiguous, all of one type (float32, bfloat16 or
    float16). Moments: float32, or with both lists of scales 8-bit codes (int8,
    uint8; a float32 scale for each 256 elements). masters: float32 values that
    the step is applied to, params then receive their rounding. step: int64[1]
    on the device, advanced by the call. No tensor may appear twice. To autograd
    the step is a write in place to params and masters: a backward pass of a graph
    that saved one of them before raises."""
    count = len(params)
    if (exp_avg_scales is None) != (exp_avg_sq_scales is None):
        raise ValueError("8-bit moments need both exp_avg_scales and exp_avg_sq_scales")
    if step.dtype != torch.int64 or step.numel() != 1 or not step.is_contiguous():
        raise ValueError(f"step: {step.dtype}{list(step.shape)}, int64[1] expected")
    dtype = params[0].dtype if count else torch.float32
    if dtype not in _DTYPES:
        raise ValueError(f"params: {dtype}, float32, bfloat16 or float16 expected")
    sizes = [t.numel() for t in params]
    p = _column(params, count, "params", dtype, sizes)
    live = [a for a, n in zip(p, sizes) if n]
    if len(set(live)) != len(live):
        raise ValueError("a parameter appears twice")
    columns = (p, _column(grads, count, "grads", dtype, sizes),
               *_moment_columns(exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales, sizes))
    master = None if masters is None else _column(masters, count, "masters", torch.float32, sizes)
    array = _descriptors(count, (*columns[:4], master, *columns[4:], sizes))
    opts = AdamwStruct(_DTYPES[dtype], 32 if exp_avg_scales is None else 8, float(lr), float(betas[0]),
                       float(betas[1]), float(eps), float(weight_decay), int(seed) & ((1 << 64) - 1))
    need = lib().rsc_adamw_workspace_bytes()
    ws = _workspace(need, step.device)
    _check(lib().rsc_adamw_step(ctypes.byref(opts), array, count, _dp(step), ws.data_ptr(), need, _stream()))
    increment_version(params)
    if masters is not None:
        increment_version(masters)


def adamw_moments(exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales, out=None):
    """(first, second) moments that 8-bit codes stand for, as lists of float32
    tensors (rsc_adamw_moments); out: two lists of contiguous float32 tensors
    to write to."""
    sizes = [t.numel() for t in exp_avgs]
    count = len(sizes)
    columns = _moment_columns(exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales, sizes)
    if out is None:
        out = tuple([torch.empty(t.shape, dtype=torch.float32, device=t.device) for t in exp_avgs] for _ in range(2))
    to = [(ctypes.c_uint64 * max(count, 1))(*_column(o, count, "out", torch.float32, sizes)) for o in out]
    array = _descriptors(count, (None, None, *columns[:2], None, *columns[2:], sizes))
    _check(lib().rsc_adamw_moments(array, count, to[0], to[1], _stream()))
    for tensors in out:
        increment_version(tensors)
    return out


def _seed_of(seed: int, group: int, count: int) -> int:
    """Each call of a step draws words of its own (a call numbers its elements
    from 0): the seed itself for the first group's first count, for the others an output
    of SplitMix64 (Steele, Lea and Flood 2014) seeded with it."""
    number = (group << 32) + count
    if number == 0:
        return seed
    mask = (1 << 64) - 1
    z = (seed + number * 0x9E3779B97F4A7C15) & mask
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
    return z ^ (z >> 31)


class AdamW(torch.optim.Optimizer):
    """AdamW (decoupled weight decay) over the library's step of many tensors.

    state_bits: 32 (float32 moments) or 8 (codes with a scale for each 256
    elements: 2.03 bytes a parameter instead of 8). 16-bit parameters keep
    float32 masters unless master_weights is False; a master is made from its
    parameter at the parameter's first step and from then on is what the step
    is applied to, so load weights before that (or load_state_dict after).

    The state of a parameter is made at its first step, which can therefore
    not be captured into a HIP graph; later ones can (a captured step holds
    lr, betas, eps and weight_decay of its capture).

    Each parameter's steps are counted, as torch's optimizer does: bias
    corrections of one whose gradients come later, or not in every step, are its
    own. Parameters that have taken the same steps share a count on the device
    and one call (group["counts"], group["count_of"]); a step in which only some of
    them have gradients gives these a count of their own, which cannot happen
    in a capture nor, since a captured step holds its counts, after one: run such
    a step once before. group["step"] counts the steps of the group (while it has
    more than one count, without those of graphs from before)."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2,
                 state_bits: int = 32, master_weights: bool = True, seed: int = 0):
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits {state_bits}: 8 or 32 expected")
        if not (0.0 <= betas[0] < 1.0 and 0.0 <= betas[1] < 1.0) or eps < 0.0 or lr < 0.0 or weight_decay < 0.0:
            raise ValueError("need 0 <= betas < 1 and lr, eps, weight_decay >= 0")
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay,
                                      state_bits=state_bits, master_weights=master_weights, seed=seed))

    def _state_of(self, p: torch.Tensor, group) -> dict:
        s = self.state[p]
        if not s:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a parameter's first step makes its state and cannot be captured")
            if not p.is_contiguous():
                raise ValueError(f"parameter of shape {tuple(p.shape)} is not contiguous")
            if group["state_bits"] == 8:
                blocks = (p.numel() + 255) // 256
                s["exp_avg"] = torch.zeros(p.shape, dtype=torch.int8, device=p.device)
                s["exp_avg_sq"] = torch.zeros(p.shape, dtype=torch.uint8, device=p.device)
                s["exp_avg_scale"] = torch.zeros(blocks, dtype=torch.float32, device=p.device)
                s["exp_avg_sq_scale"] = torch.zeros(blocks, dtype=torch.float32, device=p.device)
            else:
                s["exp_avg"] = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
                s["exp_avg_sq"] = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
            if p.dtype != torch.float32 and group["master_weights"]:
                s["master"] = p.detach().float()
        return s

    def _parts(self, group, used: list[int]) -> list[tuple[int, list[int]]]:
        """The parameters `used` by their counts: (number of the count, which of
        the group's parameters)."""
        params, capturing = group["params"], torch.cuda.is_current_stream_capturing()
        captured = self.__dict__.setdefault("_captured", [])    # counts that a graph holds
        if "counts" not in group:
            # (a state that counts by group only: its parameters go on from there)
            group["counts"] = [group["step"]] if "step" in group else []
            group["count_of"] = [0 if "step" in group and self.state.get(p) else -1 for p in params]
        counts, of = group["counts"], group["count_of"]
        of.extend([-1] * (len(params) - len(of)))
        by_count: dict[int, list[int]] = {}
        for i in used:
            by_count.setdefault(of[i], []).append(i)
        parts = []
        for count, members in by_count.items():
            if count < 0 or len(members) < of.count(count):
                if capturing or (count >= 0 and any(t is counts[count] for t in captured)):
                    raise RuntimeError("the first step with gradients for just these parameters makes their count: it "
                                       "cannot be captured, nor come after a captured step of them")
                counts.append(torch.zeros(1, dtype=torch.int64, device=params[members[0]].device) if count < 0
                              else counts[count].clone())
                count = len(counts) - 1
                for i in members:
                    of[i] = count
            parts.append((count, members))
        group.setdefault("step", counts[0])
        if capturing:
            captured.extend(counts[count] for count, _ in parts)
        return parts

    def _step_of(self, group, used: list[torch.Tensor], count: torch.Tensor, seed: int) -> None:
        states = [self.state[p] for p in used]
        bits8 = group["state_bits"] == 8
        adamw_step([p.detach() for p in used], [p.grad if p.grad.is_contiguous() else p.grad.contiguous() for p in used],
                   [s["exp_avg"] for s in states], [s["exp_avg_sq"] for s in states], count,
                   lr=group["lr"], betas=group["betas"], eps=group["eps"], weight_decay=group["weight_decay"],
                   masters=[s["master"] for s in states] if "master" in states[0] else None,
                   exp_avg_scales=[s["exp_avg_scale"] for s in states] if bits8 else None,
                   exp_avg_sq_scales=[s["exp_avg_sq_scale"] for s in states] if bits8 else None,
                   seed=seed)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        todo = []      # (every group is checked before the first one's step)
        for number, group in enumerate(self.param_groups):
            params = group["params"]
            used = [i for i, p in enumerate(params) if p.grad is not None]
            if not used:
                continue
            types = sorted({params[i].dtype for i in used}, key=str)
            if len(types) > 1:
                raise ValueError(f"a parameter group holds {types}: one type a group")
            todo.append((number, group, self._parts(group, used)))
            for i in used:
                self._state_of(params[i], group)
        for number, group, parts in todo:
            if len(group["counts"]) > 1:   # (a single count is the group's, too)
                if group["step"] is group["counts"][0]:
                    group["step"] = group["step"].clone()
                group["step"].add_(1)
            for count, members in parts:
                self._step_of(group, [group["params"][i] for i in members], group["counts"][count],
                              _seed_of(group["seed"], number, count))
        return loss

    def load_state_dict(self, state_dict) -> None:
        """As torch's, but each state keeps the type it was saved with (torch
        casts it to the parameter's)."""
        super().load_state_dict(state_dict)
        for group, saved in zip(self.param_groups, state_dict["param_groups"]):
            for p, key in zip(group["params"], saved["params"]):
                if key in state_dict["state"]:
                    self.state[p] = {name: v.detach().to(p.device, copy=True) if isinstance(v, torch.Tensor) else v
                                     for name, v in state_dict["state"][key].items()}
            if isinstance(group.get("step"), torch.Tensor) and group["params"]:
                device = group["params"][0].device
                # (none in a state that was saved when steps were counted by group only)
                if "counts" in saved:
                    group["counts"] = [t.detach().to(device, copy=True) for t in saved["counts"]]
                    group["count_of"] = list(saved["count_of"])
                group["step"] = group["counts"][0] if len(saved.get("counts", ())) == 1 \
                    else saved["step"].detach().to(device, copy=True)
        self.__dict__["_captured"] = []
