"""Operators of a layer over signature tokens: argument marshalling for the norm, the matrix product and the gated recurrence of include/sig.h.

Tokens are CUDA tensors with contiguous channels in float32 or bfloat16, [batch, time, channels] or [batch, channels]; rows that lie evenly
spaced in memory (slices of a wider projection, broadcasts) are taken as they are, other layouts are copied once.  The norm's weight, the
recurrence's rates and states, scales and their gradients are float32; a product's weight and bias have the tokens' type.  Every call enqueues on
torch's current stream and returns without synchronising; results are plain tensors without autograd history, the gradients have functions
of their own.  States that a call updates in place do not raise the tensors' version counters.
"""
from __future__ import annotations

import struct

from . import sequence as _s
from .binding import _enqueue
from .sequence import _in_place, _refuse, _scratch, _t, _tokens, _whole

_NORM = struct.Struct("5qd3q")
_LINEAR = struct.Struct("14q")
_GATED = struct.Struct("16q")
_GATED_GRADS = struct.Struct("9q")
_ACTS = {None: 0, "silu": 1, "gelu": 2}
_MOST_STRIDE = 1 << 38
_REACH = 1 << 22                                             # time strides from there on are copied away: the recurrence's kernels do not reach them


def _like(make, shape):
    """An uninitialised contiguous tensor of make's type: its own shape costs half a microsecond less by this way."""
    return _s._torch.empty_like(make) if make.shape == shape and make.is_contiguous() else make.new_empty(shape)


def _start(x, name="x"):
    """Checks a tensor of tokens; returns what makes the outputs (a plain tensor on its device, of its type), and the code of its type."""
    if _s._torch is None:
        _t()
    t = x.dtype
    if not x.is_cuda or (t is not _s._f32 and t is not _s._b16) or x.dim() not in (2, 3) or x.shape[-1] < 1:
        raise ValueError(f"{name} must be a float32 or bfloat16 CUDA tensor [B, L, D] or [B, D]")
    return x if type(x) is _s._plain else _s._torch.empty(0, dtype=t, device=x.device), 1 if t is _s._b16 else 0


def _rows(name, t, shape, dtype, index):
    """Checks tokens and returns them as evenly spaced rows: (tensor to keep alive, stride of a row)."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        _refuse(name, t, shape, dtype)
    if t.is_contiguous():
        return t, shape[-1]
    s = t.stride()
    if s[-1] == 1 or shape[-1] == 1:
        if len(s) == 2 or shape[0] <= 1:
            step = s[-2] if shape[-2] > 1 else 0
        elif shape[1] <= 1:
            step = s[0]
        else:
            step = s[1] if s[0] == shape[1] * s[1] else -1
        if 0 <= step <= _MOST_STRIDE:
            return t, step
    t = t.contiguous()
    return t, shape[-1]


def _count(shape):
    return shape[0] if len(shape) == 2 else shape[0] * shape[1]


def sig_norm_forward(x, weight, residual=None, eps=1e-6, quantize=False):
    """Root-mean-square norm of the sum total = x + residual (rounded to their type; x itself without residual):
    y = total * rsqrt(mean(total^2) + eps) * weight over the last axis.

    x, residual [B, L, D] or [B, D]; weight float32 [D].  Returns (y, total); with quantize=True (y, scale, total): y in float8_e4m3fn, and
    scale float32 [B, L] or [B] with y * scale the norm (scale = largest magnitude of the row / 448), as sig_linear_forward takes them."""
    make, kind = _start(x)
    shape, index, t = x.shape, x.get_device(), x.dtype
    D = shape[-1]
    weight = _whole("weight", weight, (D,), _s._f32, index)
    if not 0 <= eps < float("inf"):
        raise ValueError("eps must be finite and not negative")
    kept, sx = _rows("x", x, shape, t, index)
    sr = pr = pt = 0
    total = x
    if residual is not None:
        residual, sr = _rows("residual", residual, shape, t, index)
        pr = residual.data_ptr()
        total = _like(make, shape)
        pt = total.data_ptr()
    args = _NORM.pack(kind, _count(shape), D, sx, sr, eps, kept.data_ptr(), pr, weight.data_ptr())
    if quantize:
        y, scale = make.new_empty(shape, dtype=_s._torch.float8_e4m3fn), make.new_empty(shape[:-1], dtype=_s._f32)
        _enqueue(x.device, "sig_norm_forward", args, y.data_ptr(), scale.data_ptr(), pt)
        return y, scale, total
    y = _like(make, shape)
    _enqueue(x.device, "sig_norm_forward", args, y.data_ptr(), 0, pt)
    return y, total


def sig_norm_backward(total, weight, grad_out, grad_total=None, eps=1e-6):
    """Gradient of sig_norm_forward from the total that it returned: (grad_x, grad_weight), grad_x for x and residual alike.  grad_total: the
    gradient of total by its other uses, which is added.  (With quantize=True this is the gradient of the norm before its rounding to 8 bits.)"""
    make, kind = _start(total, "total")
    shape, index, t = total.shape, total.get_device(), total.dtype
    D = shape[-1]
    weight = _whole("weight", weight, (D,), _s._f32, index)
    if not 0 <= eps < float("inf"):
        raise ValueError("eps must be finite and not negative")
    total, sx = _rows("total", total, shape, t, index)
    grad_out, sy = _rows("grad_out", grad_out, shape, t, index)
    st = pt = 0
    if grad_total is not None:
        grad_total, st = _rows("grad_total", grad_total, shape, t, index)
        pt = grad_total.data_ptr()
    args = _NORM.pack(kind, _count(shape), D, sx, 0, eps, total.data_ptr(), 0, weight.data_ptr())
    gx, gw = _like(make, shape), make.new_empty(D, dtype=_s._f32)
    keep, wptr, nbytes = _scratch(make, "sig_norm_backward_workspace_bytes", args)
    _enqueue(total.device, "sig_norm_backward", args, grad_out.data_ptr(), sy, pt, st, gx.data_ptr(), gw.data_ptr(), wptr, nbytes)
    return gx, gw


def sig_quantize(x):
    """Rows of x [.., D] in 8 bits: (q float8_e4m3fn [.., D], scale float32 [..]) with q * scale about x, scale = largest magnitude of the row / 448.
    For tokens that no norm gives, and for weights [N, K] of sig_linear_forward."""
    make, kind = _start(x)
    shape = x.shape
    kept, sx = _rows("x", x, shape, x.dtype, x.get_device())
    q, scale = make.new_empty(shape, dtype=_s._torch.float8_e4m3fn), make.new_empty(shape[:-1], dtype=_s._f32)
    _enqueue(x.device, "sig_quantize", kind, _count(shape), shape[-1], sx, kept.data_ptr(), q.data_ptr(), scale.data_ptr())
    return q, scale


def _act(activation):
    try:
        return _ACTS[activation]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be None, 'silu' or 'gelu', got {activation!r}") from None


def sig_linear_forward(x, weight, bias=None, residual=None, activation=None, keep=False, x_scale=None, weight_scale=None, dtype=None):
    """y = f(x weight^T + bias) + residual, f None (the identity), "silu" or "gelu" (z Phi(z), by the error function).

    x [B, L, K] or [B, K], weight [N, K] and bias [N] of x's type, residual [.., N] likewise.  x and weight in float8_e4m3fn: x_scale float32 [B, L] or [B]
    and weight_scale float32 [N] say what their rows are to be multiplied by (None: one), y, bias and residual are of `dtype` (bfloat16 or
    float32, default bfloat16).  Returns y, or with keep=True (y, pre): what f was applied to, for sig_linear_backward (None without activation)."""
    torch = _t()
    act = _act(activation)
    eight = x.dtype is torch.float8_e4m3fn
    if not x.is_cuda or x.dim() not in (2, 3) or not (eight or x.dtype is _s._f32 or x.dtype is _s._b16):
        raise ValueError("x must be a float32, bfloat16 or float8_e4m3fn CUDA tensor [B, L, K] or [B, K]")
    shape, index, t = x.shape, x.get_device(), x.dtype
    out = (_s._b16 if dtype is None else dtype) if eight else t
    if out is not _s._f32 and out is not _s._b16:
        raise ValueError("dtype must be float32 or bfloat16")
    if not eight and (x_scale is not None or weight_scale is not None or (dtype is not None and dtype is not t)):
        raise ValueError("x_scale, weight_scale and another dtype belong to float8_e4m3fn inputs")
    K = shape[-1]
    if weight.dim() != 2 or weight.shape[0] < 1 or K < 1:
        raise ValueError("weight must be [N, K] with N, K >= 1")
    N = weight.shape[0]
    outs = (*shape[:-1], N)
    make = x if type(x) is _s._plain else torch.empty(0, dtype=t, device=x.device)
    x, sx = _rows("x", x, shape, t, index)
    weight = _whole("weight", weight, (N, K), t, index)
    pb = pr = sr = px = pw = 0
    if bias is not None:
        bias = _whole("bias", bias, (N,), out, index)
        pb = bias.data_ptr()
    if residual is not None:
        residual, sr = _rows("residual", residual, outs, out, index)
        pr = residual.data_ptr()
    if x_scale is not None:
        x_scale = _whole("x_scale", x_scale, shape[:-1], _s._f32, index)
        px = x_scale.data_ptr()
    if weight_scale is not None:
        weight_scale = _whole("weight_scale", weight_scale, (N,), _s._f32, index)
        pw = weight_scale.data_ptr()
    kind = 0 if out is _s._f32 else 1
    args = _LINEAR.pack(2 if eight else kind, kind, _count(shape), N, K, act, sx, sr, x.data_ptr(), weight.data_ptr(), pb, pr, px, pw)
    y = make.new_empty(outs, dtype=out)
    pre = make.new_empty(outs, dtype=out) if keep and act else None
    kept, wptr, nbytes = _scratch(make, "sig_linear_forward_workspace_bytes", args)
    _enqueue(x.device, "sig_linear_forward", args, y.data_ptr(), 0 if pre is None else pre.data_ptr(), wptr, nbytes)
    return (y, pre) if keep else y


def sig_linear_backward(x, weight, grad_out, activation=None, pre=None, bias=False, need_x=True, need_weight=True):
    """Gradient of sig_linear_forward: (grad_x, grad_weight, grad_bias) of x's type, None for those not asked for (need_x, need_weight, bias).
    grad_out [.., N] of x's type; pre: what the forward call with keep=True returned, needed with an activation.  The residual's gradient is
    grad_out itself.  grad_out times the activation's slope at pre is rounded to x's type before the products for grad_x and grad_weight (not for
    grad_bias): in bfloat16 their norms are 2.4e-3 off, with outputs rounded alone 1.7e-3."""
    make, kind = _start(x)
    act = _act(activation)
    shape, index, t = x.shape, x.get_device(), x.dtype
    if weight.dim() != 2 or weight.shape[0] < 1:
        raise ValueError("weight must be [N, K] with N, K >= 1")
    N, K = weight.shape[0], shape[-1]
    outs = (*shape[:-1], N)
    x, sx = _rows("x", x, shape, t, index)
    weight = _whole("weight", weight, (N, K), t, index)
    grad_out, sg = _rows("grad_out", grad_out, outs, t, index)
    pp = 0
    if act:
        if pre is None:
            raise ValueError("pre is missing: call sig_linear_forward with keep=True")
        pre = _whole("pre", pre, outs, t, index)
        pp = pre.data_ptr()
    args = _LINEAR.pack(kind, kind, _count(shape), N, K, act, sx, 0, x.data_ptr(), weight.data_ptr(), 0, 0, 0, 0)
    gx = _like(make, shape) if need_x else None
    gw = make.new_empty((N, K)) if need_weight else None
    gb = make.new_empty(N) if bias else None
    kept, wptr, nbytes = _scratch(make, "sig_linear_backward_workspace_bytes", args)
    _enqueue(x.device, "sig_linear_backward", args, grad_out.data_ptr(), sg, pp, 0 if gx is None else gx.data_ptr(), 0 if gw is None else gw.data_ptr(),
             0 if gb is None else gb.data_ptr(), wptr, nbytes)
    return gx, gw, gb


def _gated_args(x, decay_gate, input_gate, log_rate, initial_state, lengths):
    make, kind = _start(x)
    shape, index, t = x.shape, x.get_device(), x.dtype
    if len(shape) != 3:
        raise ValueError("x must be [B, L, D]")
    B, L, D = shape
    x, xs = _tokens("x", x, shape, t, index, _REACH)
    decay_gate, ps = _tokens("decay_gate", decay_gate, shape, t, index, _REACH)
    input_gate, qs = _tokens("input_gate", input_gate, shape, t, index, _REACH)
    log_rate = _whole("log_rate", log_rate, (D,), _s._f32, index)
    pi = pl = 0
    if initial_state is not None:
        initial_state = _whole("initial_state", initial_state, (B, D), _s._f32, index)
        pi = initial_state.data_ptr()
    if lengths is not None:
        lengths = _whole("lengths", lengths, (B,), _s._i32, index)
        pl = lengths.data_ptr()
    args = _GATED.pack(kind, B, L, D, xs[0], xs[1], ps[0], ps[1], qs[0], qs[1], x.data_ptr(), decay_gate.data_ptr(), input_gate.data_ptr(), log_rate.data_ptr(), pi, pl)
    return make, args, (x, decay_gate, input_gate, log_rate, initial_state, lengths)


def sig_gated_scan_forward(x, decay_gate, input_gate, log_rate, initial_state=None, lengths=None, checkpoint=False):
    """Gated linear recurrence y_t = h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(input_gate_t) x_t, a_t = exp(-exp(log_rate) sigmoid(decay_gate_t)).

    x, decay_gate, input_gate [B, L, D]; log_rate float32 [D]; initial_state float32 [B, D] (default zeros); lengths int32 [B]: tokens from there on
    are not read, give zeros and leave the state.  Returns (y [B, L, D], final state float32 [B, D]); with checkpoint=True a third
    tensor for sig_gated_scan_backward."""
    make, args, kept = _gated_args(x, decay_gate, input_gate, log_rate, initial_state, lengths)
    B, L, D = x.shape
    y, state = _like(make, x.shape), make.new_empty((B, D), dtype=_s._f32)
    ck, cptr, cbytes = _scratch(make, "sig_gated_scan_checkpoint_bytes", args) if checkpoint else (None, 0, 0)
    keep, wptr, nbytes = _scratch(make, "sig_gated_scan_forward_workspace_bytes", args)
    _enqueue(x.device, "sig_gated_scan_forward", args, y.data_ptr(), state.data_ptr(), cptr, cbytes, wptr, nbytes)
    if not checkpoint:
        return y, state
    return y, state, ck if ck is not None else make.new_empty(0, dtype=_s._torch.uint8)


def sig_gated_scan_backward(x, decay_gate, input_gate, log_rate, grad_out, checkpoint, initial_state=None, lengths=None, grad_final_state=None):
    """Gradient of sig_gated_scan_forward, whose `checkpoint` it reads: a dict of the gradients "x", "decay_gate", "input_gate", "log_rate" and
    "initial_state" (None where the input is None).  grad_out [B, L, D] of x's type, grad_final_state float32 [B, D] or None."""
    make, args, kept = _gated_args(x, decay_gate, input_gate, log_rate, initial_state, lengths)
    B, L, D = x.shape
    index = x.get_device()
    grad_out, (sb, st, _) = _tokens("grad_out", grad_out, x.shape, x.dtype, index, _REACH)
    pf = 0
    if grad_final_state is not None:
        grad_final_state = _whole("grad_final_state", grad_final_state, (B, D), _s._f32, index)
        pf = grad_final_state.data_ptr()
    if checkpoint is None or checkpoint.get_device() != index or not checkpoint.is_contiguous():
        raise ValueError("checkpoint must be the tensor that sig_gated_scan_forward returned")
    g = {k: _like(make, x.shape) for k in ("x", "decay_gate", "input_gate")}
    g["log_rate"] = make.new_empty(D, dtype=_s._f32)
    g["initial_state"] = make.new_empty((B, D), dtype=_s._f32) if initial_state is not None else None
    ptr = lambda v: 0 if v is None else v.data_ptr()                                        # noqa: E731
    grads = _GATED_GRADS.pack(sb, st, grad_out.data_ptr(), pf, *(ptr(g[k]) for k in ("x", "decay_gate", "input_gate", "log_rate", "initial_state")))
    keep, wptr, nbytes = _scratch(make, "sig_gated_scan_backward_workspace_bytes", args)
    _enqueue(x.device, "sig_gated_scan_backward", args, grads, checkpoint.data_ptr(), checkpoint.numel() * checkpoint.element_size(), wptr, nbytes)
    return g


def sig_gated_scan_step(x, decay_gate, input_gate, log_rate, state):
    """One token of every stream: x, decay_gate, input_gate [B, D]; state float32 [B, D] is updated in place.  Returns y [B, D]."""
    make, kind = _start(x)
    shape, index, t = x.shape, x.get_device(), x.dtype
    if len(shape) != 2:
        raise ValueError("x must be [B, D]")
    B, D = shape
    x, sx = _rows("x", x, shape, t, index)
    decay_gate, sp = _rows("decay_gate", decay_gate, shape, t, index)
    input_gate, sq = _rows("input_gate", input_gate, shape, t, index)
    log_rate = _whole("log_rate", log_rate, (D,), _s._f32, index)
    _in_place("state", state, shape, _s._f32, index)
    y = _like(make, shape)
    _enqueue(make.device, "sig_gated_scan_step", _GATED.pack(kind, B, 1, D, sx, 0, sp, 0, sq, 0, x.data_ptr(), decay_gate.data_ptr(), input_gate.data_ptr(), log_rate.data_ptr(), 0, 0),
             state.data_ptr(), y.data_ptr())
    return y
