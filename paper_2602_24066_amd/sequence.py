"""Sequence operators over signature tokens: argument marshalling for the calls of include/sig.h that follow a signature in a model.

Tokens are CUDA tensors [batch, time, channels] in float32 or bfloat16, with contiguous channels (a slice of a wider projection is taken as
it is; other layouts are copied once).  Parameters, recurrent states of the scan and their gradients are float32.  Every call enqueues
on torch's current stream and returns without synchronising; results are plain tensors without autograd history, the gradients have
functions of their own.  What a call writes in place (the states of the single-token calls, clipped gradients) does not raise the tensors'
version counters: autograd does not notice where it kept them for a backward pass.
"""
from __future__ import annotations

import array
import struct

from .binding import _call, _calls, _enqueue

# torch and its types, set by the first call; the checks below are written for calls of one token, whose kernels take less time than they do
_torch = _f32 = _b16 = _i32 = _plain = _KINDS = None


def _t():
    global _torch, _f32, _b16, _i32, _plain, _KINDS
    if _torch is None:
        import torch
        _f32, _b16, _i32, _plain = torch.float32, torch.bfloat16, torch.int32, torch.Tensor
        _KINDS = {_f32: 0, _b16: 1}
        _torch = torch
    return _torch


def _refuse(name, t, shape, dtype):
    raise ValueError(f"{name} must be a tensor of type {dtype} and shape {tuple(shape)} on the device of x, got {t.dtype}, {tuple(t.shape)}, {t.device}")


def _first(x, dims):
    """Checks x; returns what makes the outputs, and the code of its type."""
    if _torch is None:
        _t()
    t = x.dtype
    if not x.is_cuda or x.dim() != dims or (t is not _f32 and t is not _b16):
        raise ValueError("x must be a float32 or bfloat16 CUDA tensor " + ("[B, L, D]" if dims == 3 else "[B, D]"))
    return x if type(x) is _plain else _torch.empty(0, dtype=t, device=x.device), 1 if t is _b16 else 0


def _tokens(name, t, shape, dtype, index, most=1 << 24):
    """Checks a tensor of tokens; returns it with a contiguous last axis, and its strides.  most: time strides from there on are copied away (the scan's
    kernels do not reach them; the convolution's reach any)."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        _refuse(name, t, shape, dtype)
    s = t.stride()
    if (s[-1] != 1 and shape[-1] != 1) or (most and len(s) > 2 and s[1] >= most):
        t = t.contiguous()
        s = t.stride()
        if len(s) > 2 and (shape[1] <= 1 or t.numel() == 0):                         # such an axis keeps any stride, and nothing is reached by it
            s = (s[0], 0, *s[2:])
    return t, s


def _whole(name, t, shape, dtype, index):
    """Checks a parameter, state or list of lengths and returns it contiguous."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        _refuse(name, t, shape, dtype)
    return t if t.is_contiguous() else t.contiguous()


def _in_place(name, t, shape, dtype, index):
    if t is None:
        raise ValueError(f"{name} is missing")
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or not t.is_contiguous():
        _refuse(name + " (contiguous)", t, shape, dtype)


def _scratch(make, name, args):
    """The workspace a call asks for: (tensor to keep alive, address, bytes)."""
    n = (_calls.get(name) or _call(name))(args)
    if n == 0:
        return None, 0, 0
    t = make.new_empty(n, dtype=_torch.uint8)
    return t, t.data_ptr(), n


_CONV = struct.Struct("13q")


def _conv_args(x, weight, bias, initial_state, lengths, silu):
    make, kind = _first(x, 3)
    B, L, D = shape = x.shape
    index = x.get_device()
    if weight.dim() != 2 or not 1 <= weight.shape[1] <= 8:
        raise ValueError("weight must be [D, W] with W <= 8")
    W = weight.shape[1]
    x, (sb, st, _) = _tokens("x", x, shape, x.dtype, index, 0)
    weight = _whole("weight", weight, (D, W), _f32, index)
    pb = pi = pl = 0
    if bias is not None:
        bias = _whole("bias", bias, (D,), _f32, index)
        pb = bias.data_ptr()
    if initial_state is not None:
        initial_state = _whole("initial_state", initial_state, (B, W - 1, D), x.dtype, index)
        pi = initial_state.data_ptr()
    if lengths is not None:
        lengths = _whole("lengths", lengths, (B,), _i32, index)
        pl = lengths.data_ptr()
    args = _CONV.pack(kind, B, L, D, W, 1 if silu else 0, sb, st, x.data_ptr(), weight.data_ptr(), pb, pi, pl)
    return make, args, W, (x, weight, bias, initial_state, lengths)


def sig_conv_forward(x, weight, bias=None, initial_state=None, lengths=None, silu=True, return_state=False):
    """Causal depthwise convolution y_t = f(bias + sum_k weight[:, k] x_{t-W+1+k}), f(s) = s sigmoid(s) or (silu=False) s.

    x [B, L, D]; weight float32 [D, W], W <= 8; bias float32 [D]; initial_state [B, W-1, D] of x's type: the tokens before the first, oldest
    first (default zeros); lengths int32 [B]: tokens from there on are not read and give zeros.  Returns y [B, L, D], or with
    return_state (y, state): the last W-1 tokens of every stream, for sig_conv_step or the next prompt's initial_state."""
    make, args, W, kept = _conv_args(x, weight, bias, initial_state, lengths, silu)
    B, L, D = x.shape
    y = make.new_empty((B, L, D))
    state = make.new_empty((B, W - 1, D)) if return_state else None
    _enqueue(x.device, "sig_conv_forward", args, y.data_ptr(), state.data_ptr() if return_state else 0)
    return (y, state) if return_state else y


def sig_conv_backward(x, weight, grad_out, bias=None, initial_state=None, lengths=None, silu=True, grad_final_state=None):
    """Gradient of sig_conv_forward: (grad_x, grad_weight, grad_bias, grad_initial_state), None for those whose input is None.
    grad_out [B, L, D] and grad_final_state [B, W-1, D] are of x's type."""
    make, args, W, kept = _conv_args(x, weight, bias, initial_state, lengths, silu)
    B, L, D = x.shape
    t, index = x.dtype, x.get_device()
    grad_out, (sb, st, _) = _tokens("grad_out", grad_out, x.shape, t, index, 0)
    pf = 0
    if grad_final_state is not None:
        grad_final_state = _whole("grad_final_state", grad_final_state, (B, W - 1, D), t, index)
        pf = grad_final_state.data_ptr()
    gx, gw = make.new_empty((B, L, D)), make.new_empty((D, W), dtype=_f32)
    gb = make.new_empty(D, dtype=_f32) if bias is not None else None
    gi = make.new_empty((B, W - 1, D)) if initial_state is not None else None
    keep, wptr, nbytes = _scratch(make, "sig_conv_backward_workspace_bytes", args)
    _enqueue(x.device, "sig_conv_backward", args, grad_out.data_ptr(), sb, st, pf, gx.data_ptr(), gw.data_ptr(), 0 if gb is None else gb.data_ptr(),
             0 if gi is None else gi.data_ptr(), wptr, nbytes)
    return gx, gw, gb, gi


def sig_conv_step(x, state, weight, bias=None, silu=True):
    """One token of every stream: x [B, D], state [B, W-1, D] of x's type, shifted by it in place.  Returns y [B, D]."""
    make, kind = _first(x, 2)
    B, D = shape = x.shape
    t, index = x.dtype, x.get_device()
    if weight.dim() != 2 or not 1 <= weight.shape[1] <= 8:
        raise ValueError("weight must be [D, W] with W <= 8")
    W = weight.shape[1]
    x, (sb, _) = _tokens("x", x, shape, t, index)
    weight = _whole("weight", weight, (D, W), _f32, index)
    pb = 0
    if bias is not None:
        bias = _whole("bias", bias, (D,), _f32, index)
        pb = bias.data_ptr()
    _in_place("state", state, (B, W - 1, D), t, index)
    y = make.new_empty((B, D))
    _enqueue(x.device, "sig_conv_step", _CONV.pack(kind, B, 1, D, W, 1 if silu else 0, sb, 0, x.data_ptr(), weight.data_ptr(), pb, 0, 0),
             state.data_ptr(), y.data_ptr())
    return y


_SCAN = struct.Struct("29q")
_SCAN_GRADS = struct.Struct("13q")


def _scan_args(x, dt, A, b, c, skip, gate, dt_bias, softplus, initial_state, lengths, dims):
    make, kind = _first(x, dims)
    shape = x.shape
    D, t, index = shape[-1], x.dtype, x.get_device()
    if b.dim() == dims:                                                                     # one group
        b = b.unsqueeze(-2)
    if c.dim() == dims:
        c = c.unsqueeze(-2)
    G, N = b.shape[-2:]
    if G < 1 or D % G or not 1 <= N <= 64:
        raise ValueError("b and c must be [..., groups, states] or [..., states], the groups dividing the channels, of 1 to 64 states")
    x, xs = _tokens("x", x, shape, t, index)
    dt, ts = _tokens("dt", dt, shape, t, index)
    of_bc = (*shape[:-1], G, N)
    b, bs = _tokens("b", b, of_bc, t, index)
    c, cs = _tokens("c", c, of_bc, t, index)
    pz = ps = pd = pi = pl = 0
    zs = (0, 0, 0)
    if gate is not None:
        gate, zs = _tokens("gate", gate, shape, t, index)
        pz = gate.data_ptr()
    if A is None:
        raise ValueError("A is missing")
    A = _whole("A", A, (D, N), _f32, index)
    if skip is not None:
        skip = _whole("skip", skip, (D,), _f32, index)
        ps = skip.data_ptr()
    if dt_bias is not None:
        dt_bias = _whole("dt_bias", dt_bias, (D,), _f32, index)
        pd = dt_bias.data_ptr()
    if dims == 3:
        B, L, _ = shape
        if 0 < bs[1] < N:                                                                   # windows that overlap are copied
            b = b.contiguous()
            bs = b.stride()
        if 0 < cs[1] < N:
            c = c.contiguous()
            cs = c.stride()
        if initial_state is not None:
            initial_state = _whole("initial_state", initial_state, (B, D, N), _f32, index)
            pi = initial_state.data_ptr()
        if lengths is not None:
            lengths = _whole("lengths", lengths, (B,), _i32, index)
            pl = lengths.data_ptr()
        args = _SCAN.pack(kind, B, L, D, G, N, 1 if softplus else 0, xs[0], xs[1], ts[0], ts[1], zs[0], zs[1], bs[0], bs[1], bs[2], cs[0], cs[1], cs[2],
                          x.data_ptr(), dt.data_ptr(), pz, b.data_ptr(), c.data_ptr(), A.data_ptr(), ps, pd, pi, pl)
    else:
        args = _SCAN.pack(kind, shape[0], 1, D, G, N, 1 if softplus else 0, xs[0], 0, ts[0], 0, zs[0], 0, bs[0], 0, bs[1], cs[0], 0, cs[1],
                          x.data_ptr(), dt.data_ptr(), pz, b.data_ptr(), c.data_ptr(), A.data_ptr(), ps, pd, 0, 0)
    return make, args, G, N, (x, dt, A, b, c, skip, gate, dt_bias, initial_state, lengths)


def sig_scan_forward(x, dt, A, b, c, skip=None, gate=None, dt_bias=None, softplus=True, initial_state=None, lengths=None, checkpoint=False):
    """Selective state space scan: h_t = exp(delta_t A) h_{t-1} + delta_t x_t b_t, y_t = (sum_n c_t h_t + skip x_t) silu(gate_t), with
    delta_t = softplus(dt_t + dt_bias) (softplus=False: the sum itself).

    x, dt, gate [B, L, D]; b, c [B, L, G, N] or [B, L, N]: channel d uses group d // (D // G); A float32 [D, N]; skip, dt_bias float32 [D];
    initial_state float32 [B, D, N] (default zeros); lengths int32 [B]: tokens from there on are not read, give zeros and leave the
    state.  Returns (y [B, L, D], final state float32 [B, D, N]); with checkpoint=True a third tensor for sig_scan_backward."""
    make, args, G, N, kept = _scan_args(x, dt, A, b, c, skip, gate, dt_bias, softplus, initial_state, lengths, 3)
    B, L, D = x.shape
    y = make.new_empty((B, L, D))
    state = make.new_empty((B, D, N), dtype=_f32)
    ck, cptr, cbytes = _scratch(make, "sig_scan_checkpoint_bytes", args) if checkpoint else (None, 0, 0)
    keep, wptr, nbytes = _scratch(make, "sig_scan_forward_workspace_bytes", args)
    _enqueue(x.device, "sig_scan_forward", args, y.data_ptr(), state.data_ptr(), cptr, cbytes, wptr, nbytes)
    if not checkpoint:
        return y, state
    return y, state, ck if ck is not None else make.new_empty(0, dtype=_torch.uint8)


def sig_scan_backward(x, dt, A, b, c, grad_out, checkpoint, skip=None, gate=None, dt_bias=None, softplus=True, initial_state=None, lengths=None,
                      grad_final_state=None):
    """Gradient of sig_scan_forward, whose `checkpoint` it reads: a dict of the gradients "x", "dt", "A", "B", "C", "skip", "gate", "dt_bias"
    and "initial_state", None for those whose input is None.  grad_out [B, L, D] of x's type, grad_final_state float32 [B, D, N] or None."""
    make, args, G, N, kept = _scan_args(x, dt, A, b, c, skip, gate, dt_bias, softplus, initial_state, lengths, 3)
    B, L, D = x.shape
    t, index = x.dtype, x.get_device()
    grad_out, (sb, st, _) = _tokens("grad_out", grad_out, x.shape, t, index)
    pf = 0
    if grad_final_state is not None:
        grad_final_state = _whole("grad_final_state", grad_final_state, (B, D, N), _f32, index)
        pf = grad_final_state.data_ptr()
    if checkpoint is None or checkpoint.get_device() != index or not checkpoint.is_contiguous():
        raise ValueError("checkpoint must be the tensor that sig_scan_forward returned")
    tokens = lambda: make.new_empty((B, L, D))                                              # noqa: E731
    params = lambda *shape: make.new_empty(shape, dtype=_f32)                               # noqa: E731
    of_bc = lambda v: (B, L, N) if v.dim() == 3 else (B, L, G, N)                           # noqa: E731
    g = {"x": tokens(), "dt": tokens(), "A": params(D, N), "B": make.new_empty(of_bc(b)), "C": make.new_empty(of_bc(c)),
         "skip": params(D) if skip is not None else None, "gate": tokens() if gate is not None else None,
         "dt_bias": params(D) if dt_bias is not None else None, "initial_state": params(B, D, N) if initial_state is not None else None}
    ptr = lambda v: 0 if v is None else v.data_ptr()                                        # noqa: E731
    grads = _SCAN_GRADS.pack(sb, st, grad_out.data_ptr(), pf, ptr(g["x"]), ptr(g["dt"]), ptr(g["gate"]), ptr(g["B"]), ptr(g["C"]), ptr(g["A"]),
                             ptr(g["skip"]), ptr(g["dt_bias"]), ptr(g["initial_state"]))
    keep, wptr, nbytes = _scratch(make, "sig_scan_backward_workspace_bytes", args)
    _enqueue(x.device, "sig_scan_backward", args, grads, checkpoint.data_ptr(), checkpoint.numel() * checkpoint.element_size(), wptr, nbytes)
    return g


def sig_scan_step(x, dt, A, b, c, state, skip=None, gate=None, dt_bias=None, softplus=True):
    """One token of every stream: x, dt, gate [B, D], b, c [B, G, N] or [B, N]; state float32 [B, D, N] is updated in place.  Returns y [B, D]."""
    make, args, G, N, kept = _scan_args(x, dt, A, b, c, skip, gate, dt_bias, softplus, None, None, 2)
    B, D = shape = x.shape
    _in_place("state", state, (B, D, N), _f32, x.get_device())
    y = make.new_empty(shape)
    _enqueue(x.device, "sig_scan_step", args, state.data_ptr(), y.data_ptr())
    return y


def sig_grad_clip(grads, max_norm, out=None):
    """Scales the tensors `grads` (float32 or bfloat16, one device) in place by min(1, max_norm / (norm + 1e-6)), norm their global 2-norm, or
    writes the products into the tensors `out` (of as many elements, either type).  Returns norm, a float32 tensor of no axes on the
    device.  Tensors may have any order of axes as long as they fill their memory; those of `out` have that of their input.  Apart from
    that, no tensor that is written may share memory with another (as a gradient that is listed twice does): the order of accesses is not fixed."""
    torch = _t()
    grads = list(grads)
    outs = grads if out is None else list(out)
    n = len(grads)
    if len(outs) != n:
        raise ValueError("out must have a tensor for each of grads")
    if not max_norm >= 0:
        raise ValueError("max_norm must not be negative")
    dev = grads[0].device if n else torch.device("cuda", torch.cuda.current_device())
    if dev.type != "cuda":
        raise ValueError("grads must be CUDA tensors")
    # by calls mapped over the lists: with a few dozen small tensors these checks take longer than the kernels
    T, every = torch.Tensor, grads if out is None else grads + outs
    kinds = [_KINDS.get(t.dtype) for t in every]
    if None in kinds or not set(map(T.get_device, every)) <= {dev.index}:
        raise ValueError("grads and out must be float32 or bfloat16 tensors on one device")
    into, sizes = list(map(T.data_ptr, every)), list(map(T.numel, every))
    if out is not None and sizes[:n] != sizes[n:]:
        raise ValueError("out must have tensors of the sizes of grads")
    if not all(map(T.is_contiguous, every)):
        for g, o in zip(grads, outs):
            if not (g.is_contiguous() and o.is_contiguous()) and (g.shape != o.shape or g.stride() != o.stride() or not torch.ops.aten.is_non_overlapping_and_dense(g)):
                raise ValueError("every tensor must fill its memory, and out must have the order of axes of grads")
    tab = array.array("q", into + sizes[:n] + kinds if out is not None else into + into + sizes + kinds + kinds)
    at = tab.buffer_info()[0]
    norm = torch.empty((), dtype=_f32, device=dev)
    nbytes = (_calls.get("sig_grad_clip_workspace_bytes") or _call("sig_grad_clip_workspace_bytes"))(n, at + 16 * n)
    keep = norm.new_empty(nbytes, dtype=torch.uint8)
    _enqueue(dev, "sig_grad_clip", n, at, at + 8 * n, at + 16 * n, at + 24 * n, at + 32 * n, float(max_norm), norm.data_ptr(), keep.data_ptr(), nbytes)
    return norm
