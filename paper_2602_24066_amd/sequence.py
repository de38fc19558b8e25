"""Sequence operators over signature tokens: argument marshalling for the calls of include/sig.h that follow a signature in a model.

Tokens are CUDA tensors [batch, time, channels] in float32 or bfloat16, with contiguous channels (a slice of a wider projection is taken as
it is; other layouts are copied once).  Parameters, recurrent states of the scan and their gradients are float32.  Every call enqueues
on torch's current stream and returns without synchronising; results are plain tensors without autograd history, the gradients have
functions of their own.
"""
from __future__ import annotations

import array
import struct

from .binding import _call, _calls, _enqueue

_torch = None


def _t():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _tokens(name, t, shape, like):
    """Checks a tensor of tokens against the type and device of `like`; its last axis is contiguous on return."""
    if t.dtype is not like.dtype or t.device != like.device:
        raise ValueError(f"{name} must be of type {like.dtype} on {like.device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t if t.stride(-1) == 1 or shape[-1] == 1 else t.contiguous()


def _whole(name, t, shape, dtype, device):
    """Checks a parameter, state or list of lengths and returns it contiguous; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} must be of type {dtype} on {device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t if t.is_contiguous() else t.contiguous()


def _in_place(name, t, shape, dtype, device):
    if t is None or t.dtype is not dtype or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of type {dtype} and shape {tuple(shape)} on {device}")
    return t


def _first(x, dims):
    torch = _t()
    if not x.is_cuda or x.dim() != dims or x.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("x must be a float32 or bfloat16 CUDA tensor " + ("[B, L, D]" if dims == 3 else "[B, D]"))
    return torch, int(x.dtype is torch.bfloat16)


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _scratch(torch, name, args, device):
    """The workspace a call asks for: (tensor to keep alive, address, bytes)."""
    n = (_calls.get(name) or _call(name))(args)
    t = torch.empty(n, dtype=torch.uint8, device=device) if n else None
    return t, _ptr(t), n


_CONV = struct.Struct("13q")


def _conv_args(x, weight, bias, initial_state, lengths, silu):
    torch, kind = _first(x, 3)
    f32, dev, shape = torch.float32, x.device, x.shape
    B, L, D = shape
    if weight.dim() != 2 or weight.shape[1] < 1:
        raise ValueError("weight must be [D, W]")
    W = weight.shape[1]
    if W > 8:
        raise ValueError("filters of more than 8 tokens are not supported")
    x = _tokens("x", x, shape, x)
    weight = _whole("weight", weight, (D, W), f32, dev)
    bias = _whole("bias", bias, (D,), f32, dev)
    initial_state = _whole("initial_state", initial_state, (B, W - 1, D), x.dtype, dev)
    lengths = _whole("lengths", lengths, (B,), torch.int32, dev)
    sb, st, _ = x.stride()
    args = _CONV.pack(kind, B, L, D, W, 1 if silu else 0, sb, st, x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(initial_state), _ptr(lengths))
    return torch, args, W, (x, weight, bias, initial_state, lengths)


def sig_conv_forward(x, weight, bias=None, initial_state=None, lengths=None, silu=True, return_state=False):
    """Causal depthwise convolution y_t = f(bias + sum_k weight[:, k] x_{t-W+1+k}), f(s) = s sigmoid(s) or (silu=False) s.

    x [B, L, D]; weight float32 [D, W], W <= 8; bias float32 [D]; initial_state [B, W-1, D] of x's type: the tokens before the first, oldest
    first (default zeros); lengths int32 [B]: tokens from there on are not read and give zeros.  Returns y [B, L, D], or with
    return_state (y, state): the last W-1 tokens of every stream, for sig_conv_step or the next prompt's initial_state."""
    torch, args, W, kept = _conv_args(x, weight, bias, initial_state, lengths, silu)
    B, L, D = x.shape
    y = torch.empty((B, L, D), dtype=x.dtype, device=x.device)
    state = torch.empty((B, W - 1, D), dtype=x.dtype, device=x.device) if return_state else None
    _enqueue(x.device, "sig_conv_forward", args, y.data_ptr(), _ptr(state))
    return (y, state) if return_state else y


def sig_conv_backward(x, weight, grad_out, bias=None, initial_state=None, lengths=None, silu=True, grad_final_state=None):
    """Gradient of sig_conv_forward: (grad_x, grad_weight, grad_bias, grad_initial_state), None for those whose input is None.
    grad_out [B, L, D] and grad_final_state [B, W-1, D] are of x's type."""
    torch, args, W, kept = _conv_args(x, weight, bias, initial_state, lengths, silu)
    B, L, D = x.shape
    dev = x.device
    grad_out = _tokens("grad_out", grad_out, x.shape, x)
    grad_final_state = _whole("grad_final_state", grad_final_state, (B, W - 1, D), x.dtype, dev)
    gx = torch.empty((B, L, D), dtype=x.dtype, device=dev)
    gw = torch.empty((D, W), dtype=torch.float32, device=dev)
    gb = torch.empty(D, dtype=torch.float32, device=dev) if bias is not None else None
    gi = torch.empty((B, W - 1, D), dtype=x.dtype, device=dev) if initial_state is not None else None
    keep, wptr, nbytes = _scratch(torch, "sig_conv_backward_workspace_bytes", args, dev)
    sb, st, _ = grad_out.stride()
    _enqueue(dev, "sig_conv_backward", args, grad_out.data_ptr(), sb, st, _ptr(grad_final_state), gx.data_ptr(), gw.data_ptr(), _ptr(gb),
             _ptr(gi), wptr, nbytes)
    return gx, gw, gb, gi


def sig_conv_step(x, state, weight, bias=None, silu=True):
    """One token of every stream: x [B, D], state [B, W-1, D] of x's type, shifted by it in place.  Returns y [B, D]."""
    torch, kind = _first(x, 2)
    B, D = x.shape
    dev = x.device
    if weight.dim() != 2 or not 1 <= weight.shape[1] <= 8:
        raise ValueError("weight must be [D, W] with W <= 8")
    W = weight.shape[1]
    x = _tokens("x", x, x.shape, x)
    weight = _whole("weight", weight, (D, W), torch.float32, dev)
    bias = _whole("bias", bias, (D,), torch.float32, dev)
    _in_place("state", state, (B, W - 1, D), x.dtype, dev)
    y = torch.empty((B, D), dtype=x.dtype, device=dev)
    args = _CONV.pack(kind, B, 1, D, W, 1 if silu else 0, x.stride(0), 0, x.data_ptr(), weight.data_ptr(), _ptr(bias), 0, 0)
    _enqueue(dev, "sig_conv_step", args, state.data_ptr(), y.data_ptr())
    return y


_SCAN = struct.Struct("29q")
_SCAN_GRADS = struct.Struct("13q")


def _groups(name, t, lead, like):
    """b or c: [..., N] (one group) or [..., G, N]; (tensor with the group axis, G, N)."""
    if t.dim() == len(lead) + 1:
        t = t.unsqueeze(-2)
    if t.dim() != len(lead) + 2:
        raise ValueError(f"{name} must have the shape of the tokens before its axes [groups, states] or [states]")
    return _tokens(name, t, (*lead, *t.shape[-2:]), like)


def _scan_args(x, dt, A, b, c, skip, gate, dt_bias, softplus, initial_state, lengths, dims):
    torch, kind = _first(x, dims)
    f32, dev, shape = torch.float32, x.device, x.shape
    lead, D = shape[:-1], shape[-1]
    x = _tokens("x", x, shape, x)
    dt = _tokens("dt", dt, shape, x)
    b, c = _groups("b", b, lead, x), _groups("c", c, lead, x)
    G, N = b.shape[-2:]
    if c.shape != b.shape or G < 1 or D % G:
        raise ValueError("b and c must have the same groups and states, and the groups divide the channels")
    if not 1 <= N <= 64:
        raise ValueError("1 to 64 states are supported")
    if gate is not None:
        gate = _tokens("gate", gate, shape, x)
    A = _whole("A", A, (D, N), f32, dev)
    if A is None:
        raise ValueError("A is missing")
    skip, dt_bias = _whole("skip", skip, (D,), f32, dev), _whole("dt_bias", dt_bias, (D,), f32, dev)
    if dims == 3:
        B, L, _ = shape
        initial_state = _whole("initial_state", initial_state, (B, D, N), f32, dev)
        lengths = _whole("lengths", lengths, (B,), torch.int32, dev)
        (xb, xt, _), (tb, tt, _), (zb, zt, _) = x.stride(), dt.stride(), (0, 0, 0) if gate is None else gate.stride()
        (bb, bt, bg, _), (cb, ct, cg, _) = b.stride(), c.stride()
    else:
        B, L = shape[0], 1
        xb, xt, tb, tt, zb, zt = x.stride(0), 0, dt.stride(0), 0, 0 if gate is None else gate.stride(0), 0
        (bb, bg, _), (cb, cg, _), bt, ct = b.stride(), c.stride(), 0, 0
    args = _SCAN.pack(kind, B, L, D, G, N, 1 if softplus else 0, xb, xt, tb, tt, zb, zt, bb, bt, bg, cb, ct, cg, x.data_ptr(), dt.data_ptr(),
                      _ptr(gate), b.data_ptr(), c.data_ptr(), A.data_ptr(), _ptr(skip), _ptr(dt_bias), _ptr(initial_state), _ptr(lengths))
    return torch, args, G, N, (x, dt, A, b, c, skip, gate, dt_bias, initial_state, lengths)


def sig_scan_forward(x, dt, A, b, c, skip=None, gate=None, dt_bias=None, softplus=True, initial_state=None, lengths=None, checkpoint=False):
    """Selective state space scan: h_t = exp(delta_t A) h_{t-1} + delta_t x_t b_t, y_t = (sum_n c_t h_t + skip x_t) silu(gate_t), with
    delta_t = softplus(dt_t + dt_bias) (softplus=False: the sum itself).

    x, dt, gate [B, L, D]; b, c [B, L, G, N] or [B, L, N]: channel d uses group d // (D // G); A float32 [D, N]; skip, dt_bias float32 [D];
    initial_state float32 [B, D, N] (default zeros); lengths int32 [B]: tokens from there on are not read, give zeros and leave the
    state.  Returns (y [B, L, D], final state float32 [B, D, N]); with checkpoint=True a third tensor for sig_scan_backward."""
    torch, args, G, N, kept = _scan_args(x, dt, A, b, c, skip, gate, dt_bias, softplus, initial_state, lengths, 3)
    B, L, D = x.shape
    dev = x.device
    y = torch.empty((B, L, D), dtype=x.dtype, device=dev)
    state = torch.empty((B, D, N), dtype=torch.float32, device=dev)
    ck, cptr, cbytes = _scratch(torch, "sig_scan_checkpoint_bytes", args, dev) if checkpoint else (None, 0, 0)
    keep, wptr, nbytes = _scratch(torch, "sig_scan_forward_workspace_bytes", args, dev)
    _enqueue(dev, "sig_scan_forward", args, y.data_ptr(), state.data_ptr(), cptr, cbytes, wptr, nbytes)
    if not checkpoint:
        return y, state
    return y, state, ck if ck is not None else torch.empty(0, dtype=torch.uint8, device=dev)


def sig_scan_backward(x, dt, A, b, c, grad_out, checkpoint, skip=None, gate=None, dt_bias=None, softplus=True, initial_state=None, lengths=None,
                      grad_final_state=None):
    """Gradient of sig_scan_forward, whose `checkpoint` it reads: a dict of the gradients "x", "dt", "A", "B", "C", "skip", "gate", "dt_bias"
    and "initial_state", None for those whose input is None.  grad_out [B, L, D] of x's type, grad_final_state float32 [B, D, N] or None."""
    torch, args, G, N, kept = _scan_args(x, dt, A, b, c, skip, gate, dt_bias, softplus, initial_state, lengths, 3)
    B, L, D = x.shape
    t, dev, f32 = x.dtype, x.device, torch.float32
    grad_out = _tokens("grad_out", grad_out, x.shape, x)
    grad_final_state = _whole("grad_final_state", grad_final_state, (B, D, N), f32, dev)
    if not checkpoint.is_cuda or checkpoint.device != dev or not checkpoint.is_contiguous():
        raise ValueError("checkpoint must be the tensor that sig_scan_forward returned")
    gx, gdt = torch.empty((B, L, D), dtype=t, device=dev), torch.empty((B, L, D), dtype=t, device=dev)
    gz = torch.empty((B, L, D), dtype=t, device=dev) if gate is not None else None
    gb, gc = torch.empty((B, L, G, N), dtype=t, device=dev), torch.empty((B, L, G, N), dtype=t, device=dev)
    gA = torch.empty((D, N), dtype=f32, device=dev)
    gskip = torch.empty(D, dtype=f32, device=dev) if skip is not None else None
    gbias = torch.empty(D, dtype=f32, device=dev) if dt_bias is not None else None
    gi = torch.empty((B, D, N), dtype=f32, device=dev) if initial_state is not None else None
    sb, st, _ = grad_out.stride()
    grads = _SCAN_GRADS.pack(sb, st, grad_out.data_ptr(), _ptr(grad_final_state), gx.data_ptr(), gdt.data_ptr(), _ptr(gz), gb.data_ptr(),
                             gc.data_ptr(), gA.data_ptr(), _ptr(gskip), _ptr(gbias), _ptr(gi))
    keep, wptr, nbytes = _scratch(torch, "sig_scan_backward_workspace_bytes", args, dev)
    _enqueue(dev, "sig_scan_backward", args, grads, checkpoint.data_ptr(), checkpoint.numel() * checkpoint.element_size(), wptr, nbytes)
    if b.dim() == 3:
        gb, gc = gb.view(B, L, N), gc.view(B, L, N)
    return {"x": gx, "dt": gdt, "A": gA, "B": gb, "C": gc, "skip": gskip, "gate": gz, "dt_bias": gbias, "initial_state": gi}


def sig_scan_step(x, dt, A, b, c, state, skip=None, gate=None, dt_bias=None, softplus=True):
    """One token of every stream: x, dt, gate [B, D], b, c [B, G, N] or [B, N]; state float32 [B, D, N] is updated in place.  Returns y [B, D]."""
    torch, args, G, N, kept = _scan_args(x, dt, A, b, c, skip, gate, dt_bias, softplus, None, None, 2)
    B, D = x.shape
    _in_place("state", state, (B, D, N), torch.float32, x.device)
    y = torch.empty((B, D), dtype=x.dtype, device=x.device)
    _enqueue(x.device, "sig_scan_step", args, state.data_ptr(), y.data_ptr())
    return y


def sig_grad_clip(grads, max_norm, out=None):
    """Scales the tensors `grads` (float32 or bfloat16, one device) in place by min(1, max_norm / (norm + 1e-6)), norm their global 2-norm, or
    writes the products into the tensors `out` (of the same sizes, either type).  Returns norm, a float32 tensor of no axes on the
    device.  Tensors may have any order of axes as long as they fill their memory; those of `out` have that of their input."""
    torch = _t()
    f32, b16 = torch.float32, torch.bfloat16
    grads = list(grads)
    outs = grads if out is None else list(out)
    if len(outs) != len(grads):
        raise ValueError("out must have a tensor for each of grads")
    if not max_norm >= 0:
        raise ValueError("max_norm must not be negative")
    dev = grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
    if dev.type != "cuda":
        raise ValueError("grads must be CUDA tensors")
    for g, o in zip(grads, outs):
        if g.device != dev or o.device != dev or g.dtype not in (f32, b16) or o.dtype not in (f32, b16):
            raise ValueError("grads and out must be float32 or bfloat16 tensors on one device")
        if g.shape != o.shape or not (g.is_contiguous() and o.is_contiguous()) and (
                g.stride() != o.stride() or not torch.ops.aten.is_non_overlapping_and_dense(g)):
            raise ValueError("every tensor must fill its memory, and out must have the shape and the order of axes of grads")
    n = len(grads)
    tab = array.array("q", [g.data_ptr() for g in grads])
    tab.extend(o.data_ptr() for o in outs)
    tab.extend(g.numel() for g in grads)
    tab.extend(int(g.dtype is b16) for g in grads)
    tab.extend(int(o.dtype is b16) for o in outs)
    at, _ = tab.buffer_info()
    norm = torch.empty((), dtype=f32, device=dev)
    nbytes = (_calls.get("sig_grad_clip_workspace_bytes") or _call("sig_grad_clip_workspace_bytes"))(n, at + 16 * n)
    keep = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _enqueue(dev, "sig_grad_clip", n, at, at + 8 * n, at + 16 * n, at + 24 * n, at + 32 * n, float(max_norm), norm.data_ptr(), _ptr(keep), nbytes)
    return norm
