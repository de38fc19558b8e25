"""A small sequence model over signature tokens: trained on whole streams, then run token by token.

Every path is read through a sliding window; the signature of a window is a token.  A layer projects the tokens, mixes them over time with the
short causal convolution and the selective scan, and a read-out estimates, after every window, the path's quadratic variation so far.
Training takes the gradient through all of it back to the path, bounded by the global norm; afterwards the same parameters run as a
stream: one window at a time, with the states of the convolution and the scan carried along.

    python examples/stream_model.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2602_24066_amd as sig  # noqa: E402


class Signatures(torch.autograd.Function):
    """Signatures over windows of a path: [B, n, d] -> [B, K, |W|]."""

    @staticmethod
    def forward(ctx, path, words, windows):
        tokens = sig.sig_forward_windows(words, path, windows)
        ctx.save_for_backward(path, tokens)
        ctx.rest = words, windows
        return tokens

    @staticmethod
    def backward(ctx, grad):
        path, tokens = ctx.saved_tensors
        words, windows = ctx.rest
        return sig.sig_backward_windows(words, path, windows, tokens, grad.contiguous()), None, None


class Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        ctx.save_for_backward(x, weight, bias)
        return sig.sig_conv_forward(x, weight, bias)

    @staticmethod
    def backward(ctx, grad):
        x, weight, bias = ctx.saved_tensors
        return sig.sig_conv_backward(x, weight, grad, bias)[:3]


class Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, A, b, c, skip, gate, dt_bias):
        y, _, kept = sig.sig_scan_forward(x, dt, A, b, c, skip, gate, dt_bias, checkpoint=True)
        ctx.save_for_backward(x, dt, A, b, c, skip, gate, dt_bias, kept)
        return y

    @staticmethod
    def backward(ctx, grad):
        x, dt, A, b, c, skip, gate, dt_bias, kept = ctx.saved_tensors
        g = sig.sig_scan_backward(x, dt, A, b, c, grad, kept, skip, gate, dt_bias)
        return tuple(g[k] for k in ("x", "dt", "A", "B", "C", "skip", "gate", "dt_bias"))


def parameters(n_features, channels, states, width, rank, seed):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g) / s[-1] ** 0.5                             # noqa: E731
    p = {"embed": n(2 * channels, n_features), "conv": n(channels, width), "conv_bias": torch.zeros(channels),
         "select": n(rank + 2 * states, channels), "step": n(channels, rank), "step_bias": torch.full((channels,), -3.0),
         "log_decay": torch.arange(1.0, states + 1).log().repeat(channels, 1), "skip": torch.ones(channels), "read": n(1, channels)}
    return {k: v.cuda().requires_grad_() for k, v in p.items()}


def whole(p, tokens):
    """tokens [B, K, n_features] -> estimates [B, K]"""
    rank, states = p["step"].shape[1], p["log_decay"].shape[1]
    x, gate = (tokens @ p["embed"].t()).chunk(2, -1)
    u = Conv.apply(x, p["conv"], p["conv_bias"])
    low, b, c = (u @ p["select"].t()).split([rank, states, states], -1)
    y = Scan.apply(u, low @ p["step"].t(), -p["log_decay"].exp(), b, c, p["skip"], gate, p["step_bias"])
    return (y @ p["read"].t())[..., 0]


class Stream:
    """The same model one token at a time."""

    def __init__(self, p, batch):
        self.p = {k: v.detach() for k, v in p.items()}
        self.A = -self.p["log_decay"].exp()
        self.tail = torch.zeros(batch, self.p["conv"].shape[1] - 1, self.p["conv"].shape[0], device="cuda")
        self.state = torch.zeros(batch, *self.A.shape, device="cuda")

    def __call__(self, token):
        p = self.p
        rank, states = p["step"].shape[1], p["log_decay"].shape[1]
        x, gate = (token @ p["embed"].t()).chunk(2, -1)
        u = sig.sig_conv_step(x, self.tail, p["conv"], p["conv_bias"])
        low, b, c = (u @ p["select"].t()).split([rank, states, states], -1)
        y = sig.sig_scan_step(u, low @ p["step"].t(), self.A, b, c, self.state, p["skip"], gate, p["step_bias"])
        return (y @ p["read"].t())[..., 0]


def run(batch=32, segments=512, d=2, depth=4, window=32, hop=8, channels=64, states=16, steps=60, seed=0, log=print):
    """Trains and streams; returns the losses and the largest difference between the streamed and the whole pass' estimates."""
    rnd = torch.Generator().manual_seed(seed)
    scale = 0.5 + torch.rand(batch, 1, 1, generator=rnd)
    moves = torch.randn(batch, segments, d, generator=rnd) * scale / window ** 0.5
    path = torch.cat([torch.zeros(batch, 1, d), moves.cumsum(1)], 1).cuda()
    windows = [(e - window, e) for e in range(window, segments + 1, hop)]
    target = moves.square().sum(-1).cumsum(1)[:, window - 1::hop].cuda() * (window / segments)
    words = sig.sig_wordset_build_truncated(d, depth).upload("cuda")
    p = parameters(words.size, channels, states, 4, max(1, channels // 16), seed)
    warp = torch.zeros_like(path).requires_grad_()                                         # a correction of the path, learned with the rest
    learned = [*p.values(), warp]
    optimizer = torch.optim.Adam(learned, lr=0.01)
    losses = []
    for k in range(steps):
        tokens = Signatures.apply(path + warp, words, windows)
        loss = (whole(p, tokens) - target).square().mean()
        optimizer.zero_grad()
        loss.backward()
        norm = sig.sig_grad_clip([v.grad for v in learned], 1.0)
        optimizer.step()
        losses.append(float(loss.detach()))
        if k % 10 == 0:
            log(f"step {k:3d}  loss {losses[-1]:.4f}  gradient norm before clipping {float(norm):.3f}")
    with torch.no_grad():
        tokens = sig.sig_forward_windows(words, (path + warp).detach(), windows)
        at_once, stream = whole(p, tokens), Stream(p, batch)
        one_by_one = torch.stack([stream(tokens[:, k]) for k in range(tokens.shape[1])], 1)
    off = float((one_by_one - at_once).abs().max() / at_once.abs().max())
    log(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; streamed estimates differ from the whole pass by {off:.1e} of the largest")
    return losses, off


if __name__ == "__main__":
    run()
