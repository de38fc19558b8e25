"""Plain 64-bit implementations of the sequence operators on the CPU, one token of one stream after the other; gradients by torch's reverse
mode over them.  Shares no code with the package."""
import torch


def inputs(kind, B, L, D, G=1, N=16, W=4, dtype=torch.float32, carry=True, full=True, lengths=None, seed=0):
    """Seeded CPU inputs of the given type: values of x, dt etc. are exact in it, parameters in float32."""
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float32)                       # noqa: E731
    tok = lambda *s: n(*s).to(dtype)                                                       # noqa: E731
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    if kind == "conv":
        return dict(x=tok(B, L, D), weight=n(D, W) / W ** 0.5, bias=0.1 * n(D) if full else None, initial_state=tok(B, W - 1, D) if carry else None,
                    lengths=lens, grad_out=tok(B, L, D), grad_final_state=tok(B, W - 1, D) if carry else None)
    dt = 0.5 * n(B, L, D) - 2.0
    return dict(x=tok(B, L, D), dt=(dt if full else torch.exp(dt)).to(dtype), A=-torch.exp(0.5 * n(D, N)) * torch.arange(1, N + 1), b=tok(B, L, G, N),
                c=tok(B, L, G, N), skip=n(D) if full else None, gate=tok(B, L, D) if full else None, dt_bias=0.3 * n(D) if full else None,
                initial_state=n(B, D, N) if carry else None, lengths=lens, grad_out=tok(B, L, D), grad_final_state=n(B, D, N) if carry else None)


def _len(lengths, b, L):
    return L if lengths is None else min(max(int(lengths[b]), 0), L)


def conv(x, weight, bias=None, initial_state=None, lengths=None, silu=True):
    """(y, final state) in the inputs' own precision."""
    B, L, D = x.shape
    W = weight.shape[1]
    ys, states = [], []
    for b in range(B):
        n = _len(lengths, b, L)
        before = x.new_zeros(W - 1, D) if initial_state is None else initial_state[b]
        seen = torch.cat([before, x[b, :n]])
        rows = []
        for t in range(n):
            s = (seen[t:t + W] * weight.t()).sum(0)
            s = s if bias is None else s + bias
            rows.append(s / (1 + torch.exp(-s)) if silu else s)
        ys.append(torch.cat([torch.stack(rows) if rows else x.new_zeros(0, D), x.new_zeros(L - n, D)]))
        states.append(seen[n:])
    return torch.stack(ys), torch.stack(states)


def scan(x, dt, A, b, c, skip=None, gate=None, dt_bias=None, softplus=True, initial_state=None, lengths=None):
    B, L, D = x.shape
    N, G = A.shape[1], b.shape[2]
    ys, states = [], []
    for i in range(B):
        n = _len(lengths, i, L)
        h = x.new_zeros(D, N) if initial_state is None else initial_state[i]
        rows = []
        for t in range(n):
            d = dt[i, t] if dt_bias is None else dt[i, t] + dt_bias
            d = torch.logaddexp(d, torch.zeros_like(d)) if softplus else d
            wide = lambda v: v.repeat_interleave(D // G, 0)                                # noqa: E731
            h = torch.exp(d[:, None] * A) * h + (d * x[i, t])[:, None] * wide(b[i, t])
            s = (wide(c[i, t]) * h).sum(1)
            s = s if skip is None else s + skip * x[i, t]
            rows.append(s if gate is None else s * gate[i, t] / (1 + torch.exp(-gate[i, t])))
        ys.append(torch.cat([torch.stack(rows) if rows else x.new_zeros(0, D), x.new_zeros(L - n, D)]))
        states.append(h)
    return torch.stack(ys), torch.stack(states)


def with_gradients(f, given, grad_out, grad_final_state, **more):
    """f's outputs and the gradients of <y, grad_out> + <state, grad_final_state> in float64: (y, state, {name: gradient})."""
    wide = {k: v.detach().double().requires_grad_() if v is not None and v.is_floating_point() else v for k, v in given.items()}
    y, state = f(**wide, **more)
    B, L = y.shape[:2]
    lengths = given.get("lengths")
    live = torch.tensor([[t < _len(lengths, b, L) for t in range(L)] for b in range(B)]).reshape(B, L, 1)
    loss = (torch.where(live, y * grad_out.double(), 0.0)).sum()
    if grad_final_state is not None:
        loss = loss + (state * grad_final_state.double()).sum()
    names = [k for k, v in wide.items() if v is not None and v.is_floating_point()]
    got = torch.autograd.grad(loss, [wide[k] for k in names], allow_unused=True) if loss.requires_grad else [None] * len(names)
    return y.detach(), state.detach(), {k: torch.zeros_like(wide[k]) if v is None else v for k, v in zip(names, got)}
