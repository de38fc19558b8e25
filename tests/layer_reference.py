"""Plain 64-bit implementations of the operators of a layer on the CPU; gradients by torch's reverse mode over them.  Shares no code with the package."""
import math

import torch


def norm(total, weight, eps=1e-6):
    return total / torch.sqrt((total * total).mean(-1, keepdim=True) + eps) * weight


def act(z, name):
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    return z


def slope(z, name):
    z = z.detach().clone().requires_grad_()
    return torch.autograd.grad(act(z, name).sum(), z)[0]


def e4m3(v):
    """The nearest value of e4m3 (ties to even), from its definition: 3 fraction bits, exponents from -6, denormals below, largest value 448."""
    a = v.abs()
    e = torch.floor(torch.log2(torch.where(a > 0, a, 1.0))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.sign(v) * torch.round(a / step) * step


def _len(lengths, b, L):
    return L if lengths is None else min(max(int(lengths[b]), 0), L)


def gated(x, decay_gate, input_gate, log_rate, initial_state=None, lengths=None):
    """(y, final state), one token of one stream after the other."""
    B, L, D = x.shape
    ys, states = [], []
    for b in range(B):
        n = _len(lengths, b, L)
        h = x.new_zeros(D) if initial_state is None else initial_state[b]
        rows = []
        for t in range(n):
            u = torch.exp(log_rate) / (1 + torch.exp(-decay_gate[b, t]))
            h = torch.exp(-u) * h + torch.sqrt(-torch.expm1(-2 * u)) * x[b, t] / (1 + torch.exp(-input_gate[b, t]))
            rows.append(h)
        ys.append(torch.cat([torch.stack(rows) if rows else x.new_zeros(0, D), x.new_zeros(L - n, D)]))
        states.append(h)
    return torch.stack(ys), torch.stack(states)


def gated_inputs(B, L, D, dtype=torch.float32, carry=True, lengths=None, seed=0, rate=0.1):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)                                             # noqa: E731
    return dict(x=n(B, L, D).to(dtype), decay_gate=n(B, L, D).to(dtype), input_gate=n(B, L, D).to(dtype), log_rate=math.log(rate) + n(D),
                initial_state=n(B, D) if carry else None, lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32))
