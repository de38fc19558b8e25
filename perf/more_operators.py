"""Timed cases of the operators that, with the short convolution, make up a layer of a model over signature tokens.

A layer normalises the stream of tokens, projects it, mixes it over time and projects it back onto the stream.  Kinds of case:

  norm        root-mean-square norm of the sum of tokens and residual, the sum returned too     norm_train    the same with its gradient
  norm8       the same with an output in 8 bits (e4m3) and a scale a token
  linear      matrix product with bias, activation and residual                                  linear_train  the same with its gradient
  linear8     tokens to 8 bits with a scale each, their product with weights held in 8 bits
  gated       gated linear recurrence over a prompt, final state included                        gated_train   forward with its gradient
  gated_step  one new token of every stream, the state updated in place

`own` = False computes the plain form: elementary torch operations in float32, rounded once at the end.  `own` = True makes the calls
of this package.  Tokens are channels last, [batch, time, channels] (time = 1: [batch, channels]); `ragged` gives every stream a length of
its own (0 among them).
"""
import math

import torch

own = False


def listed():
    return [
        # a batch of streams that each get one new token: the smallest call
        dict(name="norm_bf16_64x1024", kind="norm", dtype="bf16", batch=64, time=1, chans=1024, residual=1),
        # prompts of a large batch, for a projection in 8 bits
        dict(name="norm8_bf16_8x4096x2048", kind="norm8", dtype="bf16", batch=8, time=4096, chans=2048, residual=1),
        # a training step at odd sizes
        dict(name="norm_train_f32_37x301x333", kind="norm_train", dtype="f32", batch=37, time=301, chans=333, residual=1),
        # one new token of every stream through a layer's last projection, onto the residual
        dict(name="linear_bf16_64x2048_1024", kind="linear", dtype="bf16", batch=64, time=1, chans=2048, outs=1024, bias=1, residual=1, act="none"),
        # signatures of depth 6 over four letters to the model's channels: long odd rows, float32, a number of tokens that fills no tile
        dict(name="linear_f32_7x301x5460_1024", kind="linear", dtype="f32", batch=7, time=301, chans=5460, outs=1024, bias=1, residual=0, act="none"),
        # prompts of a large batch through a layer's first projection
        dict(name="linear_bf16_8x2048x1024_4096", kind="linear", dtype="bf16", batch=8, time=2048, chans=1024, outs=4096, bias=1, residual=0, act="silu"),
        # prompts of a large batch served in 8 bits
        dict(name="linear8_bf16_8x2048x2048_2048", kind="linear8", dtype="bf16", batch=8, time=2048, chans=2048, outs=2048, bias=0, residual=1, act="none"),
        # a training step of a large batch
        dict(name="linear_train_bf16_8x2048x1024_4096", kind="linear_train", dtype="bf16", batch=8, time=2048, chans=1024, outs=4096, bias=1, residual=0, act="gelu"),
        # one long stream: few rows, all the work along time
        dict(name="gated_bf16_1x16384x1024", kind="gated", dtype="bf16", batch=1, time=16384, chans=1024, carry=1, ragged=0),
        # a training step of a large batch
        dict(name="gated_train_bf16_8x2048x2048", kind="gated_train", dtype="bf16", batch=8, time=2048, chans=2048, carry=0, ragged=0),
        # a training step at odd sizes: carried state, streams of different length
        dict(name="gated_train_f32_7x301x277", kind="gated_train", dtype="f32", batch=7, time=301, chans=277, carry=1, ragged=1),
        # a batch of streams that each get one new token
        dict(name="gated_step_bf16_64x2048", kind="gated_step", dtype="bf16", batch=64, time=1, chans=2048, carry=1, ragged=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _chans(rng, most=4096):
    """Channels of a model (a multiple of 64), the size of a signature, or anything."""
    how = rng.randrange(5)
    return 64 * _log_int(rng, 1, most // 64) if how < 2 else rng.choice([30, 258, 340, 1554, 5460]) if how == 2 else _log_int(rng, 16, most)


def draw(rng):
    kind = rng.choice(["norm", "norm8", "norm_train", "linear", "linear", "linear8", "linear_train", "linear_train", "gated", "gated", "gated_train", "gated_train",
                       "gated_step"])
    f32 = kind not in ("linear8",) and rng.randrange(2)
    c = dict(kind=kind, dtype="f32" if f32 else "bf16", batch=_log_int(rng, 1, 128), time=1)
    c["chans"] = _chans(rng)
    prompt = kind != "gated_step" and rng.randrange(4) > 0
    if prompt:
        c["time"] = _log_int(rng, 2, 16384)
    if kind.startswith("linear"):
        c["outs"] = rng.choice([_chans(rng), 64 * _log_int(rng, 1, 64)])
        c |= dict(bias=rng.randrange(2), residual=rng.randrange(2), act=rng.choice(["none", "silu", "gelu"]))
        most = 16384 * 1024 * 4096 // (8 if f32 else 1) // (c["chans"] * c["outs"])
        most = min(most, 8 * 2048 * 2048 // max(c["chans"], c["outs"]))
    elif kind.startswith("norm"):
        c["residual"] = rng.randrange(2)
        most = 8 * 2048 * 2048 // (2 if f32 else 1) // c["chans"]
    else:
        c |= dict(carry=1 if kind == "gated_step" else rng.randrange(2), ragged=rng.randrange(2) if c["time"] > 1 else 0)
        most = 8 * 2048 * 2048 // (4 if f32 else 2) // c["chans"]
    c["batch"] = max(1, min(c["batch"], most // c["time"]))
    c["time"] = max(1, min(c["time"], most // c["batch"]))
    if c["time"] == 1 and "ragged" in c:
        c["ragged"] = 0
    return c


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """Lengths spread evenly over 0 .. time, dealt out in an order that is not sorted; one stream: two thirds of it."""
    n, t = case["batch"], case["time"]
    if not case.get("ragged"):
        return [t] * n
    if n == 1:
        return [t - t // 3]
    return [t * (b * 5 % n if n % 5 else (b * 3 % n if n % 3 else b)) // (n - 1) for b in range(n)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    uniform = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    s, t, D = dict(case), _type(case), case["chans"]
    rows = (case["batch"], case["time"]) if case["time"] > 1 or case["kind"] in ("gated", "gated_train") else (case["batch"],)
    if case["kind"].startswith("norm"):
        s["x"], s["residual"] = normal(*rows, D).to(t), (2 * normal(*rows, D)).to(t) if case["residual"] else None
        s["weight"] = 1 + 0.1 * normal(D)
        s["grad_out"], s["grad_sum"] = (normal(*rows, D).to(t), normal(*rows, D).to(t)) if case["kind"] == "norm_train" else (None, None)
        return s
    if case["kind"].startswith("linear"):
        N = case["outs"]
        s["x"], s["weight"] = normal(*rows, D).to(t), (normal(N, D) / math.sqrt(D)).to(t)
        s["bias"] = (0.1 * normal(N)).to(t) if case["bias"] else None
        s["residual"] = normal(*rows, N).to(t) if case["residual"] else None
        s["grad_out"] = normal(*rows, N).to(t) if case["kind"] == "linear_train" else None
        if case["kind"] == "linear8":                                       # weights are held in 8 bits, a scale for each output
            w = s["weight"].float()
            s["weight_scale"] = w.abs().amax(1) / 448
            s["weight"] = (w / s["weight_scale"][:, None]).to(torch.float8_e4m3fn)
        return s
    wide = normal(*rows, 2 * D).to(t)                                       # one projection gives both gates
    s["x"], s["decay_gate"], s["input_gate"] = normal(*rows, D).to(t), wide[..., :D], wide[..., D:]
    s["log_rate"] = torch.log(-torch.log(0.9 + 0.099 * uniform(D)) * 8)     # decays between 0.9 and 0.999 at an eighth of the rate
    s["state"] = normal(case["batch"], D) if case["carry"] else None
    s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    if case["kind"] == "gated_train":
        s["grad_out"] = normal(*rows, D).to(t)
        s["grad_state"] = normal(case["batch"], D) if case["carry"] else None
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2602_24066_amd as sig
    kind = s["kind"]
    if kind == "norm":
        y, total = sig.sig_norm_forward(s["x"], s["weight"], s["residual"])
        return {"y": y, "sum": total}
    if kind == "norm8":
        y, scale, total = sig.sig_norm_forward(s["x"], s["weight"], s["residual"], quantize=True)
        return {"y": y, "scale": scale, "sum": total}
    if kind == "norm_train":
        y, total = sig.sig_norm_forward(s["x"], s["weight"], s["residual"])
        gx, gw = sig.sig_norm_backward(total, s["weight"], s["grad_out"], s["grad_sum"])
        return {"y": y, "sum": total, "grad_x": gx, "grad_weight": gw}
    act = None if s.get("act") == "none" else s.get("act")
    if kind == "linear":
        return {"y": sig.sig_linear_forward(s["x"], s["weight"], s["bias"], s["residual"], activation=act)}
    if kind == "linear8":
        x, scale = sig.sig_quantize(s["x"])
        y = sig.sig_linear_forward(x, s["weight"], s["bias"], s["residual"], activation=act, x_scale=scale, weight_scale=s["weight_scale"])
        return {"y": y, "x": x, "scale": scale}
    if kind == "linear_train":
        y, pre = sig.sig_linear_forward(s["x"], s["weight"], s["bias"], s["residual"], activation=act, keep=True)
        gx, gw, gb = sig.sig_linear_backward(s["x"], s["weight"], s["grad_out"], activation=act, pre=pre, bias=s["bias"] is not None)
        return {"y": y, "grad_x": gx, "grad_weight": gw} | ({} if gb is None else {"grad_bias": gb})
    gates = s["decay_gate"], s["input_gate"], s["log_rate"]
    if kind == "gated_step":
        return {"y": sig.sig_gated_scan_step(s["x"], *gates, s["state"]), "state": s["state"]}
    more = dict(initial_state=s["state"], lengths=s["lengths"])
    if kind == "gated":
        y, state = sig.sig_gated_scan_forward(s["x"], *gates, **more)
        return {"y": y, "state": state}
    y, state, kept = sig.sig_gated_scan_forward(s["x"], *gates, checkpoint=True, **more)
    grads = sig.sig_gated_scan_backward(s["x"], *gates, s["grad_out"], kept, grad_final_state=s["grad_state"], **more)
    return {"y": y, "state": state, "grads": {k: v for k, v in grads.items() if v is not None}}


def _plain(s):
    kind = s["kind"]
    return _plain_norm(s) if kind.startswith("norm") else _plain_linear(s) if kind.startswith("linear") else _plain_gated(s)


def _plain_norm(s):
    t, w = s["x"].dtype, s["weight"]
    total = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(t)      # the stream as it is kept
    r = total.float()
    size = torch.rsqrt(r.square().mean(-1, keepdim=True) + 1e-6)
    n = r * size
    y = n * w
    if s["kind"] == "norm8":
        q, scale = _eight(y)
        return {"y": q, "scale": scale, "sum": total}
    out = {"y": y.to(t), "sum": total}
    if s["kind"] == "norm_train":
        gy = s["grad_out"].float()
        h = gy * w
        out["grad_x"] = (size * (h - n * (h * n).mean(-1, keepdim=True)) + s["grad_sum"].float()).to(t)
        out["grad_weight"] = (gy * n).flatten(0, -2).sum(0)
    return out


def _eight(v):
    """Rows in e4m3, the largest of each at its largest value, and what they are to be multiplied by."""
    scale = v.abs().amax(-1) / 448
    return (v / torch.where(scale > 0, scale, 1.0)[..., None]).to(torch.float8_e4m3fn), scale


def _act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5))) if act == "gelu" else z


def _slope(z, act):
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))


def _plain_linear(s):
    t, x, w = s["x"].dtype, s["x"].float(), s["weight"].float()
    out = {}
    if s["kind"] == "linear8":
        q, scale = _eight(x)
        out = {"x": q, "scale": scale}
        z = (q.float() @ w.t()) * scale[..., None] * s["weight_scale"]
    else:
        z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out["y"] = y.to(t)
    if s["kind"] == "linear_train":
        g = s["grad_out"].float()
        if s["act"] != "none":
            g = g * _slope(z, s["act"])
        out["grad_x"] = (g @ w).to(t)
        g = g.flatten(0, -2)
        out["grad_weight"] = (g.t() @ x.flatten(0, -2)).to(t)
        if s["bias"] is not None:
            out["grad_bias"] = g.sum(0).to(t)
    return out


def _recurrence(a, b):
    """h_t = a_t h_{t-1} + b_t along axis 1 from h = 0: neighbours are joined, the sequence half as long is solved, the others follow."""
    n = a.shape[1]
    if n == 1:
        return b
    h = torch.empty_like(b)
    odd = _recurrence(a[:, 1::2] * a[:, :n - n % 2:2], b[:, 1::2] + a[:, 1::2] * b[:, :n - n % 2:2])
    h[:, 0], h[:, 1::2] = b[:, 0], odd
    h[:, 2::2] = b[:, 2::2] + a[:, 2::2] * odd[:, :(n - 1) // 2]
    return h


def _plain_gated(s):
    t, step = s["x"].dtype, s["kind"] == "gated_step"
    x, p, q = (s[k].float() for k in ("x", "decay_gate", "input_gate"))
    if step:
        x, p, q = x[:, None], p[:, None], q[:, None]
    L = x.shape[1]
    open_, i = torch.sigmoid(p), torch.sigmoid(q)
    u = torch.exp(s["log_rate"]) * open_
    a, size = torch.exp(-u), torch.sqrt(-torch.expm1(-2 * u))
    f = size * i * x
    live = None if step or s["lengths"] is None else (torch.arange(L, device="cuda")[None, :] < s["lengths"][:, None])[..., None]
    if live is not None:
        a, f = torch.where(live, a, 1.0), torch.where(live, f, 0.0)
    if s["state"] is not None:
        f[:, 0] += a[:, 0] * s["state"]
    h = _recurrence(a, f)
    if step:
        s["state"].copy_(h[:, 0])
        return {"y": h[:, 0].to(t), "state": s["state"]}
    out = {"y": (h if live is None else torch.where(live, h, 0.0)).to(t), "state": h[:, -1].clone()}
    if s["kind"] == "gated":
        return out
    g = s["grad_out"].float()
    if live is not None:
        g = torch.where(live, g, 0.0)
    if s["grad_state"] is not None:
        g[:, -1] += s["grad_state"]
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
    l = _recurrence(after.flip(1), g.flip(1)).flip(1)                       # the gradient with respect to each state
    before = torch.cat([s["state"][:, None] if s["state"] is not None else torch.zeros_like(h[:, :1]), h[:, :-1]], 1)
    first = a[:, 0] * l[:, 0]
    if live is not None:
        l = torch.where(live, l, 0.0)
    to_u = u * l * (a * a / size * i * x - a * before)                      # u times the gradient with respect to it
    out["grads"] = {"x": (l * size * i).to(t), "decay_gate": (to_u * (1 - open_)).to(t), "input_gate": (l * size * x * i * (1 - i)).to(t), "log_rate": to_u.sum((0, 1))}
    if s["state"] is not None:
        out["grads"]["initial_state"] = first
    return out


def exact(case, seed):
    """The same from the definitions in 64 bits, the recurrence one token after the other."""
    given = prepare(case, seed)
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in given.items()}
    t, kind, x, D = _type(case), case["kind"], s["x"], case["chans"]
    if kind.startswith("norm"):
        total = x if s["residual"] is None else (x + s["residual"]).to(t).double()                   # kept in the stream's type, by definition
        scale = 1 / torch.sqrt((total ** 2).sum(-1) / D + 1e-6)
        y = torch.einsum("...d,...,d->...d", total, scale, s["weight"])
        if kind == "norm8":
            top = y.abs().max(-1).values
            return {"y": torch.einsum("...d,...->...d", y, 448 / top).float().to(torch.float8_e4m3fn).double(), "scale": top / 448, "sum": total}
        out = {"y": y, "sum": total}
        if kind == "norm_train":
            along = (s["grad_out"] * y).sum(-1) / D * scale ** 2
            out["grad_x"] = s["grad_out"] * s["weight"] * scale[..., None] - total * along[..., None] + s["grad_sum"]
            out["grad_weight"] = torch.einsum("rd,rd,r->d", s["grad_out"].reshape(-1, D), total.reshape(-1, D), scale.reshape(-1))
        return out
    if kind.startswith("linear"):
        out, w = {}, s["weight"]
        if kind == "linear8":
            top = x.abs().max(-1).values
            x8 = (x * (448 / top)[..., None]).float().to(torch.float8_e4m3fn).double()
            out = {"x": x8, "scale": top / 448}
            x, w = x8 * out["scale"][..., None], w * s["weight_scale"][:, None]
        flat = x.reshape(-1, D)
        z = flat @ w.T + (s["bias"] if s["bias"] is not None else 0)
        z.requires_grad_()
        if case["act"] == "silu":
            y = z / (1 + torch.exp(-z))
        else:
            y = z * torch.special.ndtr(z) if case["act"] == "gelu" else z * 1
        if kind == "linear_train":
            g, = torch.autograd.grad(y, z, s["grad_out"].reshape(y.shape))
            out |= {"grad_x": (g @ w).reshape(x.shape), "grad_weight": g.T @ flat}
            out |= {"grad_bias": g.sum(0)} if s["bias"] is not None else {}
        y = y.detach().reshape(*x.shape[:-1], -1)
        return out | {"y": y if s["residual"] is None else y + s["residual"]}
    step, n = kind == "gated_step", case["batch"]
    p, q = s["decay_gate"], s["input_gate"]
    if step:
        x, p, q = x[:, None], p[:, None], q[:, None]
    L, ends = x.shape[1], torch.tensor(_lengths(case), device="cuda")
    rate = torch.exp(s["log_rate"])
    first = s["state"].clone() if case["carry"] else torch.zeros(n, D, dtype=torch.float64, device="cuda")
    h, y, before = first, torch.zeros_like(x), torch.empty_like(x)
    for k in range(L):
        on = (k < ends)[:, None]
        before[:, k] = h
        a = torch.exp(-rate / (1 + torch.exp(-p[:, k])))
        new = a * h + torch.sqrt((1 - a) * (1 + a)) * x[:, k] / (1 + torch.exp(-q[:, k]))
        y[:, k] = torch.where(on, new, 0)
        h = torch.where(on, new, h)
    if step:
        return {"y": y[:, 0], "state": h}
    out = {"y": y, "state": h}
    if kind == "gated":
        return out
    l = s["grad_state"].clone() if case["carry"] else torch.zeros_like(first)
    gx, gp, gq, gr = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(rate)
    for k in reversed(range(L)):
        on = (k < ends)[:, None]
        open_, i = 1 / (1 + torch.exp(-p[:, k])), 1 / (1 + torch.exp(-q[:, k]))
        a = torch.exp(-rate * open_)
        size = torch.sqrt((1 - a) * (1 + a))
        now = torch.where(on, l + s["grad_out"][:, k], 0)
        to_a = now * (before[:, k] - a / size * i * x[:, k])
        to_gate = -to_a * a * rate * open_
        gx[:, k], gq[:, k], gp[:, k] = now * size * i, now * size * x[:, k] * i * (1 - i), to_gate * (1 - open_)
        gr += to_gate.sum(0)
        l = torch.where(on, now * a, l)
    grads = {"x": gx, "decay_gate": gp, "input_gate": gq, "log_rate": gr}
    return out | {"grads": grads | ({"initial_state": l} if case["carry"] else {})}


def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    D, all_ = case["chans"], case["batch"] * case["time"]
    if kind.startswith("norm"):
        moved = all_ * D * (e * (1 + 2 * case["residual"]) + (1 if kind == "norm8" else e)) + 4 * D + (4 * all_ if kind == "norm8" else 0)
        if kind == "norm_train":    # the sum, both gradients and the tokens' gradient
            moved += 4 * all_ * D * e + 8 * D
        return {"bytes": moved, "flops": all_ * D * (18 if kind == "norm_train" else 6)}
    if kind.startswith("linear"):
        N = case["outs"]
        moved = all_ * (D + N * (1 + case["residual"])) * e + N * D * e + case["bias"] * N * e
        if kind == "linear8":       # tokens in their type once, then in 8 bits, written and read; weights in 8 bits
            moved += 2 * all_ * D - N * D * (e - 1) + 8 * all_ + 4 * N
        if kind == "linear_train":  # the intermediate written and read, tokens, weights and the gradient read, three gradients written
            moved += (2 * (case["act"] != "none") * all_ * N + all_ * (2 * D + N) + 2 * N * D + case["bias"] * N) * e
        return {"bytes": moved, "flops": all_ * N * D * (6 if kind == "linear_train" else 2)}
    live, states = sum(_lengths(case)), case["batch"] * D * 4 * (1 + case["carry"])
    moved = (3 * live + all_) * D * e + states + 4 * D
    flops = live * D * 20
    if kind == "gated_train":
        moved += (4 * live + 3 * all_) * D * e + case["carry"] * 2 * case["batch"] * D * 4 + 8 * D
        flops += live * D * 45
    return {"bytes": moved, "flops": flops}
