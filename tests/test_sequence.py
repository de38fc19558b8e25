"""Sequence operators (short causal convolution, selective scan, gradient clipping) against plain 64-bit implementations.

Tolerances.  float32 results: every token adds a handful of roundings of 6e-8, sums over tokens, streams and channels add theirs with signs
that vary; norm-wise 1e-5 leaves two digits for the decay of the states (a relative error of one rounding a token, remembered over the
10 to 100 tokens that step sizes of 0.05 and more give).  bfloat16 results are rounded once more, to 2^-9: norm-wise 2^-8.  Single values: 20
times that of the larger of their size and the root mean square, for sums whose terms cancel."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2602_24066_amd as S
from tests import seq_reference as R

TOL = {torch.float32: 1e-5, torch.bfloat16: 2.0 ** -8}
gpu = pytest.mark.gpu


def close(got, want, dtype, what):
    got, want = got.detach().double().cpu(), want.double()
    assert got.shape == want.shape, f"{what}: shape {tuple(got.shape)} for {tuple(want.shape)}"
    assert torch.isfinite(got).all(), f"{what}: not finite"
    if want.numel() == 0:
        return
    rms = float(want.square().mean().sqrt())
    off = got - want
    assert float(off.square().mean().sqrt()) <= TOL[dtype] * rms, f"{what}: {float(off.square().mean().sqrt()) / max(rms, 1e-300):.2e} of the norm"
    worst = float((off.abs() / want.abs().clamp(min=max(rms, 1e-300))).max())
    assert worst <= 20 * TOL[dtype], f"{what}: a value is {worst:.2e} off"


def up(v):
    return v.cuda() if isinstance(v, torch.Tensor) else v


def poison(case, names):
    """NaN in every token that lengths hides."""
    out = dict(case)
    for k in names:
        if out.get(k) is not None:
            out[k] = out[k].clone()
            for i in range(out[k].shape[0]):
                out[k][i, R._len(case["lengths"], i, out[k].shape[1]):] = math.nan
    return out


# ------------------------------------------------------------------------------------------------ convolution
CONV = [
    # B, L, D, W, type, carried state, bias, lengths
    (2, 33, 64, 4, "f32", True, True, None),
    (2, 33, 64, 4, "bf16", True, True, None),
    (3, 100, 37, 3, "f32", True, True, [100, 0, 41]),          # odd channels, a stream without tokens
    (3, 70, 40, 2, "bf16", False, True, [1, 70, 69]),
    (1, 1, 5, 4, "f32", True, False, None),                    # one token: most of the final state is the old one
    (2, 2, 8, 8, "bf16", True, True, [2, 1]),                  # fewer tokens than the filter has
    (4, 17, 1, 1, "f32", False, True, None),                   # a filter of one token keeps no state
    (2, 50, 24, 5, "f32", True, False, [-3, 77]),              # lengths out of range are clamped
    (1, 300, 130, 6, "bf16", False, False, None),
    (2, 64, 16, 7, "f32", True, True, [64, 5]),
]


@gpu
@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("case", range(len(CONV)))
def test_conv_and_its_gradient(case, silu):
    B, L, D, W, t, carry, bias, lengths = CONV[case]
    t = torch.float32 if t == "f32" else torch.bfloat16
    v = R.inputs("conv", B, L, D, W=W, dtype=t, carry=carry, full=bias, lengths=lengths, seed=case)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    y, state, grads = R.with_gradients(R.conv, v, gy, gs, silu=silu)
    d = {k: up(w) for k, w in poison(v, ["x"]).items()}
    got_y, got_state = S.sig_conv_forward(**d, silu=silu, return_state=True)
    close(got_y, y, t, "y")
    close(got_state, state, t, "state")
    gy = poison({"g": gy, "lengths": v["lengths"]}, ["g"])["g"]
    gx, gw, gb, gi = S.sig_conv_backward(d["x"], d["weight"], up(gy), d["bias"], d["initial_state"], d["lengths"], silu, up(gs))
    close(gx, grads["x"], t, "grad x")
    close(gw, grads["weight"], torch.float32, "grad weight")
    assert (gb is None) == (v["bias"] is None) and (gi is None) == (v["initial_state"] is None)
    if gb is not None:
        close(gb, grads["bias"], torch.float32, "grad bias")
    if gi is not None:
        close(gi, grads["initial_state"], t, "grad initial state")


@gpu
@pytest.mark.parametrize("t,D,W", [(torch.float32, 33, 4), (torch.bfloat16, 64, 3), (torch.bfloat16, 7, 2), (torch.float32, 4, 1)])
def test_conv_steps_continue_a_prompt(t, D, W):
    v = R.inputs("conv", 3, 23, D, W=W, dtype=t, lengths=None, seed=5)
    y, state, _ = R.with_gradients(R.conv, {k: v[k] for k in ("x", "weight", "bias", "initial_state")}, v["grad_out"], None)
    d = {k: up(v[k]) for k in ("x", "weight", "bias", "initial_state")}
    _, held = S.sig_conv_forward(d["x"][:, :9], d["weight"], d["bias"], d["initial_state"], return_state=True)
    rows = [S.sig_conv_step(d["x"][:, i], held, d["weight"], d["bias"]) for i in range(9, 23)]
    close(torch.stack(rows, 1), y[:, 9:], t, "y")
    assert torch.equal(held.cpu().double(), state)


# ------------------------------------------------------------------------------------------------ selective scan
SCAN = [
    # B, L, D, G, N, type, carried state, gate + skip + bias + softplus, lengths
    (2, 33, 64, 1, 16, "f32", True, True, None),
    (2, 48, 64, 1, 16, "bf16", True, True, None),
    (3, 50, 37, 1, 16, "f32", True, True, [50, 0, 17]),        # odd channels, a stream without tokens
    (2, 40, 130, 2, 12, "f32", True, True, [16, 40]),          # groups of 65 channels, states that fill no register group; a length at a tile's end
    (2, 35, 48, 3, 16, "bf16", False, True, [1, 35]),
    (1, 1, 5, 1, 16, "f32", True, True, None),                 # one token
    (1, 15, 1, 1, 1, "f32", False, False, None),               # one channel, one state
    (2, 31, 18, 18, 3, "f32", True, True, None),               # a group for every channel
    (2, 17, 40, 1, 8, "bf16", True, False, [17, 9]),
    (1, 70, 24, 2, 32, "f32", True, True, None),
    (1, 37, 20, 1, 20, "bf16", True, True, None),
    (2, 40, 9, 1, 64, "f32", True, True, [40, 33]),
    (1, 33, 12, 1, 33, "f32", False, True, None),
    (1, 600, 70, 1, 16, "f32", True, True, None),              # long: many tiles
    (2, 300, 66, 1, 4, "bf16", False, True, [-1, 1000]),       # lengths out of range are clamped
    (1, 2100, 17, 1, 16, "f32", True, True, [2077]),
    (34, 20, 512, 2, 16, "bf16", False, True, None),           # more workgroups than compute units: no time chunks
    (3, 500, 65, 1, 16, "f32", True, True, [500, 480, 31]),    # time chunks that lie beyond a stream's tokens, a length at a chunk's end
    (1, 5000, 3, 1, 8, "f32", True, False, None),              # as many time chunks as there are
    (2, 130, 33, 1, 48, "bf16", True, True, [129, 2]),
]


def scan_case(case):
    B, L, D, G, N, t, carry, full, lengths = SCAN[case]
    t = torch.float32 if t == "f32" else torch.bfloat16
    v = R.inputs("scan", B, L, D, G=G, N=N, dtype=t, carry=carry, full=full, lengths=lengths, seed=100 + case)
    return v, t, full


@gpu
@pytest.mark.parametrize("case", range(len(SCAN)))
def test_scan_and_its_gradient(case):
    v, t, full = scan_case(case)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    y, state, grads = R.with_gradients(R.scan, v, gy, gs, softplus=full)
    hidden = poison({**v, "gy": gy}, ["x", "dt", "b", "c", "gate", "gy"])
    gy = hidden.pop("gy")
    d = {k: up(w) for k, w in hidden.items()}
    got_y, got_state = S.sig_scan_forward(**d, softplus=full)
    close(got_y, y, t, "y")
    close(got_state, state, torch.float32, "state")
    again_y, again_state, ck = S.sig_scan_forward(**d, softplus=full, checkpoint=True)
    close(again_y, y, t, "y with checkpoint")
    close(again_state, state, torch.float32, "state with checkpoint")
    got = S.sig_scan_backward(**d, softplus=full, grad_out=up(gy), checkpoint=ck, grad_final_state=up(gs))
    for k, name in dict(x="x", dt="dt", A="A", b="B", c="C", skip="skip", gate="gate", dt_bias="dt_bias", initial_state="initial_state").items():
        assert (got[name] is None) == (v[k] is None), name
        if v[k] is not None:
            close(got[name], grads[k], t if k in ("x", "dt", "b", "c", "gate") else torch.float32, "grad " + name)


@gpu
@pytest.mark.parametrize("case", [0, 3, 9])
def test_scan_gradient_is_the_slope_of_the_definition(case):
    """<gradient, v> against central differences of the 64-bit forward pass along random directions v (step 1e-4: truncation of some 1e-8)."""
    v, t, full = scan_case(case)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    d = {k: up(w) for k, w in v.items()}
    got = S.sig_scan_backward(**d, softplus=full, grad_out=up(gy), checkpoint=S.sig_scan_forward(**d, softplus=full, checkpoint=True)[2],
                              grad_final_state=up(gs))
    wide = {k: w.double() if w is not None and w.is_floating_point() else w for k, w in v.items()}

    def loss(**moved):
        y, state = R.scan(**{**wide, **moved}, softplus=full)
        return float((y * gy.double()).sum() + (0.0 if gs is None else (state * gs.double()).sum()))

    rnd = torch.Generator().manual_seed(case)
    for k in ("x", "dt", "A", "b", "c", "skip", "gate", "dt_bias", "initial_state"):
        if v[k] is None:
            continue
        way = torch.randn(v[k].shape, generator=rnd, dtype=torch.float64)
        way /= way.norm()
        eps = 1e-4
        slope = (loss(**{k: wide[k] + eps * way}) - loss(**{k: wide[k] - eps * way})) / (2 * eps)
        g = got["BC"["bc".index(k)] if k in ("b", "c") else k].double().cpu()
        g = g.reshape(v[k].shape)
        assert abs(float((g * way).sum()) - slope) <= 2e-5 * float(g.norm()), k


@gpu
@pytest.mark.parametrize("t,D,G,N,full", [(torch.float32, 33, 1, 16, True), (torch.bfloat16, 64, 2, 16, True), (torch.bfloat16, 24, 1, 5, False),
                                          (torch.float32, 10, 1, 40, True)])
def test_scan_steps_continue_a_prompt(t, D, G, N, full):
    v = R.inputs("scan", 3, 21, D, G=G, N=N, dtype=t, full=full, seed=7)
    gy = v.pop("grad_out")
    v.pop("grad_final_state")
    y, state, _ = R.with_gradients(R.scan, v, gy, None, softplus=full)
    d = {k: up(w) for k, w in v.items()}
    cut = lambda a, b: {k: w[:, a:b] if k in ("x", "dt", "b", "c", "gate") and w is not None else w for k, w in d.items()}    # noqa: E731
    _, held = S.sig_scan_forward(**cut(0, 8), softplus=full)
    rows = []
    for i in range(8, 21):
        one = {k: w[:, 0] if k in ("x", "dt", "b", "c", "gate") and w is not None else w for k, w in cut(i, i + 1).items()}
        one.pop("initial_state"), one.pop("lengths")
        rows.append(S.sig_scan_step(state=held, softplus=full, **one))
    close(torch.stack(rows, 1), y[:, 8:], t, "y")
    close(held, state, torch.float32, "state")


@gpu
def test_prompts_in_two_parts_and_without_tokens():
    v = R.inputs("scan", 2, 50, 48, dtype=torch.float32, seed=3)
    v.pop("grad_out"), v.pop("grad_final_state")
    d = {k: up(w) for k, w in v.items()}
    cut = lambda a, b, h: {**{k: w[:, a:b] if k in ("x", "dt", "b", "c", "gate") else w for k, w in d.items()}, "initial_state": h}   # noqa: E731
    y, state = S.sig_scan_forward(**d)
    y1, h = S.sig_scan_forward(**cut(0, 19, d["initial_state"]))
    y0, h = S.sig_scan_forward(**cut(19, 19, h))
    assert y0.shape == (2, 0, 48)
    y2, h = S.sig_scan_forward(**cut(19, 50, h))
    close(torch.cat([y1, y2], 1), y.cpu(), torch.float32, "y")
    close(h, state.cpu(), torch.float32, "state")
    _, _, ck = S.sig_scan_forward(**cut(0, 0, d["initial_state"]), checkpoint=True)
    g = S.sig_scan_backward(**cut(0, 0, d["initial_state"]), grad_out=y0, checkpoint=ck, grad_final_state=state)
    assert torch.equal(g["initial_state"], state) and not g["A"].any() and not g["skip"].any() and not g["dt_bias"].any()
    _, kept = S.sig_conv_forward(d["x"][:, :0], torch.ones(48, 4, device="cuda"), initial_state=d["x"][:, :3].contiguous(), return_state=True)
    assert torch.equal(kept, d["x"][:, :3])


@gpu
def test_no_streams():
    x = torch.zeros(0, 9, 32, device="cuda")
    b = torch.zeros(0, 9, 16, device="cuda")
    A = -torch.ones(32, 16, device="cuda")
    w = torch.ones(32, 4, device="cuda")
    assert S.sig_conv_forward(x, w).shape == x.shape
    gx, gw, gb, _ = S.sig_conv_backward(x, w, x, bias=torch.ones(32, device="cuda"))
    assert not gw.any() and not gb.any()
    y, h, ck = S.sig_scan_forward(x, x, A, b, b, skip=A[:, 0].contiguous(), checkpoint=True)
    g = S.sig_scan_backward(x, x, A, b, b, x, ck, skip=A[:, 0].contiguous())
    assert h.shape == (0, 32, 16) and not g["A"].any() and not g["skip"].any() and g["B"].shape == b.shape
    assert S.sig_scan_step(x[:, 0], x[:, 0], A, b[:, 0], b[:, 0], h).shape == (0, 32)


@gpu
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_strided_broadcast_and_unaligned_inputs(t):
    """Slices of wider rows (also at odd offsets), expanded axes and transposed layouts give what contiguous copies give."""
    rnd = torch.Generator(device="cuda").manual_seed(1)
    B, L, D, N = 2, 37, 72, 16
    wide = torch.randn(B, L, 2 * D + 5, generator=rnd, device="cuda").to(t)
    bc = torch.randn(1, L, 2 * N + 3, generator=rnd, device="cuda").to(t)
    x, gate = wide[..., 1:D + 1], wide[..., D + 3:2 * D + 3]
    dt = (torch.randn(B, D, L, generator=rnd, device="cuda") - 2).to(t).transpose(1, 2)
    b, c = bc[..., 3:N + 3].expand(B, L, N), bc[..., N + 3:].expand(B, L, N)
    A = -torch.exp(torch.randn(N, D, generator=rnd, device="cuda")).t()
    gy = torch.randn(L, B, D, generator=rnd, device="cuda").to(t).transpose(0, 1)
    w, bias = torch.randn(4, D, generator=rnd, device="cuda").t(), torch.randn(2 * D, generator=rnd, device="cuda")[::2]
    one = lambda f: f(lambda v: v)                                                          # noqa: E731
    two = lambda f: f(lambda v: v.contiguous().clone())                                     # noqa: E731

    def everything(k):
        y, h, ck = S.sig_scan_forward(k(x), k(dt), k(A), k(b), k(c), gate=k(gate), checkpoint=True)
        g = S.sig_scan_backward(k(x), k(dt), k(A), k(b), k(c), k(gy), ck, gate=k(gate))
        return [y, h, S.sig_conv_forward(k(x), k(w), k(bias)), *S.sig_conv_backward(k(x), k(w), k(gy), k(bias))[:3],
                S.sig_conv_step(k(x[:, 3]), torch.zeros(B, 3, D, device="cuda", dtype=t), k(w)),
                S.sig_scan_step(k(x[:, 3]), k(dt[:, 3]), k(A), k(b[:, 3]), k(c[:, 3]), torch.ones(B, D, N, device="cuda"), gate=k(gate[:, 3]))] + [
                    v for v in g.values() if v is not None]

    for p, q in zip(one(everything), two(everything)):
        close(p, q.cpu(), torch.float32 if p.dtype == torch.float32 else t, "strided")


@gpu
def test_offsets_beyond_32_bits():
    """Streams that lie more than 2^32 bytes and 2^31 elements apart."""
    far = (1 << 31) + 64
    B, L, D, N = 2, 20, 64, 16
    store = torch.empty(far + L * D, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((B, L, D), (far, D, 1))
    x.copy_(torch.randn(B, L, D, device="cuda"))
    near = x.contiguous()
    b = torch.randn(B, L, N, device="cuda").bfloat16()
    A, w = -torch.ones(D, N, device="cuda"), torch.ones(D, 4, device="cuda")
    for v, u in ((x, near), (near, near)):
        got = [*S.sig_scan_forward(v, v, A, b, b, gate=v), S.sig_conv_forward(v, w), *S.sig_conv_backward(v, w, v)[:2]]
        ck = S.sig_scan_forward(v, v, A, b, b, gate=v, checkpoint=True)[2]
        got += list(S.sig_scan_backward(v, v, A, b, b, v, ck, gate=v).values())
        if v is x:
            first = got
    for p, q in zip(first, got):
        assert p is None and q is None or torch.equal(p, q)


@gpu
def test_time_strides_beyond_the_kernels_reach():
    """Tokens 2^26 elements apart are copied by the package and refused by the library; 2^22 apart they are read as they are."""
    D, N, L = 24, 16, 3
    w, A = torch.randn(D, 4, device="cuda"), -torch.ones(D, N, device="cuda")
    store = torch.empty((L - 1 << 26) + D, dtype=torch.bfloat16, device="cuda")
    b = torch.randn(1, L, N, device="cuda").bfloat16()
    for step in (1 << 26, 1 << 22):
        x = store.as_strided((1, L, D), (1, step, 1))
        x.copy_(torch.randn(1, L, D, device="cuda"))
        near = x.contiguous()
        assert torch.equal(S.sig_conv_forward(x, w), S.sig_conv_forward(near, w))
        ck = S.sig_scan_forward(near, near, A, b, b, checkpoint=True)[2]
        for p, q in zip((*S.sig_scan_forward(x, x, A, b, b, gate=x), *S.sig_scan_backward(x, x, A, b, b, x, ck, gate=x).values()),
                        (*S.sig_scan_forward(near, near, A, b, b, gate=near), *S.sig_scan_backward(near, near, A, b, b, near, ck, gate=near).values())):
            assert p is None and q is None or torch.equal(p, q)


@gpu
def test_parameters_and_subclasses_give_plain_tensors():
    class Mine(torch.Tensor):
        pass
    x, w = torch.randn(1, 9, 16, device="cuda"), torch.nn.Parameter(torch.randn(16, 4, device="cuda"))
    b, A = torch.randn(1, 9, 4, device="cuda", requires_grad=True), torch.nn.Parameter(-torch.ones(16, 4, device="cuda"))
    for v in (x.as_subclass(Mine), torch.nn.Parameter(x)):
        y = S.sig_conv_forward(v, w)
        h, state = S.sig_scan_forward(v, v, A, b, b)
        assert type(y) is torch.Tensor and type(h) is torch.Tensor and type(state) is torch.Tensor and not y.requires_grad and not h.requires_grad
        assert torch.equal(y, S.sig_conv_forward(x, w)) and torch.equal(h, S.sig_scan_forward(x, x, A, b, b)[0])


@gpu
def test_special_values():
    """Infinite decay (a state is forgotten at once), growth, step sizes of zero and very negative raw step sizes."""
    B, L, D, N = 1, 40, 16, 16
    v = R.inputs("scan", B, L, D, dtype=torch.float32, seed=11)
    gy = v.pop("grad_out")
    gs = v.pop("grad_final_state")
    v["A"][:, 0], v["A"][:, 1], v["A"][:, 2] = -1e30, 0.0, 0.05
    v["dt"][0, 5], v["dt"][0, 6] = -200.0, -30.0
    y, state, grads = R.with_gradients(R.scan, v, gy, gs)
    d = {k: up(w) for k, w in v.items()}
    got_y, got_state, ck = S.sig_scan_forward(**d, checkpoint=True)
    close(got_y, y, torch.float32, "y")
    close(got_state, state, torch.float32, "state")
    got = S.sig_scan_backward(**d, grad_out=up(gy), checkpoint=ck, grad_final_state=up(gs))
    for k in ("x", "b", "c", "gate", "skip", "initial_state"):
        close(got[{"b": "B", "c": "C"}.get(k, k)], grads[k], torch.float32, k)


@gpu
def test_a_stream_with_nan_leaves_the_others_alone():
    v = R.inputs("scan", 3, 33, 32, dtype=torch.float32, seed=2)
    gy, gs = up(v.pop("grad_out")), up(v.pop("grad_final_state"))
    d = {k: up(w) for k, w in v.items()}
    clean_y, clean_h, ck = S.sig_scan_forward(**d, checkpoint=True)
    clean = S.sig_scan_backward(**d, grad_out=gy, checkpoint=ck, grad_final_state=gs)
    d["x"][1, 20, 3] = math.nan
    y, h, ck = S.sig_scan_forward(**d, checkpoint=True)
    got = S.sig_scan_backward(**d, grad_out=gy, checkpoint=ck, grad_final_state=gs)
    for p, q in ((y, clean_y), (h, clean_h), *((got[k], clean[k]) for k in ("x", "dt", "B", "C", "gate", "initial_state"))):
        assert torch.equal(p[0], q[0]) and torch.equal(p[2], q[2])
    assert torch.equal(y[1, :20], clean_y[1, :20]) and torch.isnan(y[1, 20:, 3]).all() and torch.isfinite(y[1, :, 4]).all()
    assert torch.isnan(h[1, 3]).all()


@gpu
def test_same_inputs_same_bits_on_any_stream():
    v = R.inputs("scan", 2, 400, 96, dtype=torch.bfloat16, seed=9, lengths=[400, 123])
    gy, gs = up(v.pop("grad_out")), up(v.pop("grad_final_state"))
    d = {k: up(w) for k, w in v.items()}
    w = torch.randn(96, 4, device="cuda")

    def all_of():
        y, h, ck = S.sig_scan_forward(**d, checkpoint=True)
        g = S.sig_scan_backward(**d, grad_out=gy, checkpoint=ck, grad_final_state=gs)
        more = S.sig_conv_backward(d["x"], w, gy, lengths=d["lengths"])
        grads = [g["A"].clone(), g["x"].clone()]
        return [y, h, *g.values(), *more[:2], S.sig_grad_clip(grads, 0.5), *grads]

    first = all_of()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = all_of()
    side.synchronize()
    for p, q in zip(first, second):
        assert torch.equal(p, q)


@gpu
def test_a_captured_step_replays():
    """A training pass and a streaming step recorded in a graph give, on every replay, what eager calls give on the inputs of then."""
    v = R.inputs("scan", 2, 64, 64, dtype=torch.bfloat16, seed=4)
    gy, gs = up(v.pop("grad_out")), up(v.pop("grad_final_state"))
    v.pop("lengths")
    d = {k: up(w) for k, w in v.items()}
    w = torch.randn(64, 4, device="cuda")
    tail = torch.zeros(2, 3, 64, device="cuda", dtype=torch.bfloat16)
    h1 = torch.zeros(2, 64, 16, device="cuda")

    def all_of(tail, h1):
        u = S.sig_conv_forward(d["x"], w)
        y, h, ck = S.sig_scan_forward(**{**d, "x": u}, checkpoint=True)
        g = S.sig_scan_backward(**{**d, "x": u}, grad_out=gy, checkpoint=ck, grad_final_state=gs)
        gx, gw, _, _ = S.sig_conv_backward(d["x"], w, g["x"])
        norm = S.sig_grad_clip([gw, g["A"]], 1.0)
        s = S.sig_conv_step(d["x"][:, 0], tail, w)
        o = S.sig_scan_step(s, d["dt"][:, 0], d["A"], d["b"][:, 0], d["c"][:, 0], h1)
        return [y, h, gx, gw, g["A"], g["B"], norm, o]

    all_of(tail.clone(), h1.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = all_of(tail, h1)
    for k in range(3):
        d["x"].copy_(torch.randn(2, 64, 64, device="cuda"))
        want_tail, want_h = tail.clone(), h1.clone()
        want = all_of(want_tail, want_h)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip([*kept, tail, h1], [*want, want_tail, want_h]):
            assert torch.equal(p, q), k


# ------------------------------------------------------------------------------------------------ gradient clipping
def clip_reference(grads, max_norm):
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    return norm, [g.double() * min(1.0, max_norm / (norm + 1e-6)) for g in grads]


@gpu
@pytest.mark.parametrize("max_norm", [0.0, 0.25, 1e9])
@pytest.mark.parametrize("sizes", [[(1,)], [(5, 7), (0,), (1,), (16385,)], [(3, 3)] * 300, [(40000,), (16384,), (255,), (2, 8191)]])
@pytest.mark.parametrize("kinds", ["f32", "bf16", "mixed"])
def test_clip(sizes, kinds, max_norm):
    g = torch.Generator().manual_seed(len(sizes))
    types = [torch.bfloat16 if kinds == "bf16" or (kinds == "mixed" and i % 2) else torch.float32 for i in range(len(sizes))]
    grads = [torch.randn(*s, generator=g).to(t) for s, t in zip(sizes, types)]
    norm, want = clip_reference(grads, max_norm)
    on = [up(v) for v in grads]
    outs = [torch.full(v.shape, 7.0, device="cuda", dtype=torch.float32) for v in on]
    got = S.sig_grad_clip(on, max_norm, out=outs)
    assert got.shape == () and abs(float(got) - norm) <= 1e-6 * norm
    for p, q, v in zip(outs, want, on):
        close(p, q, torch.float32, "copies")
    assert all(torch.equal(v.cpu(), w) for v, w in zip(on, grads)), "inputs are left alone"
    assert float(S.sig_grad_clip(on, max_norm)) == float(got)
    for p, q in zip(on, want):
        close(p, q, p.dtype, "in place")
    if max_norm == 1e9:
        assert all(torch.equal(v.cpu(), w) for v, w in zip(on, grads)), "nothing to clip"


@gpu
def test_clip_of_views_layouts_and_extremes():
    flat = torch.randn(4096 + 3, device="cuda")
    views = [flat[1:1001], flat[1003:1003 + 64 * 40].view(64, 40).t(), flat[4000:4001]]          # odd offsets, a transposed matrix
    rest = flat.clone()
    norm, want = clip_reference([v.cpu() for v in views], 1.0)
    got = S.sig_grad_clip(views, 1.0)
    assert abs(float(got) - norm) <= 1e-6 * norm
    for p, q in zip(views, want):
        close(p, q, torch.float32, "views")
    untouched = torch.ones(4099, dtype=torch.bool, device="cuda")
    untouched[1:1001] = untouched[1003:1003 + 64 * 40] = untouched[4000] = False
    assert torch.equal(flat[untouched], rest[untouched])
    big = [torch.full((1000,), 1e30, device="cuda"), torch.full((10,), 1e-30, device="cuda")]    # squares that float32 does not hold
    assert abs(float(S.sig_grad_clip(big, 1.0)) / (1e30 * math.sqrt(1000)) - 1) <= 1e-6
    assert abs(float(big[0][0]) * math.sqrt(1000) - 1) <= 1e-5
    assert float(S.sig_grad_clip([torch.full((10,), 1e-30, device="cuda")], 1.0)) == pytest.approx(1e-30 * math.sqrt(10), rel=1e-6)
    bad = [torch.ones(5, device="cuda"), torch.tensor([1.0, math.nan], device="cuda")]
    assert math.isnan(float(S.sig_grad_clip(bad, 1.0))) and torch.isnan(bad[0]).all()
    far = [torch.ones(5, device="cuda"), torch.tensor([1.0, math.inf], device="cuda")]
    assert math.isinf(float(S.sig_grad_clip(far, 1.0))) and not far[0].any() and torch.isnan(far[1][1])
    assert float(S.sig_grad_clip([], 1.0)) == 0.0
    assert float(S.sig_grad_clip([torch.empty(0, device="cuda")], 1.0)) == 0.0


# ------------------------------------------------------------------------------------------------ refusals
def pack(fields, order):
    return (ctypes.c_int64 * len(order))(*[int(fields[k]) for k in order])


CONV_ORDER = "dtype B L D W silu xb xt x weight bias initial lengths".split()
SCAN_ORDER = "dtype B L D G N softplus xb xt tb tt zb zt bb bt bg cb ct cg x dt gate b c A skip bias initial lengths".split()
GRADS_ORDER = "gb gt gy gfinal gx gdt gz gbb gcc gA gskip gbias ginitial".split()


@pytest.mark.parametrize("change,code", [({"dtype": 2}, -1), ({"B": -1}, -1), ({"L": -1}, -1), ({"D": 0}, -1), ({"W": 0}, -1), ({"W": 9}, -9), ({"silu": 2}, -1),
                                         ({"x": 0}, -1), ({"weight": 0}, -1), ({"L": 1 << 41}, -7), ({"B": 0}, 0)])
def test_conv_refuses_through_the_c_abi(change, code):
    """Every refusal comes before anything touches the device (the pointers here lead nowhere)."""
    lib = S.load_library()
    ok = dict(dtype=0, B=2, L=8, D=4, W=4, silu=1, xb=32, xt=4, x=4096, weight=4096, bias=0, initial=0, lengths=0)
    args = pack({**ok, **change}, CONV_ORDER)
    assert lib.sig_conv_forward(args, 4096, 0, 0) == code
    if "L" not in change:
        assert lib.sig_conv_step(args, 4096, 4096, 0) == code
    if change != {"B": 0}:
        assert lib.sig_conv_backward(args, 4096, 32, 4, 0, 4096, 4096, 0, 0, 4096, 1 << 40, 0) == code


def test_more_refusals_of_the_conv():
    lib = S.load_library()
    args = pack(dict(dtype=0, B=2, L=8, D=4, W=4, silu=1, xb=32, xt=4, x=4096, weight=4096, bias=0, initial=0, lengths=0), CONV_ORDER)
    assert lib.sig_conv_forward(None, 4096, 0, 0) == -1
    assert lib.sig_conv_forward(args, 0, 0, 0) == -1
    assert lib.sig_conv_step(args, 0, 4096, 0) == -1
    need = lib.sig_conv_backward_workspace_bytes(args)
    assert need > 0
    assert lib.sig_conv_backward(args, 4096, 32, 4, 0, 4096, 4096, 0, 0, 4096, need - 1, 0) == -5
    assert lib.sig_conv_backward(args, 4096, 32, 4, 0, 4096, 4096, 0, 0, 0, need, 0) == -5
    assert lib.sig_conv_backward(args, 0, 32, 4, 0, 4096, 4096, 0, 0, 4096, need, 0) == -1
    assert lib.sig_conv_backward_workspace_bytes(None) == 0


@pytest.mark.parametrize("change,code", [({"dtype": -1}, -1), ({"B": -1}, -1), ({"L": -1}, -1), ({"D": 0}, -1), ({"G": 0}, -1), ({"G": 3}, -1), ({"N": 0}, -1),
                                         ({"N": 65}, -9), ({"softplus": 3}, -1), ({"x": 0}, -1), ({"dt": 0}, -1), ({"b": 0}, -1), ({"c": 0}, -1), ({"A": 0}, -1),
                                         ({"L": 1 << 40}, -7), ({"L": 1 << 31}, -7), ({"xt": 1 << 26}, -7), ({"bt": 1 << 26}, -7),
                                         ({"ct": -1}, -1), ({"B": 1 << 30}, -7), ({"B": 0}, 0)])
def test_scan_refuses_through_the_c_abi(change, code):
    lib = S.load_library()
    ok = dict.fromkeys(SCAN_ORDER, 0) | dict(dtype=0, B=2, L=8, D=4, G=2, N=4, softplus=1, x=4096, dt=4096, b=4096, c=4096, A=4096)
    args = pack({**ok, **change}, SCAN_ORDER)
    big = 1 << 60
    assert lib.sig_scan_forward(args, 4096, 4096, 4096, big, 4096, big, 0) == code
    if "L" not in change and "xt" not in change:
        assert lib.sig_scan_step(args, 4096, 4096, 0) == code
    if change != {"B": 0}:
        grads = pack(dict.fromkeys(GRADS_ORDER, 4096), GRADS_ORDER)
        assert lib.sig_scan_backward(args, grads, 4096, big, 4096, big, 0) == code


def test_the_longest_scan():
    lib = S.load_library()
    args = lambda L: pack(dict.fromkeys(SCAN_ORDER, 0) | dict(dtype=0, B=1, L=L, D=1, G=1, N=1, softplus=1, x=4096, dt=4096, b=4096, c=4096, A=4096), SCAN_ORDER)   # noqa: E731
    big = 1 << 60
    assert lib.sig_scan_checkpoint_bytes(args((1 << 30) - 1)) == 1 << 28          # 2^26 tiles, a float each
    assert lib.sig_scan_forward(args((1 << 30) - 1), 0, 0, 0, 0, 4096, big, 0) == -1
    assert lib.sig_scan_forward(args(1 << 30), 4096, 0, 0, 0, 4096, big, 0) == -7
    assert lib.sig_scan_checkpoint_bytes(args(1 << 30)) == 0


@pytest.mark.parametrize("change,code", [({"bt": 3}, -1), ({"ct": 1}, -1), ({"bt": 4, "ct": 4, "x": 0}, -1), ({"bt": 3, "L": 1, "B": 0}, 0)])
def test_overlapping_rows_are_refused_by_the_c_abi(change, code):
    lib = S.load_library()
    ok = dict.fromkeys(SCAN_ORDER, 0) | dict(dtype=0, B=2, L=8, D=4, G=1, N=4, softplus=1, x=4096, dt=4096, b=4096, c=4096, A=4096)
    assert lib.sig_scan_forward(pack({**ok, **change}, SCAN_ORDER), 4096, 0, 0, 0, 4096, 1 << 60, 0) == code


@gpu
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_overlapping_windows_as_b_and_c(t):
    B, L, D, N = 3, 37, 70, 12
    x, dt, A = torch.randn(B, L, D, device="cuda").to(t), torch.randn(B, L, D, device="cuda").to(t), -torch.rand(D, N, device="cuda")
    b, c = (torch.randn(B, L + N - 1, device="cuda").to(t).unfold(1, N, 1) for _ in range(2))
    lengths = torch.tensor([37, 0, 20], dtype=torch.int32, device="cuda")
    got = S.sig_scan_forward(x, dt, A, b, c, lengths=lengths, checkpoint=True)
    want = S.sig_scan_forward(x, dt, A, b.contiguous(), c.contiguous(), lengths=lengths, checkpoint=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one, two = (S.sig_scan_backward(x, dt, A, bb, cc, x, got[2], lengths=lengths) for bb, cc in ((b, c), (b.contiguous(), c.contiguous())))
    for k in ("x", "dt", "A", "B", "C"):
        assert torch.equal(one[k], two[k]), k


def test_more_refusals_of_the_scan():
    lib = S.load_library()
    ok = dict.fromkeys(SCAN_ORDER, 0) | dict(dtype=0, B=2, L=40, D=4, G=2, N=4, softplus=1, x=4096, dt=4096, b=4096, c=4096, A=4096, gate=4096, skip=4096, bias=4096)
    args = pack(ok, SCAN_ORDER)
    ck = lib.sig_scan_checkpoint_bytes(args)
    assert ck == 2 * 3 * 4 * 4 * 4                                   # three tiles of 16 tokens
    big = 1 << 60
    assert lib.sig_scan_forward(args, 4096, 0, 4096, ck - 1, 4096, big, 0) == -5
    assert lib.sig_scan_forward(args, 0, 0, 0, 0, 4096, big, 0) == -1
    assert lib.sig_scan_forward(None, 4096, 0, 0, 0, 0, 0, 0) == -1
    every = dict.fromkeys(GRADS_ORDER, 4096)
    need = lib.sig_scan_backward_workspace_bytes(args)
    assert need > 0
    assert lib.sig_scan_backward(args, pack(every, GRADS_ORDER), 4096, ck - 1, 4096, need, 0) == -5
    assert lib.sig_scan_backward(args, pack(every, GRADS_ORDER), 0, ck, 4096, need, 0) == -5
    assert lib.sig_scan_backward(args, pack(every, GRADS_ORDER), 4096, ck, 4096, need - 1, 0) == -5
    assert lib.sig_scan_backward(args, pack(every, GRADS_ORDER), 4096, ck, 0, need, 0) == -5
    assert lib.sig_scan_backward(args, None, 4096, ck, 4096, need, 0) == -1
    for k in ("gy", "gx", "gdt", "gz", "gbb", "gcc", "gA", "gskip", "gbias"):
        assert lib.sig_scan_backward(args, pack({**every, k: 0}, GRADS_ORDER), 4096, ck, 4096, need, 0) == -1, k
    assert lib.sig_scan_step(args, 0, 4096, 0) == -1
    assert lib.sig_scan_checkpoint_bytes(None) == 0 and lib.sig_scan_backward_workspace_bytes(None) == 0


def test_clip_refuses_through_the_c_abi():
    lib = S.load_library()
    arr = lambda *v: (ctypes.c_int64 * len(v))(*v)                                          # noqa: E731
    ptr, one, f32, b16 = arr(4096), arr(100), arr(0), arr(1)
    call = lambda n=1, i=ptr, o=ptr, s=one, a=f32, b=f32, m=1.0, norm=4096, w=4096, nb=1 << 20: lib.sig_grad_clip(n, i, o, s, a, b, m, norm, w, nb, 0)   # noqa: E731
    assert call(n=-1) == -1 and call(i=None) == -1 and call(o=None) == -1 and call(s=None) == -1 and call(a=None) == -1 and call(b=None) == -1
    assert call(m=-1.0) == -1 and call(m=math.nan) == -1 and call(norm=0) == -1
    assert call(a=arr(2)) == -1 and call(b=arr(-1)) == -1 and call(s=arr(-5)) == -1 and call(i=arr(0)) == -1 and call(o=arr(0)) == -1
    assert call(b=b16) == -1                                          # in place needs one type
    assert call(s=arr(1 << 41)) == -7 and call(w=0) == -5 and call(nb=7) == -5
    assert lib.sig_grad_clip_workspace_bytes(1, one) == 8 and lib.sig_grad_clip_workspace_bytes(0, None) == 0


def test_host_tensors_are_refused():
    x, w, b, A = torch.zeros(2, 5, 8), torch.zeros(8, 4), torch.zeros(2, 5, 16), torch.zeros(8, 16)
    for f in (lambda: S.sig_conv_forward(x, w), lambda: S.sig_conv_step(x[:, 0], x[:, :3], w), lambda: S.sig_conv_backward(x, w, x),
              lambda: S.sig_scan_forward(x, x, A, b, b), lambda: S.sig_scan_step(x[:, 0], x[:, 0], A, b[:, 0], b[:, 0], torch.zeros(2, 8, 16)),
              lambda: S.sig_grad_clip([x], 1.0), lambda: S.sig_grad_clip([x], -1.0), lambda: S.sig_grad_clip([x], 1.0, out=[])):
        with pytest.raises(ValueError):
            f()


@gpu
def test_missing_states_are_refused():
    x, w, b, A = torch.zeros(2, 5, 8, device="cuda"), torch.zeros(8, 4, device="cuda"), torch.zeros(2, 5, 16, device="cuda"), torch.zeros(8, 16, device="cuda")
    for f in (lambda: S.sig_conv_step(x[:, 0], None, w), lambda: S.sig_scan_step(x[:, 0], x[:, 0], A, b[:, 0], b[:, 0], None),
              lambda: S.sig_scan_backward(x, x, A, b, b, x, None)):
        with pytest.raises(ValueError):
            f()


@gpu
def test_python_refusals():
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device="cuda")                 # noqa: E731
    x, w, b, A = z(2, 5, 8), z(8, 4), z(2, 5, 16), z(8, 16)
    h, ck = z(2, 8, 16), S.sig_scan_forward(x, x, A, b, b, checkpoint=True)[2]
    bad = [
        lambda: S.sig_conv_forward(x.half(), w), lambda: S.sig_conv_forward(x[0], w), lambda: S.sig_conv_forward(x, w.bfloat16()),
        lambda: S.sig_conv_forward(x, z(7, 4)), lambda: S.sig_conv_forward(x, z(8, 9)), lambda: S.sig_conv_forward(x, z(8)),
        lambda: S.sig_conv_forward(x, w, z(7)), lambda: S.sig_conv_forward(x, w, initial_state=z(2, 4, 8)),
        lambda: S.sig_conv_forward(x, w, lengths=z(2)), lambda: S.sig_conv_forward(x, w, lengths=z(3, t=torch.int32)),
        lambda: S.sig_conv_forward(x, w.cpu()), lambda: S.sig_conv_backward(x, w, z(2, 4, 8)), lambda: S.sig_conv_backward(x, w, x.bfloat16()),
        lambda: S.sig_conv_step(x[:, 0], z(2, 4, 8), w), lambda: S.sig_conv_step(x[:, 0], z(2, 8, 3).transpose(1, 2), w), lambda: S.sig_conv_step(x, z(2, 3, 8), w),
        lambda: S.sig_scan_forward(x, x.bfloat16(), A, b, b), lambda: S.sig_scan_forward(x, x, A.double(), b, b), lambda: S.sig_scan_forward(x, x, z(8, 15), b, b),
        lambda: S.sig_scan_forward(x, x, A, b, b[..., :15]), lambda: S.sig_scan_forward(x, x, A, z(2, 5, 3, 16), z(2, 5, 3, 16)),
        lambda: S.sig_scan_forward(x, x, z(8, 65), z(2, 5, 65), z(2, 5, 65)), lambda: S.sig_scan_forward(x, x, A, b, b, gate=z(2, 5, 7)),
        lambda: S.sig_scan_forward(x, x, A, b, b, initial_state=z(2, 8, 15)), lambda: S.sig_scan_forward(x, x, None, b, b),
        lambda: S.sig_scan_forward(x, x, A, b[0], b[0]), lambda: S.sig_scan_forward(x, x, A, b, b, skip=z(9)),
        lambda: S.sig_scan_backward(x, x, A, b, b, z(2, 5, 9), ck), lambda: S.sig_scan_backward(x, x, A, b, b, x, ck.cpu()),
        lambda: S.sig_scan_step(x[:, 0], x[:, 0], A, b[:, 0], b[:, 0], h.bfloat16()), lambda: S.sig_scan_step(x[:, 0], x[:, 0], A, b[:, 0], b[:, 0], z(2, 16, 8).transpose(1, 2)),
        lambda: S.sig_grad_clip([x.half()], 1.0), lambda: S.sig_grad_clip([x], math.nan), lambda: S.sig_grad_clip([x], 1.0, out=[z(5)]),
        lambda: S.sig_grad_clip([x[:, ::2]], 1.0), lambda: S.sig_grad_clip([x], 1.0, out=[x.cpu()]), lambda: S.sig_grad_clip([w], 1.0, out=[z(4, 8).t()]),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was taken")
    with pytest.raises(S.SigError):                                   # a checkpoint of another call's size
        S.sig_scan_backward(x, x, A, b, b, x, ck[:16])
