"""Operators of a layer (norm with residual and 8-bit output, matrix product with epilogue, gated recurrence) against plain 64-bit implementations.

Tolerances.  H = half a step of the output's type (float32 2^-24, bfloat16 2^-8, e4m3 2^-4, relative to the value).
Norm: sum, mean, root, three products: a handful of float32 roundings; sums over a row in float32 add at most 64 roundings in a row of the lengths here
(16 values of a thread, six lane steps, sixteen wavefronts): 2^-24 * 64 = 4e-6 relative to the sum of magnitudes, half of it for the root.
Products of whole numbers are exact in float32 as long as sums stay below 2^24, so those tests ask for equality.  Other products: K + 8 roundings of the
sum of magnitudes at most, in any order of summation.
Recurrence: as the scan's: norm-wise 1e-5 in float32, 2^-8 in bfloat16, single values 20 times that."""
import ctypes
import math

import pytest
import torch

import paper_2602_24066_amd as S
from tests import layer_reference as R
from tests.test_sequence import close, poison, up

gpu = pytest.mark.gpu
H = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F32, B16, E8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def normal(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g)


def within(got, want, slack, what):
    """|got - want| <= slack, entry by entry."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, f"{what}: shape {tuple(got.shape)} for {tuple(want.shape)}"
    over = (got - want).abs() - slack
    assert not torch.isnan(over).any() and (over <= 0).all(), f"{what}: {int((~(over <= 0)).sum())} of {over.numel()} entries too far off, by {float(over.max()):.3e}"


# ------------------------------------------------------------------------------------------------ norm
NORM = [(1, 1), (3, 7), (130, 30), (5, 64), (9, 333), (2, 340), (7, 512), (64, 1024), (5, 1554), (3, 2048), (2, 4104), (3, 5460), (2, 8192), (2, 16385), (1, 40000), (2, 65544)]


@gpu
@pytest.mark.parametrize("t", [F32, B16])
@pytest.mark.parametrize("rows,C", NORM)
@pytest.mark.parametrize("residual", [False, True])
def test_norm_and_its_gradient(rows, C, t, residual):
    n = normal(C)
    x, res, w, gy, gt = n(rows, C).to(t), (2 * n(rows, C)).to(t) if residual else None, 1 + 0.2 * n(C), n(rows, C).to(t), n(rows, C).to(t)
    y, total = S.sig_norm_forward(up(x), up(w), up(res))
    want_total = x if res is None else (x.float() + res.float()).to(t)                       # of two bfloat16 values float32 holds the sum, or rounds far below a half step
    assert torch.equal(total.cpu(), want_total)
    v = want_total.double().requires_grad_()
    w64 = w.double().requires_grad_()
    want = R.norm(v, w64)
    f = 2.0 ** -24
    within(y, want.detach(), H[t] * want.abs().detach() * 1.001 + 40 * f * want.abs().detach(), "y")
    for extra in (gt, None):
        gx, gw = S.sig_norm_backward(total, up(w), up(gy), up(extra))
        a, b = torch.autograd.grad(want, (v, w64), gy.double(), retain_graph=True)
        s = 1 / torch.sqrt((v.detach() ** 2).mean(-1, keepdim=True) + 1e-6)
        size = s * (gy.double() * w.double()).abs() + v.detach().abs() * s ** 3 * (gy.double() * w.double() * v.detach()).abs().mean(-1, keepdim=True)
        if extra is not None:
            a, size = a + extra.double(), size + extra.double().abs()
        within(gx, a, H[t] * 1.001 * a.abs() + 140 * f * size, "grad x")
        # sums over rows: one after the other in a thread, then over at most 16 + 512 parts
        within(gw, b, (rows + 64 + 40) * f * (gy.double() * v.detach() * s).abs().sum(0), "grad weight")


@gpu
@pytest.mark.parametrize("t", [F32, B16])
@pytest.mark.parametrize("rows,C", NORM)
def test_rows_in_8_bits(rows, C, t):
    n = normal(C + 1)
    x, res, w = n(rows, C).to(t), n(rows, C).to(t), 1 + 0.2 * n(C)
    for kind in ("norm", "norm of the sum", "rows"):
        if kind == "rows":
            q, scale = S.sig_quantize(up(x))
            want = x.double()
        else:
            total = x if kind == "norm" else (x.float() + res.float()).to(t)
            q, scale, got = S.sig_norm_forward(up(x), up(w), up(res) if kind != "norm" else None, quantize=True)
            assert torch.equal(got.cpu(), total)
            want = R.norm(total.double(), w.double())
        assert q.dtype is E8 and q.shape == x.shape and scale.dtype is F32 and scale.shape == (rows,)
        top = want.abs().amax(-1)
        within(scale, top / 448, 44 * 2.0 ** -24 * top / 448, kind + ": scale")
        # the value is off by the norm's roundings, then half a step: 2^-4 of it, or 2^-10 below the smallest normal value
        back = q.double().cpu() * scale.double().cpu()[:, None]
        within(back, want, want.abs() * (2.0 ** -4 + 60 * 2.0 ** -24) + scale.double().cpu()[:, None] * 2.0 ** -10 * 1.001, kind)
        # and it is the nearest: at most the few values whose quotient lies next to a border differ
        near = R.e4m3(want * (448 / top)[:, None])
        assert ((q.double().cpu() != near).double().mean() <= (0.02 if t is B16 else 0.001) + 1.5 / near.numel()), kind       # quotients of bfloat16 values lie on borders now and then


@gpu
def test_special_rows_in_8_bits():
    x = torch.zeros(8, 40)
    x[1, 3] = 1e-41                                          # values whose quotient by 448 float32 does not hold
    x[2, 5] = 2.0 ** -125
    x[3, 7] = 3.3e38
    x[4] = torch.linspace(-448, 448, 40)
    x[5, 0], x[5, 1] = math.nan, 1.0
    x[6, 0], x[6, 1] = math.inf, 1.0
    x[7] = 1e-37
    q, scale = S.sig_quantize(up(x))
    q, scale = q.double().cpu(), scale.double().cpu()
    assert (q[0] == 0).all() and scale[0] == 0
    for r in (1, 2, 3, 7):
        top = float(x[r].abs().max())
        back = q[r] * scale[r]
        assert torch.isfinite(back).all() and ((back - x[r].double()).abs() <= 2.0 ** -4 * x[r].double().abs() + scale[r] * 2.0 ** -10).all(), r
        assert top < 2.0 ** -119 or abs(float(scale[r]) * 448 / top - 1) < 1e-6
    assert torch.equal(q[4], R.e4m3(x[4].double())) and scale[4] == 1
    assert not math.isfinite(scale[5]) and not math.isfinite(scale[6])
    y, s, _ = S.sig_norm_forward(torch.zeros(3, 40, device="cuda"), torch.ones(40, device="cuda"), quantize=True)
    assert not y.float().any() and not s.any()


# ------------------------------------------------------------------------------------------------ matrix product
LINEAR = [
    # rows, inputs, outputs
    (1, 1, 1), (1, 30, 64), (3, 64, 5), (1, 2048, 1024), (17, 33, 18), (64, 2048, 100), (5, 5460, 333), (130, 258, 130), (128, 64, 128), (129, 129, 257),
    (16, 96, 8200), (20, 80, 8208), (64, 160, 8224), (40, 304, 33), (31, 16, 64), (65, 208, 130), (300, 1554, 340), (512, 512, 512), (1025, 96, 700), (2, 64, 4099), (4099, 7, 3), (33, 8200, 48),
]


def whole(seed, most=3):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randint(-most, most + 1, s, generator=g).float()


@gpu
@pytest.mark.parametrize("t", [F32, B16, E8])
@pytest.mark.parametrize("M,K,N", LINEAR)
def test_products_of_whole_numbers_are_exact(M, K, N, t):
    n = whole(M + K + N)
    out = B16 if t is E8 else t
    x, w, b, r = n(M, K).to(t), n(N, K).to(t), n(N).to(out), n(M, N).to(out)
    want = x.double() @ w.double().t()
    assert want.abs().max() < 2 ** 24
    d = {k: up(v) for k, v in dict(x=x, w=w, b=b, r=r).items()}
    assert torch.equal(S.sig_linear_forward(d["x"], d["w"]).cpu(), want.to(out))
    got, pre = S.sig_linear_forward(d["x"], d["w"], d["b"], d["r"], keep=True)
    assert pre is None and torch.equal(got.cpu(), (want + b.double() + r.double()).to(out))
    if t is E8:
        return
    g = n(M, N).to(t)
    gx, gw, gb = S.sig_linear_backward(d["x"], d["w"], up(g), bias=True)
    assert torch.equal(gx.cpu(), (g.double() @ w.double()).to(t))
    assert torch.equal(gw.cpu(), (g.double().t() @ x.double()).to(t))
    assert torch.equal(gb.cpu(), g.double().sum(0).to(t))
    one = S.sig_linear_backward(d["x"], d["w"], up(g), need_weight=False)
    assert torch.equal(one[0], gx) and one[1] is None and one[2] is None
    two = S.sig_linear_backward(d["x"], d["w"], up(g), need_x=False)
    assert two[0] is None and torch.equal(two[1], gw)


@gpu
@pytest.mark.parametrize("out", [F32, B16])
def test_scales_of_8_bit_products(out):
    M, K, N = 37, 200, 45
    n, m = whole(3), normal(4)
    x, w, b, r = n(M, K).to(E8), n(N, K).to(E8), m(N).to(out), m(M, N).to(out)
    sx, sw = m(M).abs() + 0.1, m(N).abs() + 0.1
    z = (x.double() @ w.double().t()) * sx.double()[:, None] * sw.double()
    for kw, want in ((dict(x_scale=sx, weight_scale=sw), z), (dict(x_scale=sx), z / sw.double()), (dict(weight_scale=sw), z / sx.double()[:, None]), ({}, z / sw.double() / sx.double()[:, None])):
        got = S.sig_linear_forward(up(x), up(w), up(b), up(r), dtype=out, **{k: up(v) for k, v in kw.items()})
        total = want + b.double() + r.double()
        within(got, total, H[out] * 1.001 * total.abs() + 6 * 2.0 ** -24 * (want.abs() + b.double().abs() + r.double().abs()), str(list(kw)))


@gpu
@pytest.mark.parametrize("activation", [None, "silu", "gelu"])
@pytest.mark.parametrize("t", [F32, B16])
@pytest.mark.parametrize("M,K,N", [(1, 30, 64), (37, 129, 70), (200, 333, 258), (3, 5460, 5)])
def test_product_with_activation_and_its_gradient(M, K, N, t, activation):
    n = normal(M * N + K)
    x, w, b, r, g = n(M, K).to(t), (n(N, K) / math.sqrt(K)).to(t), n(N).to(t), n(M, N).to(t), n(M, N).to(t)
    f = 2.0 ** -24
    z = x.double() @ w.double().t() + b.double()
    off = (K + 8) * f * (x.double().abs() @ w.double().abs().t() + b.double().abs())          # of z
    y, pre = S.sig_linear_forward(up(x), up(w), up(b), up(r), activation=activation, keep=True)
    want = R.act(z, activation) + r.double()
    # |f'| <= 1.13 for both; f itself by exponentials and erf of a few units, relative to z
    within(y, want, H[t] * 1.001 * want.abs() + 1.13 * off + 16 * f * (z.abs() + r.double().abs()), "y")
    p = 0.0
    s = torch.ones_like(z)
    if activation:
        within(pre, z, H[t] * 1.001 * z.abs() + off, "pre")
        p = H[t] * 1.001 * z.abs() + off
        s = R.slope(z, activation)
    gx, gw, gb = S.sig_linear_backward(up(x), up(w), up(g), activation, pre, bias=True)
    gz = g.double() * s
    # the slope changes by at most 0.8 of what z is off by, is off by some units itself, and the product is rounded to the tokens' type
    og = (g.double().abs() * (0.8 * p + 16 * f) + (H[t] * gz.abs() if activation else 0.0)) * 1.01
    for got, want, size, slack, k in ((gx, gz @ w.double(), gz.abs() @ w.double().abs(), og @ w.double().abs(), "x"),
                                      (gw, gz.t() @ x.double(), gz.t().abs() @ x.double().abs(), og.t() @ x.double().abs(), "weight"),
                                      (gb, gz.sum(0), gz.abs().sum(0), og.sum(0), "bias")):
        within(got, want, H[t] * 1.001 * (want.abs() + slack) + slack + (max(M, N) + 8) * f * size, "grad " + k)


@gpu
def test_activations_at_special_values():
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 5.0, -5.0, -12.0, 30.0, -30.0, 100.0, -100.0, 3e38, -3e38, math.inf, math.nan])
    one = torch.ones(1, 1, device="cuda")
    for name in ("silu", "gelu"):
        y, pre = S.sig_linear_forward(up(v)[:, None], one, activation=name, keep=True)
        y, want = y.double().cpu()[:, 0], R.act(v.double(), name)
        assert torch.equal(pre.cpu()[:-1, 0], v[:-1]) and torch.isnan(y[-1]) and math.isinf(y[-2])
        assert ((y - want).abs()[:-2] <= 2e-6 * want.abs()[:-2] + 1e-6 * (want.abs()[:-2] < 1e-3)).all(), name
        gx, _, _ = S.sig_linear_backward(up(v)[:, None], one, torch.ones(15, 1, device="cuda"), name, pre)
        slope = R.slope(v[:13].double(), name)
        slope[12] = 0.0                                      # far below zero, where the reference divides infinities
        assert ((gx.double().cpu()[:13, 0] - slope).abs() <= 1e-6).all(), name


# ------------------------------------------------------------------------------------------------ gated recurrence
GATED = [
    # B, L, D, type, carried state, lengths
    (2, 33, 64, F32, True, None), (2, 48, 64, B16, True, None), (3, 50, 37, F32, True, [50, 0, 17]), (2, 130, 130, B16, False, [128, 130]), (1, 1, 5, F32, True, None),
    (1, 15, 1, F32, False, None), (4, 300, 66, F32, True, [300, 129, -4, 999]), (1, 700, 70, B16, True, [641]), (1, 2050, 6, F32, True, None), (5, 16, 2, B16, True, [16, 15, 1, 0, 8]),
]


@gpu
@pytest.mark.parametrize("case", range(len(GATED)))
def test_gated_scan_and_its_gradient(case):
    B, L, D, t, carry, lengths = GATED[case]
    v = R.gated_inputs(B, L, D, t, carry, lengths, seed=case)
    n = normal(case + 50)
    gy, gs = n(B, L, D).to(t), n(B, D) if carry else None
    wide = {k: w.double().requires_grad_() if w is not None and w.is_floating_point() else w for k, w in v.items()}
    y, state = R.gated(**wide)
    loss = sum((y[b, :R._len(v["lengths"], b, L)] * gy[b, :R._len(v["lengths"], b, L)].double()).sum() for b in range(B))
    loss = loss if gs is None else loss + (state * gs.double()).sum()
    names = [k for k, w in wide.items() if w is not None and w.is_floating_point()]
    grads = dict(zip(names, torch.autograd.grad(loss, [wide[k] for k in names])))
    hidden = ["x", "decay_gate", "input_gate"]
    d = {k: up(w) for k, w in poison(v, hidden).items()}
    got_y, got_state, ck = S.sig_gated_scan_forward(**d, checkpoint=True)
    close(got_y, y, t, "y")
    close(got_state, state, F32, "state")
    again, _ = S.sig_gated_scan_forward(**d)
    assert torch.equal(again, got_y)
    gy = poison({"g": gy, "lengths": v["lengths"]}, ["g"])["g"]
    got = S.sig_gated_scan_backward(d["x"], d["decay_gate"], d["input_gate"], d["log_rate"], up(gy), ck, d["initial_state"], d["lengths"], up(gs))
    for k in names:
        close(got[k], grads[k], F32 if k in ("log_rate", "initial_state") else t, "grad " + k)
    assert (got["initial_state"] is None) == (not carry)


@gpu
@pytest.mark.parametrize("t,D", [(F32, 33), (B16, 64), (B16, 7)])
def test_gated_steps_continue_a_prompt(t, D):
    v = R.gated_inputs(3, 23, D, t, seed=5)
    y, state = R.gated(**{k: w.double() if w is not None else w for k, w in v.items()})
    d = {k: up(w) for k, w in v.items()}
    _, held = S.sig_gated_scan_forward(*(d[k][:, :9] for k in ("x", "decay_gate", "input_gate")), d["log_rate"], d["initial_state"])
    rows = [S.sig_gated_scan_step(*(d[k][:, i] for k in ("x", "decay_gate", "input_gate")), d["log_rate"], held) for i in range(9, 23)]
    close(torch.stack(rows, 1), y[:, 9:], t, "y")
    close(held, state, F32, "state")


@gpu
def test_gates_at_the_ends_of_their_range():
    """Gates that are shut or open all the way, rates from nearly nothing to more than exp holds: states, and gradients against the formula."""
    p = torch.tensor([-100.0, -40.0, -10.0, 0.0, 20.0, 200.0])
    rates = torch.tensor([-30.0, -3.0, 0.0, 4.0, 30.0, 90.0])
    D, L = 36, 7
    v = dict(x=normal(1)(1, L, D), decay_gate=p.repeat(6).expand(1, L, D).contiguous(), input_gate=normal(2)(1, L, D) * 30, log_rate=rates.repeat_interleave(6), initial_state=normal(3)(1, D))
    d = {k: up(w) for k, w in v.items()}
    y, state, ck = S.sig_gated_scan_forward(**d, checkpoint=True)
    wide = {k: w.double() for k, w in v.items()}
    wide["log_rate"] = wide["log_rate"].clamp(max=64.0)      # by definition
    leaves = {k: w.requires_grad_() for k, w in wide.items()}
    want, last = R.gated(**leaves)
    close(y, want, F32, "y")
    close(state, last, F32, "state")
    gy = normal(4)(1, L, D)
    grads = torch.autograd.grad((want * gy.double()).sum(), list(leaves.values()))
    got = S.sig_gated_scan_backward(d["x"], d["decay_gate"], d["input_gate"], d["log_rate"], up(gy), ck, d["initial_state"])
    for k, g in zip(leaves, grads):
        assert torch.isfinite(g).all(), k
        close(got[k], g, F32, "grad " + k)


# ------------------------------------------------------------------------------------------------ layouts, streams, graphs
@gpu
@pytest.mark.parametrize("t", [F32, B16])
def test_strided_broadcast_and_unaligned_tokens(t):
    n = normal(9)
    B, L, D, N = 3, 21, 40, 24
    wide, w, weight, bias = up(n(B, L, 3 * D + 5).to(t)), up(1 + 0.1 * n(D)), up(n(N, D).to(t)), up(n(N).to(t))
    row, grads = up(n(1, 1, D).to(t)), up(n(B, L, N + 3).to(t))
    views = [wide[..., :D], wide[..., D:2 * D], wide[..., 3:3 + D], wide[:, 1:2, 5:5 + D], wide[:, ::2, :D], row.expand(B, L, D), wide.transpose(0, 1)[..., :D], wide[0, :, 1:1 + D],
             wide[..., ::3][..., :D], wide[..., :D].flip(0)]
    for i, x in enumerate(views):
        c = x.contiguous()
        for f in (lambda v: S.sig_norm_forward(v, w)[0], lambda v: S.sig_norm_forward(c, w, v)[0], lambda v: S.sig_norm_forward(v, w, v)[1], lambda v: S.sig_quantize(v)[0].view(torch.uint8),
                  lambda v: S.sig_norm_backward(v, w, c)[0], lambda v: S.sig_norm_backward(c, w, v, v)[0], lambda v: S.sig_norm_backward(c, w, v)[1], lambda v: S.sig_linear_forward(v, weight, bias),
                  lambda v: S.sig_linear_backward(v, weight, grads[..., :N].expand(*v.shape[:-1], N) if v.dim() == 3 and v.shape[:2] == (B, L) else c[..., :N].contiguous())[1]):
            one, two = f(x), f(c)
            # an element-wise path adds in another order than one of wide accesses
            tol = 0 if one.dtype is torch.uint8 else (2.0 ** -7 if t is B16 else 1e-5) * float(two.abs().max())
            if one.dtype is torch.uint8:
                assert (one != two).double().mean() <= 0.02, i
            else:
                assert one.shape == two.shape and float((one.float() - two.float()).abs().max()) <= tol, i
    r = grads[..., 1:1 + N]
    x = views[0]
    assert torch.equal(S.sig_linear_forward(x, weight, residual=r), S.sig_linear_forward(x, weight, residual=r.contiguous()))
    rate = up(n(D))
    for x in views[:4] + views[5:7]:
        if x.dim() == 3:
            q = x.contiguous()
            one, two = S.sig_gated_scan_forward(x, x, x, rate, checkpoint=True), S.sig_gated_scan_forward(q, q, q, rate, checkpoint=True)
            assert all(torch.equal(a, b) for a, b in zip(one[:2], two[:2]))
            g1, g2 = S.sig_gated_scan_backward(x, x, x, rate, x, one[2]), S.sig_gated_scan_backward(q, q, q, rate, q, two[2])
            assert all(torch.equal(g1[k], g2[k]) for k in ("x", "decay_gate", "input_gate", "log_rate"))


@gpu
@pytest.mark.parametrize("t", [F32, B16])
def test_nothing_to_do(t):
    z = lambda *s: torch.zeros(*s, dtype=t, device="cuda")                                  # noqa: E731
    f = lambda *s: torch.full(s, 7.0, device="cuda")                                        # noqa: E731
    assert S.sig_norm_forward(z(0, 8), f(8), z(0, 8))[0].shape == (0, 8) and S.sig_norm_forward(z(2, 0, 8), f(8), quantize=True)[1].shape == (2, 0)
    gx, gw = S.sig_norm_backward(z(0, 3, 8), f(8), z(0, 3, 8))
    assert gx.shape == (0, 3, 8) and not gw.any()
    assert S.sig_quantize(z(0, 8))[1].shape == (0,)
    assert S.sig_linear_forward(z(0, 8), z(5, 8), z(5)).shape == (0, 5)
    gx, gw, gb = S.sig_linear_backward(z(0, 8), z(5, 8) + 1, z(0, 5), bias=True)
    assert gx.shape == (0, 8) and not gw.any() and not gb.any()
    state = f(2, 8)
    y, last, ck = S.sig_gated_scan_forward(z(2, 0, 8), z(2, 0, 8), z(2, 0, 8), f(8), state, checkpoint=True)
    assert y.shape == (2, 0, 8) and torch.equal(last, state)
    g = S.sig_gated_scan_backward(z(2, 0, 8), z(2, 0, 8), z(2, 0, 8), f(8), z(2, 0, 8), ck, state, grad_final_state=2 * state)
    assert torch.equal(g["initial_state"], 2 * state) and not g["log_rate"].any()
    y, last = S.sig_gated_scan_forward(z(0, 4, 8), z(0, 4, 8), z(0, 4, 8), f(8))
    assert y.shape == (0, 4, 8) and last.shape == (0, 8)
    assert not S.sig_gated_scan_backward(z(0, 4, 8), z(0, 4, 8), z(0, 4, 8), f(8), z(0, 4, 8), ck)["log_rate"].any()
    y, last = S.sig_gated_scan_forward(z(2, 5, 8) + 1, z(2, 5, 8), z(2, 5, 8), f(8), state, torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert not y.any() and torch.equal(last, state)


def layer(t, dev="cuda"):
    """A run of the operators as a layer uses them, forward and backward: f(inputs) -> outputs."""
    n = normal(21)
    B, L, D, E = 2, 70, 48, 96
    p = {k: v.to(dev) for k, v in dict(norm=1 + 0.1 * n(D), win=(n(3 * E, D) / 7).to(t), bin=(0.1 * n(3 * E)).to(t), conv=n(E, 4) / 2, rate=n(E) - 2, wout=(n(D, E) / 10).to(t)).items()}
    x, before = n(B, L, D).to(t).to(dev), n(B, L, D).to(t).to(dev)
    gy = n(B, L, D).to(t).to(dev)
    lens = torch.tensor([70, 33], dtype=torch.int32, device=dev)

    def run():
        h, total = S.sig_norm_forward(x, p["norm"], before)
        z, pre = S.sig_linear_forward(h, p["win"], p["bin"], activation="silu", keep=True)
        u, dg, ig = z.chunk(3, -1)
        v = S.sig_conv_forward(u, p["conv"], lengths=lens)
        s, last, ck = S.sig_gated_scan_forward(v, dg, ig, p["rate"], lengths=lens, checkpoint=True)
        y = S.sig_linear_forward(s, p["wout"], residual=total)
        gs, gwout, _ = S.sig_linear_backward(s, p["wout"], gy)
        g = S.sig_gated_scan_backward(v, dg, ig, p["rate"], gs, ck, lengths=lens)
        gu, gconv, _, _ = S.sig_conv_backward(u, p["conv"], g["x"], lengths=lens)
        gh, gwin, gbin = S.sig_linear_backward(h, p["win"], torch.cat([gu, g["decay_gate"], g["input_gate"]], -1), "silu", pre, bias=True)
        gx, gnorm = S.sig_norm_backward(total, p["norm"], gh, gy)
        return dict(y=y, last=last, x=gx, norm=gnorm, win=gwin, bin=gbin, conv=gconv, rate=g["log_rate"], wout=gwout)

    return run, p, x, before, gy, lens


def test_reference_layer_by_differences():
    """The oracle's own gradients, by differences (on the CPU)."""
    v = {k: w.double() for k, w in R.gated_inputs(1, 9, 3, seed=2).items() if w is not None}
    assert torch.autograd.gradcheck(lambda *a: R.gated(*a), [w.requires_grad_() for w in v.values()])
    z = torch.linspace(-6, 6, 41, dtype=torch.float64)
    for name in ("silu", "gelu"):
        assert ((R.act(z + 1e-5, name) - R.act(z - 1e-5, name)) / 2e-5 - R.slope(z, name)).abs().max() < 1e-8


@gpu
def test_a_layer_and_its_gradient():
    run, p, x, before, gy, lens = layer(F32)
    got = run()
    w = {k: v.double().cpu().requires_grad_() for k, v in p.items()}
    x64 = x.double().cpu().requires_grad_()
    total = x64 + before.double().cpu()
    z = R.norm(total, w["norm"]) @ w["win"].t() + w["bin"]
    u, dg, ig = R.act(z, "silu").chunk(3, -1)
    from tests import seq_reference as Q
    v, _ = Q.conv(u, w["conv"], lengths=lens.cpu())
    s, last = R.gated(v, dg, ig, w["rate"], lengths=lens.cpu())
    y = s @ w["wout"].t() + total
    grads = torch.autograd.grad((y * gy.double().cpu()).sum(), [x64, *w.values()])
    close(got["y"], y, F32, "y")
    close(got["last"], last, F32, "last")
    for k, g in zip(["x", *w], grads):
        close(got[k], g, F32, k)


@gpu
@pytest.mark.parametrize("t", [F32, B16])
def test_a_layer_on_streams_and_in_a_graph(t):
    run, p, x, before, gy, lens = layer(t)
    want = {k: v.clone() for k, v in run().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(got[k], want[k]) for k in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    keep = x.clone()
    for k in range(3):
        x.copy_(keep * (1 if k != 1 else 0.5))
        for v in held.values():
            v.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        fresh = run()
        assert all(torch.equal(held[j], fresh[j]) for j in fresh), k
        if k != 1:
            assert all(torch.equal(held[j], want[j]) for j in want), k


@gpu
def test_parameters_and_subclasses_give_plain_tensors():
    class Mine(torch.Tensor):
        pass

    x = torch.randn(2, 6, 16, device="cuda").as_subclass(Mine)
    w, m = torch.nn.Parameter(torch.ones(16, device="cuda")), torch.nn.Parameter(torch.randn(8, 16, device="cuda"))
    q, s = S.sig_quantize(x)
    outs = [S.sig_norm_forward(x, w)[0], *S.sig_norm_backward(x, w, x), q, s, S.sig_linear_forward(x, m), *S.sig_linear_backward(x, m, x[..., :8])[:2],
            *S.sig_gated_scan_forward(x, x, x, w), S.sig_gated_scan_step(x[:, 0], x[:, 0], x[:, 0], w, torch.zeros(2, 16, device="cuda"))]
    assert all(type(v) is torch.Tensor and not v.requires_grad for v in outs)


# ------------------------------------------------------------------------------------------------ refusals
BIG = 1 << 60
NORM_OK = dict(dtype=0, rows=4, C=8, xs=8, rs=8, eps=1e-6, x=4096, residual=4096, weight=4096)
LINEAR_ORDER = "dtype out M N K act xs rs x weight bias residual xscale wscale".split()
LINEAR_OK = dict.fromkeys(LINEAR_ORDER, 0) | dict(dtype=1, out=1, M=4, N=8, K=8, xs=8, rs=8, x=4096, weight=4096)
GATED_ORDER = "dtype B L D xb xt db dt ib it x decay input rate initial lengths".split()
GATED_OK = dict.fromkeys(GATED_ORDER, 0) | dict(dtype=0, B=2, L=40, D=4, x=4096, decay=4096, input=4096, rate=4096)
GATED_GRADS = "gb gt gy gfinal gx gd gi grate ginitial".split()


def norm_args(**change):
    import struct
    v = {**NORM_OK, **change}
    return struct.pack("5qd3q", v["dtype"], v["rows"], v["C"], v["xs"], v["rs"], v["eps"], v["x"], v["residual"], v["weight"])


def pack(fields, order):
    return (ctypes.c_int64 * len(order))(*[int(fields[k]) for k in order])


@pytest.mark.parametrize("change,code", [({"dtype": 2}, -1), ({"rows": -1}, -1), ({"C": 0}, -1), ({"xs": -1}, -1), ({"eps": -1.0}, -1), ({"eps": math.nan}, -1), ({"eps": math.inf}, -1),
                                         ({"x": 0}, -1), ({"weight": 0}, -1), ({"rows": 1 << 40}, -7), ({"xs": 1 << 40}, -7), ({"rows": 1 << 36}, -7), ({"rows": 0}, 0)])
def test_norm_refuses_through_the_c_abi(change, code):
    """Every refusal comes before anything touches the device (the pointers here lead nowhere)."""
    lib = S.load_library()
    assert lib.sig_norm_forward(norm_args(**change), 4096, 0, 4096, 0) == code
    if "rows" not in change:
        assert lib.sig_norm_backward(norm_args(**change), 4096, 8, 0, 0, 4096, 4096, 4096, BIG, 0) == code
    if not {"eps", "weight"} & set(change):
        v = {**NORM_OK, **change}
        assert lib.sig_quantize(v["dtype"], v["rows"], v["C"], v["xs"], v["x"], 4096, 4096, 0) == code


def test_more_refusals_of_the_norm():
    lib = S.load_library()
    a = norm_args()
    assert lib.sig_norm_forward(None, 4096, 0, 4096, 0) == -1 and lib.sig_norm_forward(a, 0, 0, 4096, 0) == -1
    assert lib.sig_norm_forward(norm_args(residual=0), 4096, 0, 4096, 0) == -1              # a total without a residual is x itself
    assert lib.sig_quantize(0, 4, 8, 8, 4096, 0, 4096, 0) == -1 and lib.sig_quantize(0, 4, 8, 8, 4096, 4096, 0, 0) == -1
    need = lib.sig_norm_backward_workspace_bytes(a)
    assert need > 0 and lib.sig_norm_backward_workspace_bytes(None) == 0
    call = lambda gy=4096, ys=8, ts=8, gx=4096, gw=4096, w=4096, n=need: lib.sig_norm_backward(a, gy, ys, 4096, ts, gx, gw, w, n, 0)   # noqa: E731
    assert call(gy=0) == -1 and call(gx=0) == -1 and call(gw=0) == -1 and call(ys=-1) == -1 and call(ts=-8) == -1 and call(w=0) == -5 and call(n=need - 1) == -5


@pytest.mark.parametrize("change,code", [({"dtype": 3}, -1), ({"dtype": 0}, -1), ({"out": 2}, -1), ({"M": -1}, -1), ({"N": 0}, -1), ({"K": 0}, -1), ({"act": 3}, -1), ({"act": -1}, -1),
                                         ({"xs": -1}, -1), ({"rs": -2}, -1), ({"x": 0}, -1), ({"weight": 0}, -1), ({"xscale": 4096}, -1), ({"wscale": 4096}, -1), ({"M": 1 << 31}, -7),
                                         ({"N": 1 << 31}, -7), ({"K": 1 << 31}, -7), ({"M": 1 << 30, "N": 1 << 20}, -7), ({"xs": 1 << 40}, -7), ({"M": 0}, 0)])
def test_linear_refuses_through_the_c_abi(change, code):
    lib = S.load_library()
    a = pack({**LINEAR_OK, **change}, LINEAR_ORDER)
    assert lib.sig_linear_forward(a, 4096, 0, 4096, BIG, 0) == code
    if not {"out", "rs", "xscale", "wscale", "M"} & set(change) and change != {"dtype": 0}:
        assert lib.sig_linear_backward(a, 4096, 8, 4096, 4096, 4096, 4096, 4096, BIG, 0) == code


def test_more_refusals_of_the_linear():
    lib = S.load_library()
    a = pack(LINEAR_OK, LINEAR_ORDER)
    assert lib.sig_linear_forward(None, 4096, 0, 4096, BIG, 0) == -1 and lib.sig_linear_forward(a, 0, 0, 4096, BIG, 0) == -1
    long = pack({**LINEAR_OK, "M": 100, "K": 1 << 16, "xs": 1 << 16}, LINEAR_ORDER)
    need = lib.sig_linear_forward_workspace_bytes(long)
    assert need > 0 and lib.sig_linear_forward(long, 4096, 0, 4096, need - 1, 0) == -5 and lib.sig_linear_forward(long, 4096, 0, 0, need, 0) == -5
    need = lib.sig_linear_backward_workspace_bytes(a)
    assert need > 0
    call = lambda v=a, gy=4096, gs=8, pre=4096, w=4096, n=need: lib.sig_linear_backward(v, gy, gs, pre, 4096, 4096, 4096, w, n, 0)     # noqa: E731
    assert call(gy=0) == -1 and call(gs=-1) == -1 and call(w=0) == -5 and call(n=need - 1) == -5 and call(v=None) == -1
    assert call(v=pack({**LINEAR_OK, "act": 1}, LINEAR_ORDER), pre=0, n=BIG) == -1
    assert call(v=pack({**LINEAR_OK, "dtype": 2}, LINEAR_ORDER), n=BIG) == -1               # 8-bit products have no gradient
    assert lib.sig_linear_forward_workspace_bytes(None) == 0 and lib.sig_linear_backward_workspace_bytes(None) == 0


@pytest.mark.parametrize("change,code", [({"dtype": 2}, -1), ({"B": -1}, -1), ({"L": -1}, -1), ({"D": 0}, -1), ({"x": 0}, -1), ({"decay": 0}, -1), ({"input": 0}, -1), ({"rate": 0}, -1),
                                         ({"xb": -1}, -1), ({"dt": -1}, -1), ({"it": 1 << 22}, -7), ({"D": 1 << 22}, -7), ({"L": 1 << 30}, -7), ({"B": 1 << 30}, -7), ({"B": 0}, 0)])
def test_gated_scan_refuses_through_the_c_abi(change, code):
    lib = S.load_library()
    a = pack({**GATED_OK, **change}, GATED_ORDER)
    assert lib.sig_gated_scan_forward(a, 4096, 4096, 4096, BIG, 4096, BIG, 0) == code
    if not {"L", "dt", "it"} & set(change):
        assert lib.sig_gated_scan_step(a, 4096, 4096, 0) == code
    if change != {"B": 0}:
        assert lib.sig_gated_scan_backward(a, pack(dict.fromkeys(GATED_GRADS, 4096), GATED_GRADS), 4096, BIG, 4096, BIG, 0) == code


def test_more_refusals_of_the_gated_scan():
    lib = S.load_library()
    a = pack(GATED_OK, GATED_ORDER)
    ck = lib.sig_gated_scan_checkpoint_bytes(a)
    assert ck == 2 * 3 * 4 * 4                                       # three tiles of 16 tokens
    assert lib.sig_gated_scan_forward(a, 0, 0, 0, 0, 4096, BIG, 0) == -1 and lib.sig_gated_scan_forward(None, 4096, 0, 0, 0, 0, 0, 0) == -1
    assert lib.sig_gated_scan_forward(a, 4096, 0, 4096, ck - 1, 4096, BIG, 0) == -5
    every = dict.fromkeys(GATED_GRADS, 4096)
    need = lib.sig_gated_scan_backward_workspace_bytes(a)
    call = lambda g=every, c=4096, cb=ck, w=4096, n=need: lib.sig_gated_scan_backward(a, None if g is None else pack(g, GATED_GRADS), c, cb, w, n, 0)   # noqa: E731
    assert need > 0 and call(cb=ck - 1) == -5 and call(c=0) == -5 and call(w=0) == -5 and call(n=need - 1) == -5 and call(g=None) == -1
    for k in ("gy", "gx", "gd", "gi", "grate"):
        assert call({**every, k: 0}) == -1, k
    assert call({**every, "gt": -1}) == -1 and call({**every, "gt": 1 << 22}) == -7 and call({**every, "gb": -1}) == -1
    assert lib.sig_gated_scan_step(a, 0, 4096, 0) == -1 and lib.sig_gated_scan_step(a, 4096, 0, 0) == -1
    assert lib.sig_gated_scan_checkpoint_bytes(None) == 0 and lib.sig_gated_scan_backward_workspace_bytes(None) == 0
    long = pack({**GATED_OK, "B": 1, "L": 1 << 16}, GATED_ORDER)
    need = lib.sig_gated_scan_forward_workspace_bytes(long)
    assert need > 0 and lib.sig_gated_scan_forward(long, 4096, 0, 0, 0, 4096, need - 1, 0) == -5


def test_host_tensors_are_refused():
    x, w, m = torch.zeros(2, 5, 8), torch.zeros(8), torch.zeros(4, 8)
    for f in (lambda: S.sig_norm_forward(x, w), lambda: S.sig_norm_backward(x, w, x), lambda: S.sig_quantize(x), lambda: S.sig_linear_forward(x, m),
              lambda: S.sig_linear_backward(x, m, x[..., :4]), lambda: S.sig_gated_scan_forward(x, x, x, w), lambda: S.sig_gated_scan_step(x[:, 0], x[:, 0], x[:, 0], w, x[:, 0])):
        with pytest.raises(ValueError):
            f()


@gpu
def test_python_refusals():
    z = lambda *s, t=F32: torch.zeros(*s, dtype=t, device="cuda")                           # noqa: E731
    x, w, m, b = z(2, 5, 8), z(8), z(4, 8), z(4)
    x8, m8 = x.to(E8), m.to(E8)
    h, ck = z(2, 8), S.sig_gated_scan_forward(x, x, x, w, checkpoint=True)[2]
    bad = [
        lambda: S.sig_norm_forward(x.half(), w), lambda: S.sig_norm_forward(x[0, 0], w), lambda: S.sig_norm_forward(x, w.bfloat16()), lambda: S.sig_norm_forward(x, z(7)),
        lambda: S.sig_norm_forward(x, w, x[:, :4]), lambda: S.sig_norm_forward(x, w, x.bfloat16()), lambda: S.sig_norm_forward(x, w, eps=-1.0), lambda: S.sig_norm_forward(x, w, eps=math.nan),
        lambda: S.sig_norm_forward(x, w.cpu()), lambda: S.sig_norm_forward(z(2, 0), z(0)), lambda: S.sig_norm_backward(x, w, x[..., :7]), lambda: S.sig_norm_backward(x, w, x, x.bfloat16()),
        lambda: S.sig_quantize(x8), lambda: S.sig_quantize(x[0, 0]),
        lambda: S.sig_linear_forward(x, m.bfloat16()), lambda: S.sig_linear_forward(x, z(4, 7)), lambda: S.sig_linear_forward(x, m, z(5)), lambda: S.sig_linear_forward(x, m, b.bfloat16()),
        lambda: S.sig_linear_forward(x, m, residual=z(2, 5, 5)), lambda: S.sig_linear_forward(x, m, activation="relu"), lambda: S.sig_linear_forward(x, m, activation=["silu"]),
        lambda: S.sig_linear_forward(x, m, x_scale=z(2, 5)), lambda: S.sig_linear_forward(x, m, dtype=B16), lambda: S.sig_linear_forward(x8, m8, dtype=torch.float16),
        lambda: S.sig_linear_forward(x8, m), lambda: S.sig_linear_forward(x8, m8, x_scale=z(2, 4)), lambda: S.sig_linear_forward(x8, m8, weight_scale=z(5)), lambda: S.sig_linear_forward(x8, m8, b),
        lambda: S.sig_linear_forward(x, z(8)), lambda: S.sig_linear_forward(z(2, 0), z(4, 0)), lambda: S.sig_linear_backward(x, m, z(2, 5, 5)), lambda: S.sig_linear_backward(x, m, z(2, 5, 4), "silu"),
        lambda: S.sig_linear_backward(x, m, z(2, 5, 4), "silu", z(2, 5, 5)), lambda: S.sig_linear_backward(x8, m8, z(2, 5, 4)),
        lambda: S.sig_gated_scan_forward(x, x, x.bfloat16(), w), lambda: S.sig_gated_scan_forward(x[0], x[0], x[0], w), lambda: S.sig_gated_scan_forward(x, x[:, :4], x, w),
        lambda: S.sig_gated_scan_forward(x, x, x, z(7)), lambda: S.sig_gated_scan_forward(x, x, x, w, z(2, 7)), lambda: S.sig_gated_scan_forward(x, x, x, w, lengths=z(2)),
        lambda: S.sig_gated_scan_backward(x, x, x, w, z(2, 5, 7), ck), lambda: S.sig_gated_scan_backward(x, x, x, w, x, None), lambda: S.sig_gated_scan_backward(x, x, x, w, x, ck.cpu()),
        lambda: S.sig_gated_scan_step(x[:, 0], x[:, 0], x[:, 0], w, None), lambda: S.sig_gated_scan_step(x[:, 0], x[:, 0], x[:, 0], w, h.bfloat16()),
        lambda: S.sig_gated_scan_step(x, x, x, w, h), lambda: S.sig_gated_scan_step(x[:, 0], x[:, 0], x[:, 0], w, z(8, 2).t()),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was taken")
    with pytest.raises(S.SigError):                                   # a checkpoint of another call's size
        S.sig_gated_scan_backward(x, x, x, w, x, ck[:16])
