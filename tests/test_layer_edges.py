"""Operators of a layer where they can go wrong: large tiles and every path of the matrix product, values next to what counts, far offsets, gradients by
differences, special values that stay in their rows.  Whole numbers are exact in float32, so products of them are compared for equality; other tolerances are
stated where they are used."""
import math

import pytest
import torch

import paper_2602_24066_amd as S
from tests import layer_reference as R
from tests import test_layer as L
from tests.test_layer import B16, E8, F32, H, normal, whole, within
from tests.test_sequence import close, up

gpu = pytest.mark.gpu


def product(x, w, *more):
    """x w^T in float64 on the GPU by slices of the contraction, of whole numbers, exact; more: added."""
    out = torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64, device="cuda")
    for k in range(0, x.shape[1], 256):
        out += x[:, k:k + 256].float().double() @ w[:, k:k + 256].float().double().t()
    for m in more:
        out += m.double()
    return out


@gpu
@pytest.mark.parametrize("t", [F32, B16, E8])
@pytest.mark.parametrize("M,K,N", [(4099, 1040, 4096), (4096, 1040, 4100), (2500, 4112, 2050), (300, 16400, 70), (65, 16384, 64), (700, 40, 9000), (4100, 523, 2100), (130, 2056, 515)])
def test_tiles_and_splits(M, K, N, t):
    """Tiles of every size, their edges along all three sides, splits of the contraction, rows that are no multiples of 16 bytes; epilogues with everything."""
    n = whole(M + N, 2)
    out = B16 if t is E8 else t
    x, w, b, r = up(n(M, K).to(t)), up(n(N, K).to(t)), up(n(N).to(out)), up(n(M, N).to(out))
    want = product(x, w, b, r)
    assert torch.equal(S.sig_linear_forward(x, w, b, r), want.to(out))
    if t is not E8:
        g = up(whole(K, 2)(M, N).to(t))
        gx, gw, gb = S.sig_linear_backward(x, w, g, bias=True)
        assert torch.equal(gx, product(g, w.t().contiguous()).to(t))
        assert torch.equal(gw, product(g.t().contiguous(), x.t().contiguous()).to(t))
        assert torch.equal(gb, g.double().sum(0).to(t))


@gpu
@pytest.mark.parametrize("t", [F32, B16, E8])
@pytest.mark.parametrize("M", [3, 40, 64, 70, 300])
@pytest.mark.parametrize("K,pad", [(64, 16), (80, 16), (208, 48), (33, 3), (100, 1)])
def test_what_lies_beside_the_rows_is_not_used(M, K, pad, t):
    """NaN behind the end of every row, behind the last row and before the first: a sum that takes one of them is NaN."""
    n, N = whole(M + K, 3), 90
    nan = lambda v: v.to(t) if t is not E8 else v.to(t)                                      # noqa: E731
    big = torch.full((M + 2, K + pad), math.nan)
    big[1:M + 1, :K] = n(M, K)
    weights = torch.full((N + 2, K), math.nan)
    weights[1:N + 1] = n(N, K)
    x, w = up(nan(big))[1:M + 1, :K], up(nan(weights))[1:N + 1]
    out = B16 if t is E8 else t
    want = product(x, w)
    assert torch.equal(S.sig_linear_forward(x, w), want.to(out))
    edge = torch.full((M, N + 3), math.nan)
    edge[:, :N] = n(M, N)
    r = up(edge.to(out))[:, :N]
    assert torch.equal(S.sig_linear_forward(x, w, residual=r), (want + r.double()).to(out))
    if t is not E8:
        g = r
        gx, gw, gb = S.sig_linear_backward(x, w, g, bias=True)
        assert torch.equal(gx, product(g, w.t().contiguous()).to(t)) and torch.equal(gw, product(g.t().contiguous(), x.t().contiguous()).to(t))
        assert torch.equal(gb, g.double().sum(0).to(t))
    if t is not E8:
        y, _ = S.sig_norm_forward(x, torch.ones(K, device="cuda"), x)
        assert torch.isfinite(y).all() and torch.equal(y, S.sig_norm_forward(x.contiguous(), torch.ones(K, device="cuda"), x.contiguous())[0])


@gpu
@pytest.mark.parametrize("t", [F32, B16])
def test_outputs_end_where_they_end(t):
    """Rows behind the outputs stay as they were (through the C ABI, into one larger buffer)."""
    from tests.test_layer import GATED_ORDER, LINEAR_ORDER, norm_args, pack
    lib, kind = S.load_library(), 0 if t is F32 else 1
    stream = torch.cuda.current_stream().cuda_stream
    for M, K, N in ((5, 48, 33), (70, 64, 40), (300, 128, 130)):
        x, w = torch.ones(M, K, dtype=t, device="cuda"), torch.ones(N, K, dtype=t, device="cuda")
        y = torch.full((M * N + 64,), 7.0, dtype=t, device="cuda")
        a = pack(dict.fromkeys(LINEAR_ORDER, 0) | dict(dtype=kind, out=kind, M=M, N=N, K=K, xs=K, x=x.data_ptr(), weight=w.data_ptr()), LINEAR_ORDER)
        ws = torch.empty(lib.sig_linear_forward_workspace_bytes(a) + 1, dtype=torch.uint8, device="cuda")
        assert lib.sig_linear_forward(a, y.data_ptr(), 0, ws.data_ptr(), ws.numel(), stream) == 0
        assert (y[:M * N] == K).all() and (y[M * N:] == 7).all()
        z = torch.full((M * K + 64,), 7.0, dtype=t, device="cuda")
        ones = torch.ones(K, device="cuda")
        assert lib.sig_norm_forward(norm_args(dtype=kind, rows=M, C=K, xs=K, rs=0, x=x.data_ptr(), residual=0, weight=ones.data_ptr()), z.data_ptr(), 0, 0, stream) == 0
        assert ((z[:M * K] - 1).abs() < 1e-2).all() and (z[M * K:] == 7).all()
    for B, L, D in ((1, 130, 6), (2, 17, 33)):
        x, rate = torch.ones(B, L, D, dtype=t, device="cuda"), torch.zeros(D, device="cuda")
        y = torch.full((B * L * D + 256,), 7.0, dtype=t, device="cuda")
        lens = torch.tensor([L] + [3] * (B - 1), dtype=torch.int32, device="cuda")
        p = x.data_ptr()
        a = pack(dict(dtype=kind, B=B, L=L, D=D, xb=L * D, xt=D, db=L * D, dt=D, ib=L * D, it=D, x=p, decay=p, input=p, rate=rate.data_ptr(), initial=0, lengths=lens.data_ptr()), GATED_ORDER)
        ws = torch.empty(lib.sig_gated_scan_forward_workspace_bytes(a) + 1, dtype=torch.uint8, device="cuda")
        assert lib.sig_gated_scan_forward(a, y.data_ptr(), 0, 0, 0, ws.data_ptr(), ws.numel(), stream) == 0
        got = y[:B * L * D].reshape(B, L, D)
        assert (got[0] > 0).all() and (got[1:, :3] > 0).all() and not got[1:, 3:].any() and (y[B * L * D:] == 7).all()


@gpu
def test_offsets_beyond_32_bits():
    """Rows and streams that lie gigabytes apart."""
    far = 1 << 30
    held = torch.zeros(3 * far + 64, dtype=B16, device="cuda")
    x = held.as_strided((3, 48), (far, 1))
    x.copy_(whole(5, 3)(3, 48))
    near, w, ones = x.clone(), up(whole(6, 3)(40, 48).to(B16)), torch.ones(48, device="cuda")
    assert torch.equal(S.sig_linear_forward(x, w), S.sig_linear_forward(near, w))
    assert torch.equal(S.sig_norm_forward(x, ones, x)[0], S.sig_norm_forward(near, ones, near)[0])
    assert torch.equal(S.sig_quantize(x)[1], S.sig_quantize(near)[1])
    g = up(whole(7, 3)(3, 40).to(B16))
    assert torch.equal(S.sig_linear_backward(x, w, g)[1], S.sig_linear_backward(near, w, g)[1])
    s = held.as_strided((3, 8, 6), (far, 6, 1))
    s.copy_(normal(8)(3, 8, 6))
    c, rate = s.clone(), torch.zeros(6, device="cuda")
    one, two = S.sig_gated_scan_forward(s, s, s, rate, checkpoint=True), S.sig_gated_scan_forward(c, c, c, rate, checkpoint=True)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    assert torch.equal(S.sig_gated_scan_backward(s, s, s, rate, s, one[2])["x"], S.sig_gated_scan_backward(c, c, c, rate, c, two[2])["x"])
    time = held.as_strided((1, 5, 6), (0, 1 << 22, 1))                                       # beyond the kernels' reach: copied
    time.copy_(normal(9)(1, 5, 6))
    c = time.clone()
    assert torch.equal(S.sig_gated_scan_forward(time, time, time, rate)[0], S.sig_gated_scan_forward(c, c, c, rate)[0])
    time = held.as_strided((1, 300, 6), (0, (1 << 22) - 2, 1))                               # just within it
    time.copy_(normal(10)(1, 300, 6))
    c = time.clone()
    one, two = S.sig_gated_scan_forward(time, time, time, rate, checkpoint=True), S.sig_gated_scan_forward(c, c, c, rate, checkpoint=True)
    assert torch.equal(one[0], two[0])
    g1, g2 = S.sig_gated_scan_backward(time, time, time, rate, time, one[2]), S.sig_gated_scan_backward(c, c, c, rate, c, two[2])
    assert all(torch.equal(g1[k], g2[k]) for k in ("x", "decay_gate", "input_gate", "log_rate"))


@gpu
def test_more_than_32_bits_of_outputs():
    M, N, K = (1 << 16) + 3, (1 << 15) + 8, 16
    x, w = up(whole(1, 3)(M, K).to(B16)), up(whole(2, 3)(N, K).to(B16))
    y = S.sig_linear_forward(x, w)
    for rows in (slice(0, 300), slice(M - 300, M), slice(40000, 40100)):
        assert torch.equal(y[rows], product(x[rows], w).to(B16))
    del y
    rows, C = (1 << 20) + 1, 2056
    v = torch.ones(rows, C, dtype=B16, device="cuda")
    v[-1] = 2.0
    y, _ = S.sig_norm_forward(v, torch.ones(C, device="cuda"))
    assert ((y[-5:] - 1).abs() < 1e-2).all() and ((y[:5] - 1).abs() < 1e-2).all() and float(y.float().min()) > 0.99


@gpu
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("t", [F32, B16])
def test_values_that_are_not_finite_stay_in_their_rows(t, bad):
    n = normal(3)
    for M, K, N in ((9, 64, 40), (130, 96, 70), (130, 97, 70), (600, 520, 600)):
        x, w = up(n(M, K).to(t)), up(n(N, K).to(t))
        clean = S.sig_linear_forward(x, w)
        y0, _ = S.sig_norm_forward(x, torch.ones(K, device="cuda"))
        x[4, 5] = bad
        got = S.sig_linear_forward(x, w)
        keep = [i for i in range(M) if i != 4]
        assert torch.equal(got[keep], clean[keep]) and not torch.isfinite(got[4]).all()
        y, _ = S.sig_norm_forward(x, torch.ones(K, device="cuda"))
        assert torch.equal(y[keep], y0[keep])
    x = up(n(3, 200, 10).to(t))
    rate = torch.zeros(10, device="cuda")
    clean = S.sig_gated_scan_forward(x, x, x, rate)[0]
    x[1, 50, 4] = bad
    got, _, ck = S.sig_gated_scan_forward(x, x, x, rate, checkpoint=True)
    same = torch.ones_like(got, dtype=torch.bool)
    same[1, 50:, 4] = False
    assert torch.equal(got[same], clean[same]) and not torch.isfinite(got[1, 50, 4])
    g = S.sig_gated_scan_backward(x, x, x, rate, clean, ck)
    for k in ("x", "decay_gate", "input_gate"):
        assert torch.isfinite(g[k][[0, 2]]).all() and torch.isfinite(g[k][1][:, [0, 1, 2, 3, 5, 6, 7, 8, 9]]).all(), k


@gpu
def test_gradients_that_are_not_finite_leave_hidden_tokens_zero():
    B, L, D = 2, 150, 6
    x, rate = torch.randn(B, L, D, device="cuda"), torch.zeros(D, device="cuda")
    lens = torch.tensor([3, 140], dtype=torch.int32, device="cuda")
    _, _, ck = S.sig_gated_scan_forward(x, x, x, rate, lengths=lens, checkpoint=True, initial_state=torch.zeros(B, D, device="cuda"))
    for bad in (math.nan, math.inf):
        last = torch.full((B, D), bad, device="cuda")
        last[1] = 0.0
        g = S.sig_gated_scan_backward(x, x, x, rate, x, ck, torch.zeros(B, D, device="cuda"), lens, last)
        for k in ("x", "decay_gate", "input_gate"):
            assert not g[k][0, 3:].any() and not g[k][1, 140:].any() and torch.isfinite(g[k][1]).all() and not torch.isfinite(g[k][0, :3]).all(), k


def differences(f, leaves, grads, what):
    """The slope of f along a random direction of every leaf by central differences of the kernels' own float32 outputs, against the gradient.  f is summed in
    float64; steps of 2^-7 leave errors of the third order below 1e-3 of values around one and of rounding below 1e-4."""
    for k, v in leaves.items():
        d = up(normal(len(k))(*v.shape)) if v.dim() else None
        h = 2.0 ** -7
        a, b = (f({**leaves, k: v + s * h * d}) for s in (1, -1))
        want, got = float(a - b) / (2 * h), float((grads[k].double() * d.double()).sum())
        size = float((grads[k].double().square().sum() * d.double().square().mean()).sqrt())
        assert abs(got - want) <= 5e-3 * max(abs(want), size), f"{what}: {k}: {got} for {want}"


@gpu
def test_gradients_are_slopes():
    n = normal(12)
    x, w, m, b, gy, gt = up(n(7, 40)), up(1 + 0.2 * n(40)), up(n(24, 40) / 6), up(0.3 * n(24)), up(n(7, 24)), up(n(7, 40))
    f = lambda v: (S.sig_norm_forward(v["x"], v["w"])[0].double() * gt.double()).sum()      # noqa: E731
    gx, gw = S.sig_norm_backward(x, w, gt)
    differences(f, {"x": x, "w": w}, {"x": gx, "w": gw}, "norm")
    for act in ("silu", "gelu"):
        f = lambda v: (S.sig_linear_forward(v["x"], v["m"], v["b"], activation=act).double() * gy.double()).sum()   # noqa: E731
        _, pre = S.sig_linear_forward(x, m, b, activation=act, keep=True)
        gx, gm, gb = S.sig_linear_backward(x, m, gy, act, pre, bias=True)
        differences(f, {"x": x, "m": m, "b": b}, {"x": gx, "m": gm, "b": gb}, act)
    v = {k: up(t) for k, t in R.gated_inputs(2, 40, 9, seed=4).items() if t is not None}
    go, gs = up(n(2, 40, 9)), up(n(2, 9))

    def g(v):
        y, s = S.sig_gated_scan_forward(**v)
        return (y.double() * go.double()).sum() + (s.double() * gs.double()).sum()

    _, _, ck = S.sig_gated_scan_forward(**v, checkpoint=True)
    grads = S.sig_gated_scan_backward(v["x"], v["decay_gate"], v["input_gate"], v["log_rate"], go, ck, v["initial_state"], grad_final_state=gs)
    differences(g, v, grads, "gated scan")


@gpu
@pytest.mark.parametrize("L", [127, 128, 129, 1000, 4097])
@pytest.mark.parametrize("t", [F32, B16])
def test_chunks_of_long_streams(L, t):
    """Few streams of any length: time chunks, against the same recurrence token by token (the single-token calls)."""
    B, D = 2, 70
    v = {k: up(w) for k, w in R.gated_inputs(B, L, D, t, seed=L, rate=0.02).items() if w is not None}
    lens = torch.tensor([L, L - 100], dtype=torch.int32, device="cuda")
    y, last, ck = S.sig_gated_scan_forward(**v, lengths=lens, checkpoint=True)
    held = v["initial_state"].clone()
    rows, end = [], None
    for i in range(L):
        if i == L - 100:
            end = held[1].clone()
        rows.append(S.sig_gated_scan_step(v["x"][:, i], v["decay_gate"][:, i], v["input_gate"][:, i], v["log_rate"], held))
    want = torch.stack(rows, 1)
    want[1, L - 100:] = 0
    close(y, want.cpu(), t, "y")
    close(last, torch.stack([held[0], end]).cpu(), F32, "state")
    g = up(normal(L)(B, L, D).to(t))
    whole_pass = S.sig_gated_scan_backward(v["x"], v["decay_gate"], v["input_gate"], v["log_rate"], g, ck, v["initial_state"], lens, last)
    # the same from the definition, reversed in time, in 64 bits on the GPU
    s = {k: w.double() for k, w in v.items()}
    open_, i = torch.sigmoid(s["decay_gate"]), torch.sigmoid(s["input_gate"])
    u = torch.exp(s["log_rate"]) * open_
    a, size = torch.exp(-u), torch.sqrt(-torch.expm1(-2 * u))
    h = [s["initial_state"]]
    for k in range(L):
        on = (k < lens)[:, None]
        h.append(torch.where(on, a[:, k] * h[-1] + size[:, k] * i[:, k] * s["x"][:, k], h[-1]))
    back, gx, gp = last.double(), torch.zeros_like(s["x"]), torch.zeros_like(s["x"])
    for k in reversed(range(L)):
        on = (k < lens)[:, None]
        lam = torch.where(on, back + g[:, k].double(), 0)
        gx[:, k] = lam * size[:, k] * i[:, k]
        gp[:, k] = lam * u[:, k] * (1 - open_[:, k]) * (a[:, k] ** 2 / size[:, k] * i[:, k] * s["x"][:, k] - a[:, k] * h[k])
        back = torch.where(on, lam * a[:, k], back)
    close(whole_pass["x"], gx.cpu(), t, "grad x")
    close(whole_pass["decay_gate"], gp.cpu(), t, "grad decay gate")
    close(whole_pass["initial_state"], back.cpu(), F32, "grad initial state")


@gpu
def test_rates_next_to_nothing_keep_their_precision():
    """1 - a^2 of decays next to one: relative precision of the states that a first token gives, over the border between the two ways it is computed."""
    u = torch.logspace(-12, 1, 400).double()
    u = torch.cat([u, torch.linspace(0.24, 0.26, 101).double()])
    D = u.numel()
    rate = torch.log(2 * u).float()                                                          # gates of zero: half of it
    x = torch.ones(1, 1, D, device="cuda")
    z = torch.zeros_like(x)
    y, _ = S.sig_gated_scan_forward(x, z, z, up(rate))
    want = 0.5 * torch.sqrt(-torch.expm1(-torch.exp(rate.double())))
    # exp(log_rate) carries |log_rate| 2^-24 of rounding, half of it after the root; the series' end and the difference 2e-7 and 4e-7, likewise
    within(y[0, 0], want, want * (8 + rate.double().abs()) * 2.0 ** -24 + want * 5e-7, "y")


@gpu
def test_two_graphs_and_eager_work_side_by_side():
    """Two captured calls of the same operators on other inputs, replayed in turn with eager work between: workspaces are not shared."""
    n = normal(30)
    def make(seed):
        m = normal(seed)
        x, w, g = up(m(2, 300, 72).to(B16)), up((m(40, 72) / 8).to(B16)), up(m(2, 300, 40).to(B16))
        rate, norm = up(m(72) - 2), up(1 + 0.1 * m(72))

        def run():
            y, s, ck = S.sig_gated_scan_forward(x, x, x, rate, checkpoint=True)
            b = S.sig_gated_scan_backward(x, x, x, rate, x, ck)
            q, total = S.sig_norm_forward(y, norm, x)
            z, pre = S.sig_linear_forward(q, w, activation="gelu", keep=True)
            return [y, s, b["x"], b["log_rate"], q, z, *S.sig_linear_backward(q, w, g, "gelu", pre, bias=True), *S.sig_norm_backward(total, norm, y)]
        return run
    runs = [make(1), make(2)]
    want = [[v.clone() for v in r()] for r in runs]
    graphs, held = [], []
    for r in runs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(r())
    for k in range(4):
        graphs[k % 2].replay()
        eager = runs[1 - k % 2]()
        graphs[1 - k % 2].replay()
        torch.cuda.synchronize()
        for got, ok in ((held[0], want[0]), (held[1], want[1]), (eager, want[1 - k % 2])):
            assert all(torch.equal(a, b) for a, b in zip(got, ok)), k


# ------------------------------------------------------------------------------------------------ every way through the product
@gpu
@pytest.mark.parametrize("activation", [None, "silu", "gelu"])
@pytest.mark.parametrize("t", [F32, B16])
@pytest.mark.parametrize("M,K,N", [(1, 32, 64), (37, 128, 72), (200, 336, 264), (70, 40, 8), (300, 8, 136)])
def test_activations_and_gradients_of_whole_chunks(M, K, N, t, activation):
    """Rows of whole 16-byte chunks take other kernels than the sizes of the general test."""
    L.test_product_with_activation_and_its_gradient(M, K, N, t, activation)


@gpu
@pytest.mark.parametrize("out", [F32, B16])
@pytest.mark.parametrize("M,K,N", [(1, 64, 24), (33, 4112, 45), (64, 256, 100), (65, 1040, 48), (300, 4096, 70)])
def test_scales_over_tiles_splits_and_few_tokens(M, K, N, out):
    n, m = whole(M + N), normal(M)
    x, w, b, r = n(M, K).to(E8), n(N, K).to(E8), m(N).to(out), m(M, N).to(out)
    sx, sw = m(M).abs() + 0.1, m(N).abs() + 0.1
    want = (x.double() @ w.double().t()) * sx.double()[:, None] * sw.double()          # the sums are exact: two products with scales, two additions
    got = S.sig_linear_forward(up(x), up(w), up(b), up(r), x_scale=up(sx), weight_scale=up(sw), dtype=out)
    total = want + b.double() + r.double()
    within(got, total, H[out] * 1.001 * total.abs() + 6 * 2.0 ** -24 * (want.abs() + b.double().abs() + r.double().abs()), "y")


@gpu
@pytest.mark.parametrize("t", [F32, B16])
@pytest.mark.parametrize("activation", [None, "gelu"])
@pytest.mark.parametrize("M,K,N", [(70, 128, 72), (65, 100, 50), (300, 64, 24)])
def test_any_choice_of_gradients(M, K, N, activation, t):
    """What is not asked for changes nothing in the rest."""
    n = normal(M + K)
    x, w, g, pre = up(n(M, K).to(t)), up(n(N, K).to(t)), up(n(M, N).to(t)), up(n(M, N).to(t))
    every = S.sig_linear_backward(x, w, g, activation, pre, bias=True)
    for k in range(8):
        asked = [bool(k & 1), bool(k & 2), bool(k & 4)]
        some = S.sig_linear_backward(x, w, g, activation, pre, bias=asked[2], need_x=asked[0], need_weight=asked[1])
        for want, got, yes in zip(every, some, asked):
            assert torch.equal(got, want) if yes else got is None, k


@gpu
@pytest.mark.parametrize("t", [F32, B16])
@pytest.mark.parametrize("activation", [None, "silu"])
def test_gradients_through_the_c_abi_from_anywhere(activation, t):
    """grad_y, the workspace and the outputs at odd places, grad_y's rows apart or one row for all tokens; what lies behind the outputs stays."""
    from tests.test_layer import LINEAR_ORDER, pack
    lib, kind = S.load_library(), 0 if t is F32 else 1
    stream = torch.cuda.current_stream().cuda_stream
    M, K, N = 200, 136, 72
    n = normal(5) if activation else whole(5)                       # without activation the kernel may be another one: whole numbers are exact in any order
    x, w, pre = up(n(M, K).to(t)), up(n(N, K).to(t)), up(n(M, N).to(t))
    a = pack(dict.fromkeys(LINEAR_ORDER, 0) | dict(dtype=kind, out=kind, M=M, N=N, K=K, act=1 if activation else 0, xs=K, x=x.data_ptr(), weight=w.data_ptr()), LINEAR_ORDER)
    wide = up(n(M, N + 13).to(t))
    for g, stride in ((wide[:, 8:8 + N], N + 13), (wide[:, 1:1 + N], N + 13), (wide[:1, 3:3 + N].expand(M, N), 0)):
        whole_g = g.contiguous()
        want = S.sig_linear_backward(x, w, whole_g, activation, pre, bias=True)
        for shift in (0, 1):
            outs = [torch.full((s + 64,), 7.0, dtype=t, device="cuda") for s in (M * K, N * K, N)]
            ws = torch.empty(lib.sig_linear_backward_workspace_bytes(a) + 4, dtype=torch.uint8, device="cuda")
            at = [v.data_ptr() + shift * v.element_size() for v in outs]
            assert lib.sig_linear_backward(a, g.data_ptr(), stride, pre.data_ptr(), *at, ws.data_ptr() + 4 * shift, ws.numel() - 4 * shift, stream) == 0
            for v, e in zip(outs, want):
                assert torch.equal(v[shift:shift + e.numel()], e.flatten()) and (v[:shift] == 7).all() and (v[shift + e.numel():] == 7).all()


@gpu
@pytest.mark.parametrize("t", [F32, B16])
def test_one_residual_row_for_all_tokens(t):
    n = normal(6)
    for M, K, N in ((5, 64, 40), (300, 64, 40), (130, 2056, 64), (9, 33, 7)):
        x, w, r = up(n(M, K).to(t)), up(n(N, K).to(t)), up(n(1, N).to(t)).expand(M, N)
        assert torch.equal(S.sig_linear_forward(x, w, residual=r), S.sig_linear_forward(x, w, residual=r.contiguous()))
        h, f = up(n(1, K).to(t)).expand(M, K), up(n(K))
        for one, two in zip(S.sig_norm_forward(x, f, h), S.sig_norm_forward(x, f, h.contiguous())):
            assert torch.equal(one, two)


def test_more_outputs_than_a_launch_numbers():
    """Refused before anything is enqueued (the pointers here lead nowhere)."""
    from tests.test_layer import BIG, LINEAR_OK, LINEAR_ORDER, pack
    a = pack({**LINEAR_OK, "M": 0, "N": 1 << 28}, LINEAR_ORDER)
    assert S.load_library().sig_linear_backward(a, 4096, 8, 0, 0, 0, 4096, 4096, BIG, 0) == -7


@gpu
@pytest.mark.parametrize("t", [F32, B16, E8])
def test_long_products_of_rows_that_are_no_whole_chunks(t):
    """Large enough that the operands are copied into aligned rows first: both, x alone (rows aligned, their start not), or the weight alone; NaN between the rows."""
    M, K, N = 4000, 3999, 2050
    n, out = whole(1, 2), B16 if t is E8 else t
    wide = torch.full((M, K + 18), math.nan)
    wide[:, 1:K + 2] = n(M, K + 1)
    wide, w0, b, r = up(wide.to(t)), up(n(N, K + 1).to(t)), up(n(N).to(out)), up(n(M, N).to(out))
    flat = torch.empty(N * 4000 + 16, dtype=t, device="cuda")
    moved = flat[1:1 + N * 4000].view(N, 4000)                       # whole rows that begin beside a 16-byte address
    moved.copy_(w0)
    aligned = wide[:, 1:].contiguous()[:, :4000].contiguous()
    for x, w in ((wide[:, 1:K + 1], w0[:, :K].contiguous()), (wide[:, 1:K + 2], w0), (aligned, moved)):
        g = up(whole(2, 2)(M, N).to(out))
        assert torch.equal(S.sig_linear_forward(x, w, b, r), product(x, w, b, r).to(out))
        if t is not E8:
            gx, gw, gb = S.sig_linear_backward(x, w, g, bias=True)
            assert torch.equal(gx, product(g, w.t().contiguous()).to(t)) and torch.equal(gw, product(g.t().contiguous(), x.t().contiguous()).to(t))
            assert torch.equal(gb, g.double().sum(0).to(t))


def test_gradient_of_rows_beyond_32_bit_offsets():
    """Rows of a tile are reached by 32-bit offsets: refused before anything is enqueued (the pointers here lead nowhere)."""
    from tests.test_layer import BIG, LINEAR_OK, LINEAR_ORDER, pack
    for change in ({"N": 1 << 22}, {"K": 1 << 22, "xs": 1 << 22}):
        a = pack({**LINEAR_OK, **change}, LINEAR_ORDER)
        assert S.load_library().sig_linear_backward(a, 4096, 1 << 22, 0, 4096, 4096, 4096, 4096, BIG, 0) == -7


@gpu
def test_narrow_products_of_more_rows_than_small_tiles_number():
    """Half a thousand million rows of eight values: tiles of 64 rows would be more than a launch numbers."""
    M = (1 << 29) + 77
    x, w = torch.empty(M, 8, dtype=B16, device="cuda").random_(-3, 4), up(whole(3, 3)(8, 8).to(B16))
    rows = (slice(0, 300), slice(M - 300, M), slice(M // 2, M // 2 + 100), slice((1 << 29) - 100, (1 << 29) + 60))
    y = S.sig_linear_forward(x, w)
    gx, _, _ = S.sig_linear_backward(x, w, x, need_weight=False)
    for r in rows:
        assert torch.equal(y[r], product(x[r], w).to(B16)) and torch.equal(gx[r], product(x[r], w.t().contiguous()).to(B16))


@gpu
@pytest.mark.parametrize("t", [F32, B16])
def test_rates_beyond_their_limit_have_no_gradient(t):
    """log_rate counts as min(log_rate, 64), so its gradient is zero beyond; that of gates so far shut that u is of the size of one is what it is at 64.
    Tolerance: exp(log_rate) and the gate are off by up to 64 times 1.5 * 2^-24 each, u by 1.2e-5 of itself; gradients of tokens by that times a few."""
    rates = torch.tensor([60.0, 63.5, 64.0, 64.001, 65.0, 90.0, math.inf])
    D, L = rates.numel(), 40
    n = normal(8)
    v = dict(x=n(2, L, D).to(t), decay_gate=(-63 + n(2, L, D)).to(t), input_gate=n(2, L, D).to(t), log_rate=rates, initial_state=n(2, D))
    gy = n(2, L, D).to(t)
    d = {k: up(w) for k, w in v.items()}
    y, _, ck = S.sig_gated_scan_forward(**d, checkpoint=True)
    got = S.sig_gated_scan_backward(d["x"], d["decay_gate"], d["input_gate"], d["log_rate"], up(gy), ck, d["initial_state"])
    leaves = {k: w.double().requires_grad_() for k, w in v.items()}
    want, _ = R.gated(**{**leaves, "log_rate": leaves["log_rate"].clamp(max=64.0)})
    grads = dict(zip(leaves, torch.autograd.grad((want * gy.double()).sum(), list(leaves.values()))))
    assert not got["log_rate"][rates > 64].any() and grads["log_rate"][:3].abs().min() > 0.01
    for k in ("x", "decay_gate", "input_gate", "log_rate", "initial_state"):
        slack = 1e-3 if t is F32 or k in ("log_rate", "initial_state") else 2.0 ** -7
        within(got[k], grads[k], slack * (grads[k].abs() + grads[k].square().mean().sqrt()), k)


@gpu
@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("t", [F32, B16])
def test_activations_keep_their_relative_precision_far_below_zero(t, name):
    """Values and slopes down to 1e-31, relative to what they are; a weight of one leaves the products exact.  In half steps of float32 (u = 2^-24):
    SiLU   the exponent -z log2(e) is rounded (constant included) by 1.25 |z|, the exponential 2, the sum 1, the quotient 2, the product 1; slope: two more.
    GELU   exp(-z^2 / 2) by 1.125 z^2 and 2; t P(t) by 25 in the worst case that its roundings and the fit's 5e-8 allow (degree 5: 178, the fit's 1e-5),
           summed by running error analysis over [-13, 0]; the slope z phi + Phi by as much of both its terms, and two roundings.
    bfloat16 adds half a step of its own."""
    u, h = 2.0 ** -24, 0.0 if t is F32 else H[B16] * 1.001
    z = (-torch.linspace(0.001, 12.0 if name == "gelu" else 70.0, 4001)).to(t)
    one, w = torch.ones(z.numel(), 1, dtype=t, device="cuda"), torch.ones(1, 1, dtype=t, device="cuda")
    y, pre = S.sig_linear_forward(up(z)[:, None], w, activation=name, keep=True)
    assert torch.equal(pre.cpu()[:, 0], z)
    gx, _, _ = S.sig_linear_backward(up(z)[:, None], w, one, name, pre)
    v = z.double()
    want, slope = R.act(v, name), R.slope(v, name)
    if name == "silu":
        off, s = (6 + 1.25 * v.abs()) * u, 1 / (1 + torch.exp(-v))
        size, of_slope = s * (1 + v.abs() * (1 - s)), off + 2 * u
    else:
        off = ((25 if t is F32 else 178) + 1.2 * v * v) * u
        size, of_slope = v.abs() * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi) + 0.5 * torch.special.erfc(-v / math.sqrt(2.0)), off + 2 * u
    within(y[:, 0], want, (off + h) * want.abs(), "value")
    within(gx[:, 0], slope, of_slope * size + h * (slope.abs() + of_slope * size), "slope")
