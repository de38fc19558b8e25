"""Sequence operators at the edges of what their contract allows, against the plain 64-bit implementations."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

import paper_2602_24066_amd as S
from tests import seq_reference as R
from tests.test_sequence import CONV_ORDER, SCAN_ORDER, close, gpu, pack, poison, up

TOKENS = ("x", "dt", "b", "c", "gate")
NAMES = dict(x="x", dt="dt", A="A", b="B", c="C", skip="skip", gate="gate", dt_bias="dt_bias", initial_state="initial_state")


def chunk_of(which, B, L, D, G, N):
    """Tokens of a time chunk of the forward or backward kernels (L where there is one), by the workspace that they ask for."""
    lib = S.load_library()
    args = pack(dict.fromkeys(SCAN_ORDER, 0) | dict(dtype=0, B=B, L=L, D=D, G=G, N=N, softplus=1), SCAN_ORDER)
    tiles, runs = -(-L // 16), G * -(-(D // G) // 64)
    if which == "forward":
        count = lib.sig_scan_forward_workspace_bytes(args) // (4 * B * D * (N + 1))
    else:
        # sums of dB and dC, then for each chunk the parameters' gradients, and with more than one chunk their states
        states = 8 if N <= 8 else 16 if N <= 16 else 32 if N <= 32 else 64
        left = lib.sig_scan_backward_workspace_bytes(args) // 4 - B * tiles * runs * states * 32
        count = left // (B * D * (N + 2))
        if count > 1:
            count = left // (B * D * (2 * N + 3))
    return -(-tiles // count) * 16 if count > 1 else L


# ------------------------------------------------------------------------------------------------ states that grow
# A chunk's growth of 2^150: its exponent, 104 in natural units, is off by a rounding of A, of A log2(e) and of their product, 3 * 2^-24 each
# at the most, and the factor by 104 times that, 1.9e-5; the rest as for other float32 results.
GROWTH_TOL = 3e-5


def near(got, want, what):
    got, want = got.detach().double().cpu(), want.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    assert float((got - want).norm()) <= GROWTH_TOL * float(want.norm()), what


@gpu
@pytest.mark.parametrize("by", ["A", "steps"])
@pytest.mark.parametrize("D,N", [(70, 16), (20, 40), (33, 4)])
def test_growth_over_chunks_leaves_zeros_alone(D, N, by):
    """States that grow by 2^150 over a chunk and are zero until the last tokens; adjoint states that are zero from the first tokens on."""
    L = 640
    chunk = min(chunk_of("forward", 1, L, D, 1, N), chunk_of("backward", 1, L, D, 1, N))
    assert 16 <= chunk <= L // 3, "the case is for several time chunks"
    v = R.inputs("scan", 1, L, D, N=N, carry=False, full=False, seed=21)
    gy = v.pop("grad_out")
    v.pop("grad_final_state")
    v["dt"].fill_(1.0 if by == "A" else -1.0)
    v["A"].fill_(-0.05 if by == "A" else 0.05)
    v["A"][:, 0] = 150 * math.log(2.0) / chunk * float(v["dt"][0, 0, 0])
    v["x"][:, :-4] = 0
    gy[:, 4:] = 0
    y, state, grads = R.with_gradients(R.scan, v, gy, None, softplus=False)
    d = {k: up(w) for k, w in v.items()}
    got_y, got_state, ck = S.sig_scan_forward(**d, softplus=False, checkpoint=True)
    near(got_y, y, "y")
    near(got_state, state, "state")
    got = S.sig_scan_backward(**d, softplus=False, grad_out=up(gy), checkpoint=ck)
    for k in ("x", "dt", "A", "b", "c"):
        near(got[NAMES[k]], grads[k], "grad " + k)


@gpu
@pytest.mark.parametrize("from_end", [False, True])
def test_growth_over_a_chunk_of_small_states(from_end):
    """A state (or, from the end, an adjoint state) of 2^-100 that grows by 2^150 over one chunk: the chunk's factor is more than float32 holds, the
    result is not."""
    L, D, N = 640, 70, 16
    chunk = chunk_of("backward" if from_end else "forward", 1, L, D, 1, N)
    assert chunk <= L // 3, "the case is for several time chunks"
    v = R.inputs("scan", 1, L, D, N=N, carry=True, full=False, seed=22)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    v["dt"].zero_()
    at = slice((L - 1) // chunk * chunk, L) if from_end else slice(0, chunk)
    v["dt"][:, at] = 1.0
    v["A"].fill_(150 * math.log(2.0) / (L - at.start if from_end else chunk))
    v["x"].zero_()
    gy.zero_()
    v["initial_state"] *= 2.0 ** (-60 if from_end else -100)
    gs *= 2.0 ** -100
    y, state, grads = R.with_gradients(R.scan, v, gy, gs, softplus=False)
    d = {k: up(w) for k, w in v.items()}
    got_y, got_state, ck = S.sig_scan_forward(**d, softplus=False, checkpoint=True)
    near(got_y, y, "y")
    near(got_state, state, "state")
    got = S.sig_scan_backward(**d, softplus=False, grad_out=up(gy), checkpoint=ck, grad_final_state=up(gs))
    for k in ("x", "A", "b", "initial_state"):
        near(got[NAMES[k]], grads[k], "grad " + k)


# ------------------------------------------------------------------------------------------------ decay rates
@gpu
@pytest.mark.parametrize("B,L,D,N,lengths", [(2, 39, 20, 16, [39, 17]), (1, 700, 70, 4, None), (1, 45, 33, 40, None)])
def test_the_lowest_decay_rates(B, L, D, N, lengths):
    """A down to float32's lowest value: a state is forgotten at once, and kept where the step size is zero."""
    v = R.inputs("scan", B, L, D, N=N, dtype=torch.float32, lengths=lengths, seed=33)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    v["A"][:, 0], v["A"][0, 1], v["A"][1, 1] = torch.finfo(torch.float32).min, -3e38, -2e38
    y, state, grads = R.with_gradients(R.scan, v, gy, gs)
    d = {k: up(w) for k, w in v.items()}
    got_y, got_state, ck = S.sig_scan_forward(**d, checkpoint=True)
    close(got_y, y, torch.float32, "y")
    close(got_state, state, torch.float32, "state")
    got = S.sig_scan_backward(**d, grad_out=up(gy), checkpoint=ck, grad_final_state=up(gs))
    for k, name in NAMES.items():
        close(got[name], grads[k], torch.float32, "grad " + name)
    # steps that add nothing and decay nothing: softplus(-200) is zero in float32, and the step of one token has to agree
    d["dt"][:, 5] = d["dt"][:, 20] = -200.0
    first = {k: w[:, :21] if k in TOKENS else w for k, w in d.items() if k != "lengths"}
    _, one = S.sig_scan_forward(**first)
    _, held = S.sig_scan_forward(**{k: w[:, :4] if k in TOKENS else w for k, w in first.items()})
    for i in range(4, 21):
        S.sig_scan_step(state=held, **{k: w[:, i] if k in TOKENS else w for k, w in first.items() if k != "initial_state"})
    close(one, held.cpu(), torch.float32, "state by steps")


@gpu
@pytest.mark.parametrize("B,L,D,N,lengths", [(2, 39, 20, 12, [39, 24]), (1, 700, 70, 13, None), (1, 640, 33, 40, None)])
def test_the_largest_step_sizes(B, L, D, N, lengths):
    """Tokens without an input whose step size is near float32's largest value forget what decays and keep what does not, several of them in a row
    and in states that are there to fill a register only."""
    v = R.inputs("scan", B, L, D, N=N, dtype=torch.float32, lengths=lengths, seed=34)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    v["A"][:, 3] = 0.0
    for t in (5, 6, 20, L // 2, L // 2 + 1):
        v["dt"][:, t], v["x"][:, t] = 2.5e38, 0.0
    y, state, grads = R.with_gradients(R.scan, v, gy, gs)
    d = {k: up(w) for k, w in v.items()}
    got_y, got_state, ck = S.sig_scan_forward(**d, checkpoint=True)
    close(got_y, y, torch.float32, "y")
    close(got_state, state, torch.float32, "state")
    got = S.sig_scan_backward(**d, grad_out=up(gy), checkpoint=ck, grad_final_state=up(gs))
    for k in ("b", "c", "gate", "skip", "initial_state"):        # those of x, dt and A are of the steps' own size
        close(got[NAMES[k]], grads[k], torch.float32, "grad " + k)


# ------------------------------------------------------------------------------------------------ filter weights that are not finite
@gpu
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("t,D,W", [(torch.float32, 8, 4), (torch.float32, 5, 3), (torch.bfloat16, 8, 4), (torch.bfloat16, 5, 8)])
def test_filter_weights_that_are_not_finite(t, D, W, bad):
    """They reach the gradients of the tokens that they are multiplied with: none that does not count, and none by way of such a token."""
    lengths = [50, 20, 0, 3, 17]
    v = R.inputs("conv", 5, 50, D, W=W, dtype=t, lengths=lengths, seed=31)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    v["weight"][0, 0] = bad
    v["weight"][D - 1, W - 1] = bad
    _, _, grads = R.with_gradients(R.conv, v, gy, gs, silu=False)
    d = {k: up(w) for k, w in v.items()}
    gx, gw, gb, gi = S.sig_conv_backward(d["x"], d["weight"], up(gy), d["bias"], d["initial_state"], d["lengths"], False, up(gs))
    for got, want, kind in ((gx, grads["x"], t), (gi, grads["initial_state"], t), (gw, grads["weight"], torch.float32), (gb, grads["bias"], torch.float32)):
        ok = torch.isfinite(want)
        assert torch.equal(torch.isfinite(got.cpu()), ok) and torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
        assert torch.equal(got.cpu()[~ok & ~torch.isnan(want)].double(), want[~ok & ~torch.isnan(want)])
        close(torch.where(ok, got.cpu(), 0), torch.where(ok, want, 0), kind, "gradient")
    for i, n in enumerate(lengths):
        assert not gx[i, n:].any()


# ------------------------------------------------------------------------------------------------ strides that are not used
@gpu
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_one_token_of_a_time_major_batch(t):
    """A time axis of length one has a stride that nothing is reached by, however large."""
    B, D, N = 3, 24, 16
    v = R.inputs("scan", B, 1, D, N=N, dtype=t, seed=41)
    gy, gs = up(v.pop("grad_out")), up(v.pop("grad_final_state"))
    d = {k: up(w) for k, w in v.items()}
    far = lambda w: w.as_strided(w.shape, (w.stride(0), 1 << 26, *w.stride()[2:]))          # noqa: E731
    e = {k: far(w) if k in TOKENS else w for k, w in d.items()}
    w = torch.randn(D, 4, device="cuda")

    def everything(a, g):
        y, h, ck = S.sig_scan_forward(**a, checkpoint=True)
        grads = S.sig_scan_backward(**a, grad_out=g, checkpoint=ck, grad_final_state=gs)
        return [y, h, *grads.values(), *S.sig_conv_forward(a["x"], w, return_state=True), *S.sig_conv_backward(a["x"], w, g)[:2]]

    for p, q in zip(everything(e, far(gy)), everything(d, gy)):
        assert torch.equal(p, q)


# ------------------------------------------------------------------------------------------------ strides that need no copy
@gpu
def test_the_convolution_reads_far_tokens_where_they_are():
    w = torch.randn(24, 4, device="cuda")
    store = torch.empty((2 << 26) + 24, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((1, 3, 24), (1, 1 << 26, 1))
    x.copy_(torch.randn(1, 3, 24, device="cuda"))
    near_, counts = x.contiguous(), []
    for v in (x, near_):
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        y, g = S.sig_conv_forward(v, w), S.sig_conv_backward(v, w, v)
        counts.append((torch.cuda.memory_stats()["allocation.all.allocated"] - before, y, *g[:2]))
    assert counts[0][0] == counts[1][0], "as many tensors as for tokens side by side"
    assert all(torch.equal(p, q) for p, q in zip(counts[0][1:], counts[1][1:]))


# ------------------------------------------------------------------------------------------------ calls of one token
def scan_args(**change):
    return pack(dict.fromkeys(SCAN_ORDER, 0) | dict(dtype=0, B=2, L=8, D=4, G=2, N=4, softplus=1, x=4096, dt=4096, b=4096, c=4096, A=4096) | change, SCAN_ORDER)


def conv_args(**change):
    return pack(dict(dtype=0, B=2, L=8, D=4, W=4, silu=1, xb=32, xt=4, x=4096, weight=4096, bias=0, initial=0, lengths=0) | change, CONV_ORDER)


@pytest.mark.parametrize("change", [{"L": 1 << 41}, {"L": -5}, {"xt": 1 << 40}, {"xt": -3}])
def test_calls_of_one_token_do_not_look_at_time(change):
    lib = S.load_library()
    assert lib.sig_conv_step(conv_args(**change), 0, 4096, 0) == -1                # for its missing state
    assert lib.sig_conv_step(conv_args(**change, B=0), 4096, 4096, 0) == 0
    for more in ({}, {"tt": 1 << 40, "zt": -1}):
        assert lib.sig_scan_step(scan_args(**change, **more), 0, 4096, 0) == -1
        assert lib.sig_scan_step(scan_args(**change, **more, B=0), 4096, 4096, 0) == 0


# ------------------------------------------------------------------------------------------------ launches beyond what the hardware numbers
@pytest.mark.parametrize("change", [
    dict(B=4096, D=2048, G=2048, N=16),              # 2^23 workgroups of 512 threads
    dict(B=1 << 24, D=64, G=1, N=8),                 # 2^24 of 256
    dict(B=1 << 22, D=16, G=1, N=64),                # 2^22 of 1,024
    dict(B=1, D=(1 << 24) - 1, G=1, N=16, L=0),      # 2^28 sums of parameters' gradients of 16 threads (the gradient alone)
])
def test_scan_launches_of_too_many_threads_are_refused(change):
    lib = S.load_library()
    args, big = scan_args(**{"L": 1, **change}), 1 << 60
    if "L" not in change:
        assert lib.sig_scan_forward(args, 4096, 0, 0, 0, 4096, big, 0) == -7
    grads = (ctypes.c_int64 * 13)(*[4096] * 13)
    grads[0] = grads[1] = 0
    assert lib.sig_scan_backward(args, grads, 4096, big, 4096, big, 0) == -7


@pytest.mark.parametrize("B,D,N", [(1 << 20, 1 << 10, 1), (1 << 20, 1 << 10, 16), (1 << 15, 1 << 14, 17), (1 << 15, 1 << 13, 64)])
def test_scan_steps_of_too_many_threads_are_refused(B, D, N):
    assert S.load_library().sig_scan_step(scan_args(B=B, D=D, G=1, N=N), 4096, 4096, 0) == -7


@pytest.mark.parametrize("change,aligned", [(dict(B=1 << 16, L=1, D=1 << 16), False), (dict(B=1 << 17, L=1, D=1 << 17), True), (dict(B=1, L=1, D=1 << 25, W=8), None)])
def test_conv_launches_of_too_many_threads_are_refused(change, aligned):
    """The third is one of the filter's sums, in the gradient alone."""
    lib = S.load_library()
    args = conv_args(**change, xb=0, xt=0, x=4096 if aligned else 4100)
    if aligned is not None:
        assert lib.sig_conv_forward(args, 4096, 0, 0) == -7
        assert lib.sig_conv_step(args, 4096, 4096, 0) == -7
    assert lib.sig_conv_backward(args, 4096, 0, 0, 0, 4096, 4096, 0, 0, 4096, 1 << 60, 0) == -7


# ------------------------------------------------------------------------------------------------ shapes of gradients
@gpu
@pytest.mark.parametrize("b_group,c_group", [(False, True), (True, False)])
def test_gradients_have_the_shapes_of_their_inputs(b_group, c_group):
    x, A = torch.randn(2, 9, 8, device="cuda"), -torch.ones(8, 4, device="cuda")
    b, c = torch.randn(2, 9, 4, device="cuda"), torch.randn(2, 9, 4, device="cuda")
    ck = S.sig_scan_forward(x, x, A, b, c, checkpoint=True)[2]
    want = S.sig_scan_backward(x, x, A, b, c, x, ck)
    b, c = b.unsqueeze(2) if b_group else b, c.unsqueeze(2) if c_group else c
    got = S.sig_scan_backward(x, x, A, b, c, x, ck)
    assert got["B"].shape == b.shape and got["C"].shape == c.shape
    assert torch.equal(got["B"].reshape(2, 9, 4), want["B"]) and torch.equal(got["C"].reshape(2, 9, 4), want["C"])


# ------------------------------------------------------------------------------------------------ host memory that runs out
NO_MEMORY = r"""
#include <cstdlib>
#include <new>
static bool none = false;
void* operator new(std::size_t n) { if (none) throw std::bad_alloc(); if (void* p = std::malloc(n ? n : 1)) return p; throw std::bad_alloc(); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
#include "kernels.hpp"
static int set = 0;
extern "C" hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
extern "C" hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { set++; return hipSuccess; }
int main()
{
    int k = 0;
    none = true;
    if (sig::ensure_dynamic_lds(&k, 100000) != hipSuccess || set != 1) return 1;
    none = false;
    if (sig::ensure_dynamic_lds(&k, 100000) != hipSuccess || set != 2) return 2;     // not remembered then, so set again
    if (sig::ensure_dynamic_lds(&k, 100000) != hipSuccess || set != 2) return 3;
    return 0;
}
"""


def test_a_lack_of_host_memory_does_not_leave_a_launch_as_an_exception(tmp_path):
    gxx, csrc = shutil.which("g++"), os.path.join(os.path.dirname(S.lib_path()), "csrc")
    if gxx is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("no g++ or no HIP headers")
    (tmp_path / "a.cpp").write_text(NO_MEMORY)
    subprocess.run([gxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", csrc, "-I", "/opt/rocm/include", str(tmp_path / "a.cpp"), "-o", str(tmp_path / "a")], check=True)
    assert subprocess.run([str(tmp_path / "a")]).returncode == 0


# ------------------------------------------------------------------------------------------------ forms that the sizes and the alignment choose
@gpu
@pytest.mark.parametrize("B,L,D,W,t,lengths", [
    (3, 40, 333, 3, "f32", [40, 0, 23]),             # channels that no vector access fits, a thread each: more than a workgroup's
    (2, 40, 1024, 4, "bf16", [40, 33]),              # as many groups of four as a workgroup has threads
    (2, 40, 512, 4, "f32", [17, 40]),                # and of two
    (2, 70, 258, 4, "bf16", None),
    (2, 40, 1554, 2, "bf16", [1, 39]),
    (1, 33, 2048, 8, "f32", None),
])
def test_convolutions_over_many_channels(B, L, D, W, t, lengths):
    t = torch.float32 if t == "f32" else torch.bfloat16
    v = R.inputs("conv", B, L, D, W=W, dtype=t, lengths=lengths, seed=D)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    y, state, grads = R.with_gradients(R.conv, v, gy, gs)
    d = {k: up(w) for k, w in (poison(v, ["x"]) if lengths else v).items()}
    got_y, got_state = S.sig_conv_forward(**d, return_state=True)
    close(got_y, y, t, "y")
    close(got_state, state, t, "state")
    got = S.sig_conv_backward(d["x"], d["weight"], up(gy), d["bias"], d["initial_state"], d["lengths"], True, up(gs))
    for k, g in zip(("x", "weight", "bias", "initial_state"), got):
        close(g, grads[k], t if k in ("x", "initial_state") else torch.float32, "grad " + k)


@gpu
@pytest.mark.parametrize("B,L,D,G,N,t,lengths", [
    (2, 400, 70, 1, 40, "f32", [400, 290]),          # several time chunks, more than 32 states, more channels than a wavefront has lanes
    (2, 330, 130, 2, 64, "bf16", [330, 17]),
    (1, 500, 66, 1, 24, "f32", [499]),
])
def test_scans_of_many_states_in_time_chunks(B, L, D, G, N, t, lengths):
    assert chunk_of("backward", B, L, D, G, N) < L
    t = torch.float32 if t == "f32" else torch.bfloat16
    v = R.inputs("scan", B, L, D, G=G, N=N, dtype=t, lengths=lengths, seed=N)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    y, state, grads = R.with_gradients(R.scan, v, gy, gs)
    hidden = poison({**v, "gy": gy}, [*TOKENS, "gy"])
    gy = up(hidden.pop("gy"))
    d = {k: up(w) for k, w in hidden.items()}
    got_y, got_state, ck = S.sig_scan_forward(**d, checkpoint=True)
    close(got_y, y, t, "y")
    close(got_state, state, torch.float32, "state")
    got = S.sig_scan_backward(**d, grad_out=gy, checkpoint=ck, grad_final_state=up(gs))
    for k, name in NAMES.items():
        close(got[name], grads[k], t if k in TOKENS else torch.float32, "grad " + name)


@gpu
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_time_strides_just_within_the_kernels_reach(t):
    """Rows 2^24 - 8 elements apart, three tiles of them: a tile's last row lies nearly 2^30 bytes from its first."""
    L, D, N, far = 40, 24, 16, (1 << 24) - 8
    store = torch.empty((L - 1) * far + 4 * D, dtype=t, device="cuda")
    v = R.inputs("scan", 1, L, D, N=N, dtype=t, lengths=[L - 3], seed=51)
    gy, gs = up(v.pop("grad_out")), up(v.pop("grad_final_state"))
    d = {k: up(w) for k, w in v.items()}
    e, at = dict(d), 0
    for k in ("x", "gate", "b", "c"):                # the rows of all lie behind one another
        w = d[k]
        e[k] = store.as_strided(w.shape, (1, far, *w.stride()[2:]), at)
        e[k].copy_(w)
        at += w[0, 0].numel()

    def everything(a):
        y, h, ck = S.sig_scan_forward(**a, checkpoint=True)
        return [y, h, *S.sig_scan_backward(**a, grad_out=gy, checkpoint=ck, grad_final_state=gs).values()]

    for p, q in zip(everything(e), everything(d)):
        assert torch.equal(p, q)


@gpu
@pytest.mark.parametrize("full", [True, False])
def test_gradients_of_the_step_sizes_at_special_values(full):
    """States that are forgotten at once, kept and grow; step sizes that vanish."""
    v = R.inputs("scan", 1, 40, 16, dtype=torch.float32, full=full, seed=11)
    gy, gs = v.pop("grad_out"), v.pop("grad_final_state")
    v["A"][:, 0], v["A"][:, 1], v["A"][:, 2] = -1e30, 0.0, 0.05
    v["dt"][0, 5], v["dt"][0, 6] = (-200.0, -30.0) if full else (0.0, 1e-13)
    _, _, grads = R.with_gradients(R.scan, v, gy, gs, softplus=full)
    d = {k: up(w) for k, w in v.items()}
    if not full:                                     # A times a state that is kept is 1e30 at token 5: the others are looked at alone
        grads["dt"][0, 5] = 0
    ck = S.sig_scan_forward(**d, softplus=full, checkpoint=True)[2]
    got = S.sig_scan_backward(**d, softplus=full, grad_out=up(gy), checkpoint=ck, grad_final_state=up(gs))
    if not full:
        got["dt"][0, 5] = 0
    for k in ("dt", "A", "dt_bias"):
        if v[k] is not None:
            close(got[k], grads[k], torch.float32, "grad " + k)


@gpu
@pytest.mark.parametrize("max_norm", [0.25, 1e9])
@pytest.mark.parametrize("off", [0, 1, 3])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_clip_into_tensors_of_either_type_and_alignment(kind, off, max_norm):
    """The products of either type into bfloat16 and float32, from and to addresses that agree or not."""
    g = torch.Generator().manual_seed(off)
    t = torch.float32 if kind == "f32" else torch.bfloat16
    flat = up(torch.randn(70000, generator=g).to(t))
    grads = [flat[1:10], flat[off + 16:off + 16 + 33 * 41].view(33, 41), flat[2001:2001 + 60000]]
    total = math.sqrt(sum(float(w.double().square().sum()) for w in grads))
    want = [w.double().cpu() * min(1.0, max_norm / (total + 1e-6)) for w in grads]
    for o in (torch.float32, torch.bfloat16):
        store = torch.full((70000,), 7.0, device="cuda", dtype=o)
        outs = [store[off:off + 9], store[off + 30:off + 30 + 33 * 41].view(33, 41), store[5002 + off:5002 + off + 60000]]
        norm = S.sig_grad_clip(grads, max_norm, out=outs)
        assert abs(float(norm) - total) <= 1e-6 * total
        for p, q in zip(outs, want):
            close(p, q, o, "products")
        left = torch.ones(70000, dtype=torch.bool, device="cuda")
        for p in outs:
            left[p.storage_offset():p.storage_offset() + p.numel()] = False
        assert (store[left] == 7.0).all()


@gpu
def test_clip_of_more_than_the_cache_holds():
    """71 million elements, 284 MB of products: they are stored past the cache, and a workgroup takes more elements than it does of fewer."""
    n = 71_000_003
    big = torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    grads = [big[1:n - 1], torch.randn(77, device="cuda").bfloat16()]
    total = float(torch.sqrt(sum(w.double().square().sum() for w in grads)))
    want = [w.double() * (1.0 / (total + 1e-6)) for w in grads]
    outs = [torch.empty(n - 2, device="cuda"), torch.empty(77, device="cuda")]
    for into in (outs, None):
        norm = S.sig_grad_clip(grads, 1.0, out=into)
        assert abs(float(norm) - total) <= 1e-6 * total
        for p, q in zip(into or grads, want):
            off = (p.double() - q).abs()
            assert float((off - q.abs() * (2.0 ** -22 if p.dtype is torch.float32 else 2.0 ** -8)).max()) <= 0
    assert not torch.isnan(big).any()
