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
from tests.test_sequence import CONV_ORDER, SCAN_ORDER, close, gpu, pack, up

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
# A chunk's growth of 2^150: its exponent, 104 in natural units, is off by a rounding of A, of D log2(e) and of their product, 3 * 2^-24 each
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
