"""What the operators of a layer decide on the host, or by arithmetic that the host runs too: checked there over whole ranges."""
import os
import shutil
import subprocess

import pytest

import paper_2602_24066_amd as S
from tests.test_layer import LINEAR_OK, LINEAR_ORDER, pack

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2602_24066_amd", "csrc")


def host_program(name, where, *args):
    """Runs tests/c_abi/<name>.cpp, which prints what is wrong."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(where / name)
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", CSRC, os.path.join(HERE, "c_abi", name + ".cpp"), "-o", exe], check=True)
    out = subprocess.run([exe, *args], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


def test_lanes_of_the_gated_recurrence_read_channels_that_are_there(tmp_path):
    """No lane reads a channel behind the last (of the rates, the states, the checkpoint), pairs stay pairs, and every channel is stored once."""
    host_program("gated_lanes", tmp_path, "1000")


# ------------------------------------------------------------------------------------------------ what a launch can number
def refused(a, gradient, **pointers):
    """The code of a call whose pointers lead nowhere: it has to be refused before anything is enqueued."""
    lib = S.load_library()
    p = dict(pre=4096, gx=4096, gw=4096, gb=4096) | pointers
    if gradient:
        return lib.sig_linear_backward(a, 4096, a[3], p["pre"], p["gx"], p["gw"], p["gb"], 4096, 1 << 60, 0)
    return lib.sig_linear_forward(a, 4096, 0, 4096, 1 << 60, 0)


def test_products_are_refused_before_any_of_their_launches():
    """Too many tiles of float32 outputs (a terabyte of them): neither the copies of rows that are no whole chunks nor the slopes, the bias's sums or the
    first of the gradient's products go before the refusal."""
    a = lambda **v: pack({**LINEAR_OK, "dtype": 0, "out": 0, **v}, LINEAR_ORDER)             # noqa: E731
    assert refused(a(M=1 << 24, N=1 << 14, K=1001, xs=1001), False) == -7                    # copies of both operands first
    assert refused(a(M=1 << 24, N=1 << 14, K=1008, xs=1008), False) == -7
    wide = dict(M=1 << 24, N=4, K=1 << 14, xs=1 << 14)                                       # the gradient of x: as many tiles
    assert refused(a(**wide, act=1), True) == -7                                             # slopes first
    assert refused(a(**wide), True) == -7                                                    # the bias's sums first
    assert refused(a(**wide), True, gb=0) == -7
    many = dict(M=(1 << 31) - 300, N=4, K=4, xs=4)                                           # a workgroup for every 64 rows of the slopes and the bias's sums
    assert refused(a(**many, act=1), True) == -7 and refused(a(**many), True) == -7


def test_every_product_that_fits_the_memory_has_tiles_that_a_launch_numbers(tmp_path):
    """Narrow products of many rows among them, which the launch's model alone would give more small tiles than that."""
    host_program("linear_tiles", tmp_path)
