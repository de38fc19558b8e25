"""What the operators of a layer decide on the host, or by arithmetic that the host runs too: checked there over whole ranges."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2602_24066_amd", "csrc")


def test_lanes_of_the_gated_recurrence_read_channels_that_are_there(tmp_path):
    """No lane reads a channel behind the last (of the rates, the states, the checkpoint), pairs stay pairs, and every channel is stored once."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "gated_lanes")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", CSRC, os.path.join(HERE, "c_abi", "gated_lanes.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe, "1000"], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
