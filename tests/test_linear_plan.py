"""How a linear layer's products are cut and what space they ask for (no GPU)."""

import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2605_21177_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000                       # an address that is never touched


def _space(T, n_in, out, backward, dtype=B.BF16):
    layer = B.LinearLayer(dtype, B.ACT_NONE, out, n_in, T, P, n_in, P, n_in, None, None, 0)
    return B.lib().chunkft_linear_workspace_bytes(C.byref(layer), backward)


def _slabs(T, out, most=16):
    """Bytes of the sums of `most` slabs of a product [T, out]."""
    return most * T * ((out + 31) // 32 * 32) * 4


# 16-byte rows of x and W, whatever the number of W's rows: nothing of them is copied, so the space is at most the slabs'
@pytest.mark.parametrize("T,n_in,out", [(1024, 4096, 50257), (4096, 4104, 4097), (512, 768, 50257), (64, 4096, 50257), (4096, 4104, 4095), (2048, 1024, 2049)])
def test_rows_of_pieces_along_k_are_not_copied(T, n_in, out):
    copies = (T + out) * n_in * 2
    assert _space(T, n_in, out, 0) in {0} | {_slabs(T, out, s) for s in range(2, 17)}
    # the slabs of so many tiles are few: a copy of W alone would be more than all of the space
    assert _space(T, n_in, out, 0) < copies


@pytest.mark.parametrize("T,n_in,out", [(1024, 4096, 50257), (4096, 4104, 4097)])
def test_rows_of_pieces_fill_the_units_as_neighbours_of_their_size_do(T, n_in, out):
    """One row of W more or less changes nothing about how the others are taken."""
    assert _space(T, n_in, out, 0) == _space(T, n_in, out // 8 * 8, 0) == 0


def test_host_code_of_the_plan_under_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    assert gxx, "g++ is part of the image"
    csrc, exe = os.path.join(ROOT, "paper_2605_21177_amd", "csrc"), str(tmp_path / "linear_plan_sanitize")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-I", csrc,
           os.path.join(ROOT, "tests", "linear_plan_sanitize.cpp"), os.path.join(csrc, "layers_shape.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok:"), (r.stdout[-1000:], r.stderr[-3000:])


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("T,n_in,out", [(1000000, 3, 64), (1000000, 64, 3), (1 << 24, 1, 1), (100000, 17, 1000), (200000, 33, 31), (65536, 9, 4097)])
def test_operands_are_not_copied_into_rows_that_are_mostly_padding(T, n_in, out, backward):
    """The space is at most twice the operands and the sums over the tokens or the slabs (which are few where the tokens are many)."""
    operands = 2 * (T * (out if backward else n_in) + out * n_in)
    assert _space(T, n_in, out, backward) <= 2 * operands + (2 << 20)
