"""Parts of the layer products' epilogue on the CPU: their own source, compiled for the host
and run a lane at a time over arrays that end at memory that cannot be
accessed, so that an access past an operand shows without a GPU. (Unoptimised: a load
whose value goes unused stays.)"""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_1909_10616_amd import build
    exe = tmp_path_factory.mktemp("epilogue") / "layers_epilogue"
    subprocess.run([build.HIPCC, "-O0", "-std=c++17", "--offload-host-only", "-I", os.path.join(ROOT, "include"),
                    "-I", build.CSRC, "-x", "hip", os.path.join(HERE, "layers_epilogue.cpp"), "-o", str(exe)],
                   check=True, capture_output=True)
    return str(exe)


def test_a_slice_of_a_few_rows_writes_its_own_sums(program):
    """Quads that only pad a row are not stored among the slices' sums, where they would fall on the
    up half, on the next row or past the last one."""
    r = subprocess.run([program, "part"], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout)


def test_whole_tiles_stay_inside_their_operands(program):
    """Bias, residual, kept pre-activations and outputs that end with the last row of a tile, in
    every tile, type and form."""
    r = subprocess.run([program, "whole"], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout)
