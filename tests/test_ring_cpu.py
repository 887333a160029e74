"""What a ring of loads does after a wait ran out (csrc/ecq_ring.h), on counters in place of barriers: whatever was issued
has landed at the end, and no wait is for good.  The kernels' own waits cannot be made to run out at every point."""
import ctypes
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1806_08054_b200", "csrc")
CXX = os.environ.get("CXX") or shutil.which("g++")


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    if not CXX:
        pytest.skip("no C++ compiler")
    so = str(tmp_path_factory.mktemp("ring") / "ring_model.so")
    subprocess.check_call([CXX, "-std=c++17", "-O2", "-shared", "-fPIC", "-I" + CSRC, os.path.join(HERE, "ring_model.cpp"), "-o", so])
    return ctypes.CDLL(so).ring_model


@pytest.mark.parametrize("ctas", [1, 2])
@pytest.mark.parametrize("stages", [2, 5, 6, 7])
@pytest.mark.parametrize("begin,steps", [(0, 1), (0, 9), (3, 64), (5, 3)])
def test_all_that_was_issued_lands(model, ctas, stages, begin, steps):
    assert model(stages, ctas, begin, steps, 1000 * stages + steps, 2000, 1) == 0


def test_the_model_sees_loads_on_their_way(model):
    assert model(6, 2, 0, 9, 1, 200, 0) > 0
