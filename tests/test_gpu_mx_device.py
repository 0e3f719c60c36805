"""Device functions of the microscaled kernels by themselves (mx_device_kernels.cu), where a call
cannot show what they do."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2509_24416_gb300 import build

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))
DEV = "cuda"


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("mx") / "mx_device_kernels.so")
    r = subprocess.run([build._nvcc(), *build.ARCH, *build.FLAGS, "-shared", os.path.join(HERE, "mx_device_kernels.cu"), "-o", so],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(so)


def P(t):
    return ctypes.c_void_p(t.data_ptr())


def test_two_warps_give_up_together(lib):
    """Pairs of warps whose own waits end differently leave in the same turn: none stays at a barrier
    that its partner does not come to."""
    warps, n = 8, 6
    votes = torch.ones((n, warps), dtype=torch.int32)
    votes[0, 0] = 0  # the first pair: one warp gives up at once
    votes[3, 3] = 0  # the second: the other one, later
    votes[5, 4:6] = 0  # the third: both
    turns = torch.full((warps,), -1, dtype=torch.int32, device=DEV)
    assert lib.run_pairs(P(votes.to(DEV)), n, warps, P(turns)) == 0
    assert turns.tolist() == [0, 0, 3, 3, 5, 5, n, n]
