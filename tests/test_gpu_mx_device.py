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


def every_value(dtype):
    """Every finite value of a 16-bit type, as fp32."""
    v = torch.arange(65536, device=DEV).to(torch.int32).to(torch.uint16).view(dtype).float()
    return v[torch.isfinite(v)]


def activation(lib, x, up=None):
    assert x.numel() % 2 == 0
    y = torch.empty_like(x)
    assert lib.run_activation(P(x), None if up is None else P(up), x.numel() // 2, P(y)) == 0
    return y


# Half of the smallest subnormal: what rounding the result itself may cost next to 0.
TINY = 2.0 ** -150


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_gelu_of_every_16_bit_value(lib, dtype):
    """Within 2^-21 of |x| of the exact one."""
    x = every_value(dtype)
    y = activation(lib, x).double()
    want = 0.5 * x.double() * torch.special.erfc(-x.double() / 2 ** 0.5)
    off = (y - want).abs() / (x.double().abs() * 2.0 ** -21 + TINY)
    assert off.max() <= 1, (float(off.max()), float(x[off.argmax()]))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("up", [1.0, -0.3701171875, 25.875, 2.0 ** -14, -60000.0])
def test_swiglu_of_every_16_bit_gate(lib, dtype, up):
    """Within 2^-21 of |g u| of the exact one, where that is a finite fp32 value."""
    g = every_value(dtype)
    g = g[(g.double() * up).abs() <= torch.finfo(torch.float32).max]
    g = g[:g.numel() // 2 * 2].contiguous()
    y = activation(lib, g, torch.full_like(g, up)).double()
    size = (g.double() * up).abs()
    want = g.double() * torch.sigmoid(g.double()) * up
    off = (y - want).abs() / (size * 2.0 ** -21 + TINY * max(1, 2 * abs(up)))
    assert off.max() <= 1, (float(off.max()), float(g[off.argmax()]))
