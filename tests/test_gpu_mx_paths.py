"""Microscaled operators on the GPU: paths, tiles and orders of calls that the shapes of
test_gpu_mx.py do not reach, against their definitions in 64 bits (mx_utils)."""
import pytest
import torch

from paper_2509_24416_gb300 import clq, mx

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


@pytest.fixture(autouse=True)
def no_device_error():
    yield
    assert clq.device_status() == 0


@pytest.mark.parametrize("make", ["quantize", "route"])
def test_dropped_results_of_another_stream_are_not_handed_out_again(make):
    """While the caller's stream has work queued, what it was given by a call on another stream and
    has dropped does not become that stream's next buffer."""
    side = torch.cuda.Stream()
    X = torch.randn((512, 512), generator=gen(1), device=DEV).to(BF16)
    torch.cuda.synchronize()
    if make == "quantize":
        out = mx.quantize(X, "block16", stream=side)
        blocks = [out.codes, out.scales, out.row_scale]
    else:
        out = mx.route(X, 32, stream=side)
        blocks = [out.experts, out.weights]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(200_000_000)  # clocks: a tenth of a second
    like = [(t.shape, t.dtype, t.data_ptr()) for t in blocks]
    del out, blocks
    with torch.cuda.stream(side):
        again = [torch.empty(shape, dtype=dtype, device=DEV) for shape, dtype, _ in like]
    assert not torch.cuda.current_stream().query()  # still at work
    assert not {t.data_ptr() for t in again} & {ptr for _, _, ptr in like}
    torch.cuda.synchronize()
