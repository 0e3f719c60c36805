"""CPU-only checks of the microscaled calls: what a call with an explicit stream hands back to the
caller's stream, and what calls refuse."""
import random

import pytest
import torch

import mx_tiles as tiles
from paper_2509_24416_gb300 import build, clq, mx
from test_streams_cpu import HERE, FakeStream, fake  # noqa: F401
from test_mx_cpu import tensor


@pytest.fixture
def recorded(fake, monkeypatch):  # noqa: F811
    """Calls of the library are fakes; the (data_ptr, stream) pairs that a call records."""
    monkeypatch.setattr(mx, "_on_gpu", lambda *t: None)
    for f in mx.EXPORTS:
        monkeypatch.setattr(mx, f, lambda *a: 0)
    monkeypatch.setattr(mx, "clq_mx_plan_rows", lambda *a: 128)
    monkeypatch.setattr(mx, "clq_mx_plan_bytes", lambda *a: 256)
    seen = []
    monkeypatch.setattr(clq, "_record", lambda ts, s: seen.extend(
        (t.data_ptr(), s.cuda_stream) for t in ts if isinstance(t, torch.Tensor)))
    return seen


X = torch.zeros((4, 64), dtype=torch.bfloat16)
ROUTING = mx.Routing(torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)), 3)
RESULTS = {
    "quantize_block32": (lambda s: mx.quantize(X, "block32", stream=s), lambda q: [q.codes, q.scales]),
    "quantize_block16": (lambda s: mx.quantize(X, "block16", stream=s), lambda q: [q.codes, q.scales, q.row_scale]),
    "route": (lambda s: mx.route(torch.zeros((4, 8)), 2, stream=s), lambda r: [r.experts, r.weights]),
    "plan": (lambda s: mx.plan(ROUTING, stream=s), lambda r: [r[0], r[1]]),
    "dequantize": (lambda s: mx.dequantize(tensor(4, 64), stream=s), lambda y: [y]),
    "linear": (lambda s: mx.linear(tensor(4, 64), tensor(8, 64), stream=s), lambda y: [y]),
}


@pytest.mark.parametrize("name", sorted(RESULTS))
def test_results_are_recorded_on_the_callers_stream(fake, recorded, name):  # noqa: F811
    """The caller may read and drop what a call on another stream made: every tensor of it."""
    call, parts = RESULTS[name]
    out = call(fake.side)
    assert sorted(recorded) == sorted((t.data_ptr(), HERE) for t in parts(out))
    recorded.clear()
    call(None)
    call(FakeStream(HERE, fake.log))
    assert not recorded


@pytest.mark.parametrize("bad", [256, -1, 1 << 32])
@pytest.mark.parametrize("dtype", [torch.int16, torch.int32, torch.int64])
def test_codes_that_are_no_bytes_are_refused(bad, dtype):
    w = tensor(8, 64)
    codes = torch.arange(256).view(8, 32).to(dtype)
    assert torch.equal(mx.MXTensor(codes, w.scales).codes.to(dtype), codes)
    if bad <= torch.iinfo(dtype).max:
        codes[3, 5] = bad
        with pytest.raises(ValueError, match="0 to 255"):
            mx.MXTensor(codes, w.scales)
    assert mx.MXTensor(codes[:0], w.scales[:0]).rows == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.int8, torch.bool, torch.complex64])
def test_codes_of_other_types_are_refused(dtype):
    w = tensor(8, 64)
    with pytest.raises(ValueError, match="uint8"):
        mx.MXTensor(w.codes.to(dtype), w.scales)


P = 1 << 20  # a 16-byte aligned "device" address that nothing reads


@pytest.mark.parametrize("T,k", [(1 << 30, 1), ((1 << 31) - 1, 1), (1, 1 << 30), (1, (1 << 31) - 1)])
def test_combine_refuses_what_its_indices_do_not_hold(T, k):
    build.build()
    assert mx.clq_mx_combine(P, 0, P, P, T, k, 8, 8, P, None) == 2


def test_shapes_of_the_tests_take_every_tile(tmp_path):
    lib = tiles.library(tmp_path)
    for M, K, N, tile in tiles.DENSE:
        assert tiles.dense(lib, M, N, K) == tile, (M, K, N)
    for T, k, E, N, K, tile in tiles.GROUPED:
        assert tiles.grouped(lib, T, k, E, N, K) == tile, (T, k, E, N, K)
    # no shape takes another one
    rng = random.Random(5)
    log = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
    seen = {tiles.dense(lib, log(1, 40000), log(1, 20000), 32 * log(1, 512)) for _ in range(20000)}
    assert seen == {t[-1] for t in tiles.DENSE}
    seen = {tiles.grouped(lib, log(1, 40000), rng.choice((1, 2, 4, 8)), log(8, 512), log(1, 8000), 32 * log(1, 512))
            for _ in range(20000)}
    assert seen == {t[-1] for t in tiles.GROUPED}
