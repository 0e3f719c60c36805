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


def P(t):
    return None if t is None else t.data_ptr()


def stream():
    return torch.cuda.current_stream().cuda_stream


def quantized_weights(g, E, N, K, fmt, dtype):
    """E matrices of random codes with scales around 1."""
    codes = torch.randint(0, 256, (E, N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    one = 126 if fmt == "block32" else 52
    scales = (one + torch.randint(0, 3, (E, *mx.scale_shape(N, K, fmt)), generator=g, device=DEV)).to(torch.uint8)
    rows = torch.full((E, N), 0.25, device=DEV) if fmt == "block16" else None
    return mx.MXTensor(codes, scales, rows, fmt)


def random_routing(g, T, k, E, experts=None):
    """k different ones of `experts` (all E) for each token."""
    among = torch.arange(E, device=DEV) if experts is None else torch.tensor(experts, device=DEV)
    at = among[torch.rand((T, among.numel()), generator=g, device=DEV).argsort(1)[:, :k]]
    return mx.Routing(at.to(torch.int32).contiguous(), torch.ones((T, k), device=DEV), E)


@pytest.mark.parametrize("T,k,E,N,K", [(20, 2, 16, 256, 256), (300, 2, 64, 384, 256), (900, 4, 8, 128, 512)])
def test_product_right_behind_its_plan(T, k, E, N, K):
    """clq_mx_plan and clq_mx_grouped_linear with nothing in between, two routings in turn through one
    plan: the product starts while its plan is being written over the other one."""
    g = gen(T)
    w = quantized_weights(g, E, N, K, "block32", F16)
    turns = []
    for part in (range(E // 2), range(E // 2, E)):  # different experts: an old list is a wrong one
        r = random_routing(g, T, k, E, list(part))
        rows, space, R = mx.plan(r)
        q = mx._empty(R, K, "block32", DEV)
        X = torch.randn((T, K), generator=g, device=DEV).to(F16)
        assert mx.clq_mx_quantize(P(X), 0, T, K, K, None, 1, 0, 0, P(q[0]), P(q[1]), None, P(rows), k, R, stream()) == 0
        turns.append([r, rows, q, torch.empty_like(rows), torch.zeros((R, N), dtype=F16, device=DEV), None])
    nbytes = mx.clq_mx_plan_bytes(T, k, E)
    space = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)

    def plan(t):
        return mx.clq_mx_plan(P(t[0].experts), T, k, E, P(t[3]), P(space), nbytes, stream())

    def product(t):
        return mx.clq_mx_grouped_linear(P(t[2][0]), P(t[2][1]), None, P(space), P(w.codes), P(w.scales), None, None, T, k, E, N,
                                        K, 1, 0, 0, P(t[4]), stream())
    for t in turns:
        assert plan(t) == 0
        torch.cuda.synchronize()
        assert product(t) == 0
        t[5] = t[4][t[1].flatten().long()]
        some = torch.randint(0, T * k, (8,), generator=g, device=DEV).tolist()
        for i in some:  # and what was made in order is the product
            e, row = int(t[0].experts.flatten()[i]), int(t[1].flatten()[i])
            x = mx.dequantize(mx.MXTensor(t[2][0], t[2][1]), F16)[row].double()
            want = mx.dequantize(mx.MXTensor(w.codes[e], w.scales[e]), F16).double() @ x
            assert (t[5][i].double() - want).abs().max() <= 2.0 ** -10 * want.abs().max()
    for _ in range(100):
        for t in turns:
            t[4].zero_()
            assert plan(t) == 0 and product(t) == 0
        for t in turns:
            assert torch.equal(t[3], t[1]) and torch.equal(t[4][t[1].flatten().long()], t[5])
