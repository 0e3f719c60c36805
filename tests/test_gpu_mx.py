"""Microscaled operators on the GPU against their definitions in 64 bits (mx_utils)."""
import numpy as np
import pytest
import torch

import mx_utils as ref
from paper_2509_24416_gb300 import clq, mx

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows_of(g, M, K, dtype):
    """N(0, 1) with a few large channels."""
    s = torch.ones(K, device=DEV)
    s[torch.randperm(K, generator=g, device=DEV)[:max(1, K // 50)]] = 37.0
    return (torch.randn((M, K), generator=g, device=DEV) * s).to(dtype)


def perm_of(g, K):
    return torch.randperm(K, generator=g, device=DEV).to(torch.int32)


def to64(t):
    return t.detach().cpu().double().numpy()


@pytest.fixture(autouse=True)
def no_device_error():
    yield
    assert clq.device_status() == 0


def check_quantized(q, v, slack=0.0):
    """q holds the codes of v (float64, [rows, K]); slack: relative error of the library's v."""
    fmt, block = q.fmt, ref.BLOCK[q.fmt]
    w = v.reshape(v.shape[0], -1, block)
    amax = np.abs(w).max(2)
    byte = ref.scale_bytes(q.scales, q.rows, q.K // block)
    if fmt == "block32":
        with np.errstate(divide="ignore"):
            e = np.maximum(np.ceil(np.log2(amax / 6)), -127)
        if slack == 0:
            np.testing.assert_array_equal(byte, e + 127)
        else:
            near = np.abs(np.log2(np.maximum(amax, 1e-300) / 6) - np.rint(np.log2(np.maximum(amax, 1e-300) / 6))) < 4 * slack
            assert np.all((byte == e + 127) | near)
    else:
        row = q.row_scale.cpu().numpy().astype(np.float64)
        np.testing.assert_allclose(row, np.maximum(amax.max(1) / 2688, 2.0 ** -100), rtol=2.0 ** -23 + slack)
        t = amax / (6 * row[:, None])
        step = np.where(t < 2.0 ** -6, 2.0 ** -9, 2.0 ** (np.floor(np.log2(np.maximum(t, 2.0 ** -6))) - 3))
        # nearest E4M3 value, up to the fp32 steps' error
        assert np.all(np.abs(ref.e4m3(byte) - np.minimum(t, 448)) <= step * 0.5 + t * (2.0 ** -21 + 2 * slack))
    s = ref.scales_of(q)
    x = np.where(s[:, :, None] > 0, w / np.where(s > 0, s, 1)[:, :, None], 0)
    code = ref.codes_of(q.codes).reshape(w.shape)
    miss = ref.nearest_slack(x, code)
    assert miss.max() <= (0 if fmt == "block32" and slack == 0 else 6 * 2.0 ** -21 + 12 * slack)


SHAPES = [(1, 32), (3, 64), (33, 96), (127, 160), (128, 1152), (129, 1184), (5, 4608), (2, 16384), (300, 256)]


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_quantize(fmt, M, K, dtype):
    X = rows_of(gen(M * K), M, K, dtype)
    q = mx.quantize(X, fmt)
    check_quantized(q, to64(X))
    for out in (F16, BF16):
        got, want = to64(mx.dequantize(q, out)), ref.values_of(q)
        eps = 2.0 ** -11 if out == F16 else 2.0 ** -8
        assert np.all(np.abs(got - want) <= np.abs(want) * eps * 1.001 + 2.0 ** -24)
    # blocks past the last one of a row have scale 0
    blocks = K // ref.BLOCK[fmt]
    assert np.all(ref.scale_bytes(q.scales, M, 4 * -(-blocks // 4))[:, blocks:] == 0)


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("M,K,b", [(2, 32, 32), (7, 96, 16), (65, 1152, 64), (40, 1152, 128), (9, 512, 256),
                                   (3, 16384, 256), (12, 160, 2), (12, 160, 1), (200, 4608, 8)])
@pytest.mark.parametrize("swap", [False, True])
def test_quantize_rotated(fmt, M, K, b, swap):
    """Inputs of few bits, so that the rotation is exact in fp32."""
    g = gen(K + b)
    X = (torch.randint(-64, 65, (M, K), generator=g, device=DEV) / 16).to(F16)
    perm = perm_of(g, K) if swap else None
    check_quantized(mx.quantize(X, fmt, perm, b), ref.hadamard(to64(X), perm, b))


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,K,b", [(6601, 1152, 64), (6601, 1152, 128), (120003, 64, 64), (117001, 128, 128), (900, 12288, 128),
                                   (12001, 704, 64), (2500, 4608, 64), (9001, 512, 128)])
def test_quantize_many_rows(fmt, dtype, M, K, b):
    """Many swapped and rotated rows take a kernel of their own: the same bytes as in small parts."""
    g = gen(M + b)
    big = rows_of(g, M, K + 8, dtype)
    X = big[:, :K]
    X[M // 3, 5], X[M // 2, 3] = float("inf"), float("nan")
    X[M // 5] = 0
    perm = perm_of(g, K)
    q = mx.quantize(X, fmt, perm, b)
    step = 128 * max(1, 60000 // K // 128)
    parts = [mx.quantize(X[i:i + step], fmt, perm, b) for i in range(0, M, step)]
    assert torch.equal(q.codes, torch.cat([p.codes for p in parts]))
    blocks = 4 * -(-K // (4 * ref.BLOCK[fmt]))
    got = ref.scale_bytes(q.scales, M, blocks)
    np.testing.assert_array_equal(got, np.concatenate([ref.scale_bytes(p.scales, p.rows, blocks) for p in parts]))
    if fmt == "block16":
        want = torch.cat([p.row_scale for p in parts])
        assert torch.equal(q.row_scale.nan_to_num(-1), want.nan_to_num(-1))
    # into other rows, some of them twice or nowhere
    T, k = M, 2
    rows = torch.stack((torch.randperm(M, generator=g, device=DEV), torch.full((M,), -1, device=DEV)), 1).to(torch.int32)
    rows[::2, 1] = M + torch.arange((M + 1) // 2, device=DEV).to(torch.int32)
    R = M + (M + 1) // 2
    out = mx._empty(R, K, fmt, DEV)
    P = lambda t: None if t is None else t.data_ptr()
    assert mx.clq_mx_quantize(P(X), 0 if dtype == F16 else 1, M, K, X.stride(0), P(perm), b, 0, mx.FORMATS[fmt], *map(P, out),
                              P(rows), k, R, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out[0][rows[:, 0].long()], q.codes) and torch.equal(out[0][M:], q.codes[::2])


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("M,K,b,swap", [(3, 96, 1, False), (130, 1536, 32, True)])
def test_quantize_activation(fmt, act, M, K, b, swap):
    g = gen(K)
    X = rows_of(g, M, 2 * K if act == "swiglu" else K, BF16)
    perm = perm_of(g, K) if swap else None
    v = ref.hadamard(ref.act(to64(X), act), perm, b)
    # the library's fp32 activation is within 2^-22 of |x|, and a rotation adds 32 of them: against
    # a block's largest value less than 2^-18 at these sizes
    check_quantized(mx.quantize(X, fmt, perm, b, act), v, slack=2.0 ** -18)


@pytest.mark.parametrize("fmt", ["block32", "block16"])
def test_quantize_gelu_tail(fmt):
    """Blocks of nothing but GELU's negative side, where 1 + erf would cancel."""
    K = 512
    X = -3 - 6 * torch.rand((40, K), generator=gen(2), device=DEV)
    X[:20] = X[:20].sort(1).values  # blocks of like sizes
    X = X.to(BF16)
    # exp's argument, up to 40, is rounded three times: 3 * 40 * 2^-24 of the value, and 2^-21 of it
    # for the rest
    check_quantized(mx.quantize(X, fmt, act="gelu"), ref.act(to64(X), "gelu"), slack=2.0 ** -17)


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
def test_quantize_activation_extremes(fmt, act):
    K = 96
    low, big = torch.finfo(BF16).min, torch.finfo(BF16).max
    X = torch.ones((5, 2 * K if act == "swiglu" else K), dtype=BF16, device=DEV)
    X[0, 1] = low  # nothing is left of it; its neighbours are as they would be
    X[1, 1] = big
    X[2, 1] = float("inf")
    X[3, 1] = float("nan")
    q = mx.quantize(X, fmt, act=act)
    v = mx.dequantize(q)
    one = ref.act(to64(X[4:]), act)[0, 0]
    assert v[0, 1] == 0 and q.codes[0, 0] >> 4 in (0, 8)
    unit = 2.0 ** -3 if fmt == "block32" else 2.0 ** -4  # of the largest, half a step between 4 and 6
    assert torch.all((v[0, 2:].double() - one).abs() <= unit * one) and torch.all((v[4].double() - one).abs() <= unit * one)
    if fmt == "block32":  # 1.99 * 2^127 is nearest to 4 * 2^126, which a float does not hold
        assert ref.scale_bytes(q.scales, 5, 3)[1, 0] == 253 and q.codes[1, 0] >> 4 == 6
    else:
        assert torch.isfinite(v[1]).all() and v[1, 1] >= 0.8 * big
    for row in (2, 3):
        first = 32 if fmt == "block32" else K
        assert v[row, :first].isnan().all() and torch.isfinite(v[row, first:]).all()


def test_quantize_extremes():
    K = 96
    X = torch.zeros((6, K), dtype=BF16, device=DEV)
    X[1, 40] = float("inf")
    X[2, 3] = float("nan")
    X[3] = torch.finfo(BF16).max
    X[4] = 2.0 ** -126
    X[5, :32] = 1e-30
    q = mx.quantize(X, "block32")
    byte = ref.scale_bytes(q.scales, 6, 3)
    assert byte[1].tolist() == [0, 255, 0] and byte[2].tolist() == [255, 0, 0]
    v = mx.dequantize(q)
    assert v[1, 32:64].isnan().all() and v[2, :32].isnan().all() and (v[1, :32] == 0).all()
    check_quantized(mx.quantize(X[3:], "block32"), to64(X[3:]))
    q = mx.quantize(X, "block16")
    v = mx.dequantize(q)
    assert v[1].isnan().all() and v[2].isnan().all() and (v[0] == 0).all() and (v[4] == 0).all()
    assert torch.isfinite(v[3]).all()


def test_quantize_strides_and_views():
    big = rows_of(gen(1), 50, 512, F16)
    X = big[3:20, 64:320]
    a, c = mx.quantize(X), mx.quantize(X.contiguous())
    assert torch.equal(a.codes, c.codes)
    np.testing.assert_array_equal(ref.scale_bytes(a.scales, 17, 8), ref.scale_bytes(c.scales, 17, 8))
    assert mx.quantize(X[:0]).codes.shape == (0, 128)


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("M,K,N", [
    (1, 32, 1), (1, 4096, 1000), (2, 64, 8), (31, 1184, 130), (32, 256, 128), (33, 288, 257), (127, 1152, 1152),
    (128, 96, 1003), (129, 512, 64), (255, 2048, 384), (511, 320, 264), (512, 320, 264), (600, 1152, 129),
    (1357, 1184, 1003), (2048, 4608, 1152), (513, 16384, 40)])
def test_linear(fmt, M, K, N):
    g = gen(M + N)
    dtype = F16 if (M + N) % 2 else BF16
    x = mx.quantize(rows_of(g, M, K, dtype), fmt)
    w = mx.quantize((0.05 * torch.randn((N, K), generator=g, device=DEV)).to(dtype), fmt)
    bias = torch.randn(N, generator=g, device=DEV).to(dtype) if N % 3 else None
    xv, wv = ref.values_of(x), ref.values_of(w)
    want = xv @ wv.T / 4
    if bias is not None:
        want = want + to64(bias)
    got = to64(mx.linear(x, w, bias, 4, dtype))
    bound = ref.product_bound(xv, wv, want, dtype, K)
    assert np.all(np.abs(got - want) <= bound), np.abs((got - want) / bound).max()


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("M", [1, 40, 700])
def test_linear_exact_codes(fmt, M):
    """Every code and many scales, sums that fp32 holds: the product is exact."""
    K, N = 640, 200
    g = gen(M)
    def tensor(rows):
        codes = torch.randint(0, 256, (rows, K // 2), generator=g, device=DEV, dtype=torch.uint8)
        # E8M0 2^-2 .. 2; E4M3 powers of two 2^-2 .. 2: sums of multiples of 2^-6 below 2^18
        pick = torch.tensor([125, 126, 127, 128] if fmt == "block32" else [40, 48, 56, 64], dtype=torch.uint8, device=DEV)
        scales = pick[torch.randint(0, 4, mx.scale_shape(rows, K, fmt), generator=g, device=DEV)]
        rs = torch.full((rows,), 0.5, device=DEV) if fmt == "block16" else None
        return mx.MXTensor(codes, scales, rs, fmt)
    x, w = tensor(M), tensor(N)
    want = ref.values_of(x) @ ref.values_of(w).T
    got = mx.linear(x, w, dtype=F16)
    wide = torch.from_numpy(want).float()
    assert torch.equal(got.cpu(), wide.to(F16))


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("M,K,N", [(20, 8192, 140), (70, 2048, 129), (300, 8192, 700), (600, 4096, 1100), (1500, 1152, 3456),
                                   (4096, 2048, 1152), (8192, 512, 1304)])
def test_linear_every_step_takes_its_own_scales(fmt, M, K, N):
    """Scales of 1 and 2 at random over many K steps, sums that fp32 holds: exact, in every tile shape."""
    g = gen(M + K)
    one, two = (127, 128) if fmt == "block32" else (56, 64)
    def tensor(rows):
        codes = torch.randint(0, 256, (rows, K // 2), generator=g, device=DEV, dtype=torch.uint8)
        pick = torch.randint(0, 2, mx.scale_shape(rows, K, fmt), generator=g, device=DEV)
        scales = (one + (two - one) * pick).to(torch.uint8)
        return mx.MXTensor(codes, scales, torch.ones(rows, device=DEV) if fmt == "block16" else None, fmt)
    x, w = tensor(M), tensor(N)
    rows = torch.randperm(M, generator=g, device=DEV)[:200].cpu().numpy()  # of the result
    want = ref.values_of(x)[rows] @ ref.values_of(w).T
    # multiples of 1/4 below 36 K: at most 4 * 36 * 8192 < 2^24 steps
    for _ in range(3):
        got = mx.linear(x, w, dtype=F16)[torch.from_numpy(rows).to(DEV)]
        assert torch.equal(got.cpu(), torch.from_numpy(want).to(torch.float32).to(F16))


def test_linear_nan_scale_stays_in_its_row():
    X = rows_of(gen(3), 300, 256, BF16)
    X[37, 100] = float("nan")
    w = mx.quantize(rows_of(gen(4), 96, 256, BF16))
    y = mx.linear(mx.quantize(X), w)
    bad = y.isnan().any(1)
    assert bad[37] and bad.sum() == 1 and y[37].isnan().all()


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("M,b", [(1, 64), (333, 128)])
def test_layer_rotated_is_near_full_precision(fmt, M, b):
    g = gen(b)
    K, N = 1152, 480
    X = rows_of(g, M, K, BF16)
    W = (0.02 * torch.randn((N, K), generator=g, device=DEV)).to(BF16)
    bias = torch.randn(N, generator=g, device=DEV).to(BF16)
    layer = mx.MXLinear.from_weight(W, fmt, perm_of(g, K), b, bias)
    y = to64(layer(X))
    want = to64(X) @ to64(W).T + to64(bias)
    # two operands of about 10 % quantization error each
    assert np.linalg.norm(y - want) / np.linalg.norm(want - to64(bias)) < 0.2


ROUTES = [
    # T, E, k, scoring, balance, groups, top_groups, group_top
    (1, 1, 1, "softmax", False, 1, 1, 2), (5, 8, 2, "softmax", False, 1, 1, 2), (33, 60, 4, "softmax", True, 4, 2, 2),
    (64, 64, 6, "sigmoid", True, 8, 3, 2), (100, 160, 6, "softmax", False, 8, 3, 1), (257, 256, 8, "sigmoid", True, 8, 4, 2),
    (31, 384, 8, "sigmoid", False, 1, 1, 2), (20, 512, 32, "softmax", False, 1, 1, 2), (9, 12, 12, "sigmoid", True, 12, 5, 2),
]


@pytest.mark.parametrize("case", ROUTES)
@pytest.mark.parametrize("dtype", [torch.float32, F16, BF16])
def test_route(case, dtype):
    T, E, k, scoring, balance, groups, top_groups, group_top = case
    g = gen(E)
    logits = torch.randn((T, E + 3), generator=g, device=DEV).to(dtype)[:, :E]
    logits[T // 2, ::2] = -float("inf")
    logits[T // 3] = -float("inf")
    bal = 0.1 * torch.randn(E, generator=g, device=DEV) if balance else None
    r = mx.route(logits, k, scoring, bal, groups, top_groups, group_top, scale=2.5)
    experts, weights, margin = ref.routing(to64(logits), None if bal is None else to64(bal), k, scoring, groups,
                                           top_groups, group_top, scale=2.5)
    # fp32 scores are within 2^-20 of the exact ones; a choice closer than that may fall either
    # way, and scores of 16-bit logits tie exactly: there the lowest index is asked for
    got = r.experts.cpu().numpy()
    clear = (margin > 2.0 ** -20) | (margin == 0)
    assert clear.mean() > 0.9
    np.testing.assert_array_equal(got[clear], experts[clear])
    np.testing.assert_allclose(r.weights.cpu().numpy()[clear], weights[clear], rtol=1e-5, atol=1e-9)


def test_route_extremes():
    inf, nan, big = float("inf"), float("nan"), torch.finfo(torch.float32).max
    L = torch.tensor([[1.0, nan, 2.0, -inf], [-inf] * 4, [-big] * 4, [inf, 0, inf, 0], [nan] * 4, [3.0] * 4], device=DEV)
    r = mx.route(L, 3)
    assert r.experts.tolist() == [[2, 0, -1], [-1] * 3, [0, 1, 2], [0, 2, 1], [-1] * 3, [0, 1, 2]]
    w = r.weights.cpu()
    assert w[1].tolist() == [0, 0, 0] and w[4].tolist() == [0, 0, 0]
    torch.testing.assert_close(w[2], torch.full((3,), 1 / 3))
    torch.testing.assert_close(w[3], torch.tensor([0.5, 0.5, 0]))
    s = mx.route(L, 3, "sigmoid", renormalize=False)
    assert s.experts.tolist() == r.experts.tolist()
    assert s.weights[3].tolist() == [1.0, 1.0, 0.5]
    assert mx.route(L[:0], 2).experts.shape == (0, 2)


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 4, 64), (33, 2, 4), (500, 8, 60), (512, 3, 512), (513, 3, 512),
                                   (3000, 4, 16), (9000, 2, 128)])
def test_plan(T, k, E):
    g = gen(T)
    experts = torch.rand((T, E), generator=g, device=DEV).argsort(1)[:, :k].to(torch.int32)
    experts[torch.rand((T, k), generator=g, device=DEV) < 0.1] = -1
    r = mx.Routing(experts.contiguous(), torch.ones((T, k), device=DEV), E)
    rows, space, R = mx.plan(r)
    e, rows = experts.cpu().numpy(), rows.cpu().numpy()
    want = np.full((T, k), -1)
    start = 0
    for x in range(E):
        t, j = np.nonzero(e == x)
        want[t, j] = start + np.arange(t.size)
        start += -(-t.size // 128) * 128
    np.testing.assert_array_equal(rows, want)
    assert start <= R


def experts_case(g, T, D, F, E, k, fmt, act, dtype, bias):
    N1 = 2 * F if act == "swiglu" else F
    W1 = (0.05 * torch.randn((E, N1, D), generator=g, device=DEV)).to(dtype)
    W2 = (0.05 * torch.randn((E, D, F), generator=g, device=DEV)).to(dtype)
    b1 = torch.randn((E, N1), generator=g, device=DEV).to(dtype) if bias else None
    b2 = torch.randn((E, D), generator=g, device=DEV).to(dtype) if bias else None
    return W1, W2, b1, b2


@pytest.mark.parametrize("T,D,F,E,k,fmt,act,bias", [
    (1, 256, 128, 8, 2, "block32", "swiglu", False), (7, 96, 64, 4, 4, "block16", "gelu", True),
    (32, 288, 160, 16, 3, "block32", "gelu", True), (33, 512, 96, 60, 6, "block16", "swiglu", True),
    (300, 1152, 288, 3, 2, "block32", "swiglu", True), (600, 256, 256, 5, 2, "block16", None, False),
    (700, 320, 544, 8, 3, "block32", "swiglu", False), (2000, 128, 128, 2, 1, "block16", "gelu", True)])
def test_experts(T, D, F, E, k, fmt, act, bias):
    g = gen(T + E)
    dtype = BF16 if T % 2 else F16
    W1, W2, b1, b2 = experts_case(g, T, D, F, E, k, fmt, act, dtype, bias)
    b = 32
    perm = perm_of(g, D)
    layer = mx.MXExperts.from_weights(W1, W2, fmt, act, perm, b, b1, b2)
    X = rows_of(g, T, D, dtype)
    logits = torch.randn((T, E), generator=g, device=DEV)
    logits[T // 2] = -float("inf")  # a token that no expert takes
    r = mx.route(logits, k)
    y = to64(layer(X, r))
    # step by step with the library's own quantized rows (checked above): products in 64 bits
    x = ref.values_of(mx.quantize(X, fmt, perm, b))
    e, w = r.experts.cpu().numpy(), to64(r.weights)
    want, bound = np.zeros((T, D)), np.zeros((T, D))
    eps = 2.0 ** -11 if dtype == F16 else 2.0 ** -8
    for i in range(E):
        t, j = np.nonzero(e == i)
        if not t.size:
            continue
        pick = lambda s: mx.MXTensor(s.codes[i], s.scales[i], None if s.row_scale is None else s.row_scale[i], fmt)
        w1, w2 = ref.values_of(pick(layer.w1)), ref.values_of(pick(layer.w2))
        h = torch.from_numpy(x[t] @ w1.T / b + (to64(b1[i]) if bias else 0)).to(dtype)
        a = ref.values_of(mx.quantize(h.to(DEV), fmt, act=act))
        v = a @ w2.T + (to64(b2[i]) if bias else 0)
        want[t] += w[t, j][:, None] * v
        bound[t] += w[t, j][:, None] * (np.abs(v) * eps + 2.0 ** -24)
    assert np.all(y[T // 2] == 0)
    # h may round to the neighbouring 16-bit value, and its code then to the neighbouring one: rare,
    # so most outputs agree to their rounding and all of them to a few percent of their size
    off = np.abs(y - want)
    close = off <= bound + eps * np.abs(want) + 1e-4 * np.sqrt(np.mean(want ** 2))
    assert close.mean() > 0.9
    assert np.linalg.norm(y - want) <= 1e-2 * np.linalg.norm(want)


@pytest.mark.parametrize("act", ["swiglu", "gelu", None])
@pytest.mark.parametrize("T,E,F,dtype", [(5, 4, 32, BF16), (32, 60, 96, F16), (33, 3, 160, BF16), (500, 4, 544, F16),
                                         (3000, 4, 288, BF16)])
def test_fused_activation_is_the_separate_one(act, T, E, F, dtype):
    """The product that quantizes its output against the product, then the quantization."""
    g, K, k = gen(T + F), 256, 2
    N = 2 * F if act == "swiglu" else F
    W = torch.stack([mx.quantize((0.1 * torch.randn((N, K), generator=g, device=DEV)).to(dtype)).codes for _ in range(E)])
    Ws = torch.full((E, *mx.scale_shape(N, K, "block32")), 123, dtype=torch.uint8, device=DEV)
    bias = torch.randn((E, N), generator=g, device=DEV).to(dtype)
    X = rows_of(g, T, K, dtype)
    r = mx.route(torch.randn((T, E), generator=g, device=DEV), k)
    rows, space, R = mx.plan(r)
    st, dt = torch.cuda.current_stream().cuda_stream, 0 if dtype == F16 else 1
    q = mx._empty(R, K, "block32", DEV)
    P = lambda t: t.data_ptr()
    assert mx.clq_mx_quantize(P(X), dt, T, K, K, None, 1, 0, 0, P(q[0]), P(q[1]), None, P(rows), k, R, st) == 0
    Y = torch.zeros((R, N), dtype=dtype, device=DEV)
    assert mx.clq_mx_grouped_linear(P(q[0]), P(q[1]), None, P(space), P(W), P(Ws), None, P(bias), T, k, E, N, K, 1, 0, dt,
                                    P(Y), st) == 0
    a = [torch.zeros_like(t) for t in mx._empty(R, F, "block32", DEV)[:2]]
    f = [torch.zeros_like(t) for t in a]
    assert mx.clq_mx_quantize_rows(P(Y), dt, P(space), T, k, E, F, N, mx.ACTS[act], 0, P(a[0]), P(a[1]), None, st) == 0
    assert mx.clq_mx_grouped_linear_act(P(q[0]), P(q[1]), P(space), P(W), P(Ws), P(bias), T, k, E, N, K, 1, dt,
                                        mx.ACTS[act], P(f[0]), P(f[1]), st) == 0
    used = rows.flatten().cpu().numpy()
    va, vf = (ref.values_of(mx.MXTensor(*t))[used] for t in (a, f))
    if act is None:
        np.testing.assert_array_equal(va, vf)
    # the activations differ by 2^-20 of |h| at most: a value between two codes (or a block's largest
    # value at a power of two) within that falls either way, about one in 2^17
    assert (va != vf).mean() < 2.0 ** -12
    blocks = F // 32
    pad = ref.scale_bytes(f[1], R, 4 * -(-blocks // 4))[used][:, blocks:]
    assert np.all(pad == 0)


def test_combine():
    g = gen(0)
    Y = torch.randn((256, 64), generator=g, device=DEV).to(F16)
    rows = torch.tensor([[3, -1], [255, 0]], dtype=torch.int32, device=DEV)
    w = torch.tensor([[0.5, 9.0], [2.0, -1.0]], device=DEV)
    out = torch.empty((2, 64), dtype=F16, device=DEV)
    assert mx.clq_mx_combine(Y.data_ptr(), 0, rows.data_ptr(), w.data_ptr(), 2, 2, 64, 256, out.data_ptr(),
                             torch.cuda.current_stream().cuda_stream) == 0
    want = torch.stack([0.5 * Y[3].double(), 2 * Y[255].double() - Y[0].double()])
    assert (out.double() - want).abs().max() <= 2.0 ** -10 * want.abs().max()


def test_bad_indices_are_reported():
    X = rows_of(gen(1), 4, 64, F16)
    perm = torch.arange(64, dtype=torch.int32, device=DEV)
    perm[5] = 64
    mx.quantize(X, perm=perm)
    assert clq.device_status() == 7
    perm[5] = -1
    mx.quantize(X, perm=perm)
    assert clq.device_status() == 7


def test_other_stream():
    g = gen(5)
    X, W = rows_of(g, 200, 512, BF16), rows_of(g, 256, 512, BF16)
    layer = mx.MXLinear.from_weight(W)
    want = layer(X)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = layer(X, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("fmt", ["block32", "block16"])
def test_example_runs(fmt):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "sparse_feed_forward.py")
    spec = importlib.util.spec_from_file_location("sparse_feed_forward", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    # three products in a row of operands with about 10 % error each, the middle one squared by the
    # gate: far from 1 still
    assert m.main(["--tokens", "300", "--hidden", "512", "--ffn", "256", "--experts", "4", "--format", fmt]) < 0.7
