"""Norm with the residual's addition and a quantised output on the GPU, against its definition in 64 bits, and
the 8-bit format's quantisation (block_utils)."""
import pytest
import torch

import block_utils as ref
from paper_2509_24416_gb300 import clq, mx

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
FORMATS = ["block32_e4m3", "block32", "block16"]
DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows_of(g, M, K, dtype, big=37.0):
    s = torch.ones(K, device=DEV)
    s[torch.randperm(K, generator=g, device=DEV)[:max(1, K // 50)]] = big
    return (torch.randn((M, K), generator=g, device=DEV) * s).to(dtype)


def perm_of(g, K):
    return torch.randperm(K, generator=g, device=DEV).to(torch.int32)


@pytest.fixture(autouse=True)
def no_device_error():
    yield
    assert clq.device_status() == 0


def rotated_off(v, perm, b, rel):
    """Error of v's rotation where each of its values is off by `rel` of itself and log2 b sums round."""
    a = v.abs() if perm is None else v.abs()[:, perm.long()]
    total = a.view(a.shape[0], -1, b).sum(2, keepdim=True).expand(-1, -1, b).reshape(a.shape)
    return total * (rel + (b.bit_length() - 1) * 2.0 ** -24) * 1.01


# of a normed value: the sum of squares 16 + 10 roundings and a product (their square root's half), the
# reciprocal root and two products; 2^-24 each, relative
NORM_OFF = 20 * 2.0 ** -24


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,K", [(1, 32), (3, 64), (33, 96), (127, 160), (300, 512), (129, 1184), (700, 1152), (5, 4608), (2, 16384),
                                 (2, 8224), (1500, 256)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("residual", [False, True])
def test_norm(fmt, M, K, dtype, residual):
    g = gen(M * K)
    X = rows_of(g, M, K, dtype)
    R = rows_of(g, M, K, dtype, 5.0) if residual else None
    w = (1 + 0.3 * torch.randn(K, generator=g, device=DEV)).to(dtype)
    h, v = ref.norm(X, R, w, 1e-5, dtype)
    q = mx.rms_norm(X, w, R, eps=1e-5, fmt=fmt)
    if residual:
        q, s = q
        assert torch.equal(s.double(), h)
    ref.check_codes(q, v, v.abs() * NORM_OFF)
    blocks = K // ref.BLOCK[fmt]
    full = mx.MXTensor(torch.zeros((M, 4 * -(-blocks // 4) * ref.BLOCK[fmt] // (1 if fmt == "block32_e4m3" else 2)),
                                   dtype=torch.uint8, device=DEV), q.scales, q.row_scale, fmt)
    assert (ref.scale_bytes(full)[:, blocks:] == 0).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,K,b", [(2, 32, 32), (7, 96, 16), (65, 1152, 64), (400, 1152, 128), (9, 512, 256), (3, 16384, 256),
                                   (12, 160, 2), (12, 160, 1), (200, 4608, 8), (2000, 576, 64)])
@pytest.mark.parametrize("swap,residual", [(False, True), (True, False), (True, True)])
def test_norm_rotated(fmt, M, K, b, swap, residual):
    g = gen(K + b)
    X = rows_of(g, M, K, BF16)
    R = rows_of(g, M, K, BF16, 3.0) if residual else None
    w = (1 + 0.3 * torch.randn(K, generator=g, device=DEV)).to(BF16)
    perm = perm_of(g, K) if swap else None
    h, v = ref.norm(X, R, w, 1e-6, BF16)
    q = mx.rms_norm(X, w, R, fmt=fmt, perm=perm, b=b)
    q = q[0] if residual else q
    ref.check_codes(q, ref.hadamard(v, perm, b), rotated_off(v, perm, b, NORM_OFF))


MANY = [(6601, 1152, 64), (9001, 1152, 128), (12003, 640, 64), (14001, 512, 128), (900, 10240, 128), (3001, 4608, 64), (20001, 96, 32),
        (2500, 8000, 64)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,K,b", MANY)
@pytest.mark.parametrize("residual", [False, True])
def test_norm_many_rows(fmt, dtype, M, K, b, residual):
    """Many swapped and rotated rows, several a block: the same bytes as in small parts, some of one row."""
    g = gen(M + b)
    X = rows_of(g, M, K + 8, dtype)[:, :K]
    R = rows_of(g, M, 2 * K, dtype, 3.0)[:, K:] if residual else None
    X[M // 3, 5], X[M // 2, 3] = float("inf"), float("nan")
    X[M // 5] = 0
    if dtype == BF16:
        X[M // 7, 9], X[M // 6] = 1e25, 3e38
    w = (1 + 0.3 * torch.randn(K, generator=g, device=DEV)).to(dtype)
    perm = perm_of(g, K)
    call = lambda i, j: mx.rms_norm(X[i:j], w, R[i:j] if residual else None, fmt=fmt, perm=perm, b=b)
    q, step = call(0, M), 128 * max(1, M // 9 // 128)
    parts = [call(i, min(M, i + step)) for i in range(0, M, step)]
    for i in (0, M // 5, M - 1):  # (a block of its own has whole warps)
        one = call(i, i + 1)
        assert torch.equal((one[0] if residual else one).codes[0], (q[0] if residual else q).codes[i])
    if residual:
        q, s = q
        assert torch.equal(s, (X.float() + R.float()).to(dtype)) or s.isnan().any()
        assert torch.equal(s.nan_to_num(0), torch.cat([p[1] for p in parts]).nan_to_num(0))
        parts = [p[0] for p in parts]
    assert torch.equal(q.codes, torch.cat([p.codes for p in parts]))
    assert torch.equal(ref.scale_bytes(q), torch.cat([ref.scale_bytes(p) for p in parts]))
    if fmt == "block16":
        assert torch.equal(q.row_scale.nan_to_num(-1), torch.cat([p.row_scale for p in parts]).nan_to_num(-1))
    keep = torch.tensor([0, 1, M // 5, M // 4, M - 1] + ([M // 7] if dtype == BF16 else []), device=DEV)
    h, v = ref.norm(X[keep], R[keep] if residual else None, w, 1e-6, dtype)
    few = mx.MXTensor(q.codes[keep].contiguous(), torch.zeros(mx.scale_shape(len(keep), K, fmt), dtype=torch.uint8, device=DEV),
                      q.row_scale[keep].contiguous() if fmt == "block16" else None, fmt)
    r, c = torch.arange(len(keep), device=DEV)[:, None], torch.arange(K // ref.BLOCK[fmt], device=DEV)[None, :]
    few.scales[r // 128, c // 4, r % 32, r % 128 // 32, c % 4] = ref.scale_bytes(q)[keep].to(torch.uint8)
    ref.check_codes(few, ref.hadamard(v, perm, b), rotated_off(v, perm, b, NORM_OFF))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,K", [(700, 8224), (470, 16384), (305, 9216)])
def test_wide_rows_in_place(fmt, M, K):
    """Rows that are a block each, several a block, summed in place: the same bytes as in small parts."""
    g = gen(M)
    X, R = rows_of(g, M, K, BF16), rows_of(g, M, K + 16, BF16, 3.0)[:, :K]
    parts = [mx.rms_norm(X[i:i + 128].clone(), None, R[i:i + 128].clone(), fmt=fmt) for i in range(0, M, 128)]
    for place in (R, X):
        x, r = X.clone(), R.clone()
        q, s = mx.rms_norm(x, None, r, fmt=fmt, out=r if place is R else x)
        assert torch.equal(s, (X.float() + R.float()).to(BF16)) and torch.equal(q.codes, torch.cat([p[0].codes for p in parts]))
        assert torch.equal(ref.scale_bytes(q), torch.cat([ref.scale_bytes(p[0]) for p in parts]))
    v = ref.norm(X, R, None, 1e-6, BF16)[1]
    ref.check_codes(q, v, v.abs() * NORM_OFF)


def test_many_rows_in_place():
    g = gen(11)
    M = 14001
    X, R = rows_of(g, M, 1152, BF16), rows_of(g, M, 1152, BF16)
    perm = perm_of(g, 1152)
    want, s = mx.rms_norm(X, None, R, perm=perm, b=64)
    for place in ("residual", "input"):
        x, r = X.clone(), R.clone()
        q, t = mx.rms_norm(x, None, r, perm=perm, b=64, out=r if place == "residual" else x)
        assert torch.equal(q.codes, want.codes) and torch.equal(t, s)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,K,b", [(6601, 1152, 64), (6601, 1152, 128), (900, 12288, 128), (12001, 704, 64)])
def test_quantize_e4m3_many_rows(dtype, M, K, b):
    g = gen(M + b)
    X = rows_of(g, M, K + 8, dtype)[:, :K]
    X[M // 3, 5], X[M // 2, 3], X[M // 5] = float("inf"), float("nan"), 0
    perm = perm_of(g, K)
    q, step = mx.quantize(X, "block32_e4m3", perm, b), 128 * max(1, 60000 // K // 128)
    parts = [mx.quantize(X[i:i + step], "block32_e4m3", perm, b) for i in range(0, M, step)]
    assert torch.equal(q.codes, torch.cat([p.codes for p in parts]))
    assert torch.equal(ref.scale_bytes(q), torch.cat([ref.scale_bytes(p) for p in parts]))
    blocks = K // 32
    if blocks % 4:
        assert (q.scales[:, -1, :, :, blocks % 4:].transpose(1, 2).reshape(-1, 4 - blocks % 4)[:M] == 0).all()


def test_rows_apart_and_in_place():
    """Strides of input, residual and sum that are not K; the sum over the residual, and over the input."""
    g = gen(3)
    big = rows_of(g, 70, 3 * 640, BF16)
    X, R, S = big[:, :640], big[:, 640:1280], torch.zeros((70, 1000), dtype=BF16, device=DEV)[:, 8:648]
    q, s = mx.rms_norm(X, None, R, out=S)
    q2, s2 = mx.rms_norm(X.contiguous(), None, R.contiguous())
    assert s is S and torch.equal(s, s2) and torch.equal(q.codes, q2.codes)
    assert torch.equal(ref.scale_bytes(q), ref.scale_bytes(q2))  # (bytes of rows past the last are anything)
    for place in ("residual", "input"):
        x, r = X.clone(), R.clone()
        to = r if place == "residual" else x
        q3, s3 = mx.rms_norm(x, None, r, out=to)
        assert s3 is to and torch.equal(s3, s2) and torch.equal(q3.codes, q2.codes)


@pytest.mark.parametrize("fmt", FORMATS)
def test_extremes(fmt):
    """Rows of zeros, of the largest and smallest values, with an infinity and a NaN; a row's neighbours keep theirs."""
    K = 1152
    g = gen(9)
    X = rows_of(g, 9, K, BF16)
    clean = mx.rms_norm(X, fmt=fmt)
    X[1] = 0
    X[2] = 3e38
    X[3] = 1e-30
    X[4, 7] = 1e25  # whose square fp32 does not hold
    X[5, 100] = float("inf")
    X[6, 100] = float("nan")
    q = mx.rms_norm(X, fmt=fmt)
    for i in (0, 7, 8):
        assert torch.equal(q.codes[i], clean.codes[i])
    keep = [0, 1, 2, 3, 4, 7, 8]
    h, v = ref.norm(X[keep], None, None, 1e-6, BF16)
    part = mx.rms_norm(X[keep].contiguous(), fmt=fmt)
    assert torch.equal(part.codes, q.codes[keep])
    ref.check_codes(part, v, v.abs() * NORM_OFF)
    d = ref.values(q)
    assert (d[1] == 0).all() and d[2].abs().sub(1).abs().max() < 0.1
    # as the formula has it: 0 beside an infinity (block16: its row's scale covers them all), NaN beside a NaN
    assert d[6].isnan().all()
    assert d[5, 96:112].isnan().all() and (d[5].isnan().all() if fmt == "block16" else (d[5, 128:] == 0).all())


def test_eps_counts():
    X = torch.full((4, 64), 2.0 ** -10, dtype=F16, device=DEV)
    for eps in (1e-8, 1e-6, 1e-2, 1e30):
        h, v = ref.norm(X, None, None, eps, F16)
        ref.check_codes(mx.rms_norm(X, eps=eps), v, v.abs() * NORM_OFF)


def test_sum_alone_rounds_once():
    """Sums that lie between two numbers of the type: to the even one, and the norm is that number's."""
    X = torch.full((3, 32), 1.0, dtype=BF16, device=DEV)
    R = torch.tensor([2.0 ** -8, 3 * 2.0 ** -8, 2.0 ** -9], device=DEV).to(BF16)[:, None].expand(3, 32).contiguous()
    q, s = mx.rms_norm(X, None, R)
    assert s[:, 0].tolist() == [1.0, 1.0 + 4 * 2.0 ** -8, 1.0]


def test_index_outside_is_reported():
    X = torch.ones((4, 64), dtype=F16, device=DEV)
    perm = torch.arange(64, device=DEV).to(torch.int32)
    perm[5] = 64
    mx.rms_norm(X, perm=perm)
    torch.cuda.synchronize()
    assert clq.device_status() == 7  # and is cleared by the look at it


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,K", [(1, 32), (127, 160), (129, 1184), (5, 4608), (2, 16384), (3000, 256)])
def test_quantize_e4m3(dtype, M, K):
    X = rows_of(gen(K), M, K, dtype)
    q = mx.quantize(X, "block32_e4m3")
    assert q.codes.shape == (M, K) and q.K == K
    ref.check_codes(q, X.double(), torch.zeros_like(X.double()))
    for out in (F16, BF16):
        got, want = mx.dequantize(q, out).double(), ref.values(q)
        assert ((got - want).abs() <= want.abs() * ref.HALF_STEP[out] + ref.TINY[out]).all()


@pytest.mark.parametrize("M,K,b", [(7, 96, 16), (65, 1152, 64), (9, 512, 256), (6601, 1152, 64)])
def test_quantize_e4m3_rotated(M, K, b):
    g = gen(K + b)
    X = (torch.randint(-64, 65, (M, K), generator=g, device=DEV) / 16).to(F16)
    perm = perm_of(g, K)
    v = ref.hadamard(X.double(), perm, b)
    ref.check_codes(mx.quantize(X, "block32_e4m3", perm, b), v, torch.zeros_like(v))


def test_quantize_e4m3_every_value():
    """Every finite 16-bit value, alone in its block and beside a larger one; the bytes of the type's own conversion."""
    for dtype in (F16, BF16):
        v = torch.arange(-32768, 32768, device=DEV, dtype=torch.int16).view(dtype)
        v = v[torch.isfinite(v)]
        X = torch.zeros((v.numel(), 64), dtype=dtype, device=DEV)
        X[:, 3], X[:, 40], X[:, 41] = v, v, 100.0
        q = mx.quantize(X, "block32_e4m3")
        ref.check_codes(q, X.double(), torch.zeros_like(X.double()))
        s = ref.scales(q)[:, 1]
        big = v.abs() <= 100
        want = (v.float() / s.float()).to(torch.float8_e4m3fn).view(torch.uint8)
        zero = v == 0
        assert torch.equal(q.codes[:, 40][big & ~zero], want[big & ~zero]) and (q.codes[:, 40][zero] == 0).all()
    X = torch.ones((2, 64), dtype=F16, device=DEV)
    X[0, 3], X[1, 40] = float("inf"), float("nan")
    q = mx.quantize(X, "block32_e4m3")
    assert ref.scale_bytes(q).tolist() == [[255, 119], [119, 255]] and (q.codes[0, :32] == 0).all()
    assert mx.dequantize(q).isnan().sum() == 64


@pytest.mark.parametrize("M,K,b", [(50, 160, 1), (50, 160, 32), (14001, 1152, 64), (14001, 1152, 128)])
def test_quantize_e4m3_into_rows(M, K, b):
    """Each row into two others or nowhere, through clq_mx_quantize; what is in no row's place stays."""
    g = gen(M)
    X = rows_of(g, M, K, F16)
    perm = perm_of(g, K) if b > 1 else None
    q = mx.quantize(X, "block32_e4m3", perm, b)
    rows = torch.randperm(3 * M, generator=g, device=DEV)[:2 * M].view(M, 2).to(torch.int32)
    rows[::3, 1] = -1
    out = mx._empty(3 * M, K, "block32_e4m3", DEV)
    out[0].fill_(0xAB), out[1].fill_(0xCD)
    P = lambda t: None if t is None else t.data_ptr()
    assert mx.clq_mx_quantize(P(X), 0, M, K, K, P(perm), b, 0, mx.FORMATS["block32_e4m3"], P(out[0]), P(out[1]), None, P(rows), 2,
                              3 * M, torch.cuda.current_stream().cuda_stream) == 0
    t = mx.MXTensor(out[0], out[1], None, "block32_e4m3")
    left = torch.ones(3 * M, dtype=torch.bool, device=DEV)
    for j in range(2):
        at = rows[:, j]
        to = at[at >= 0].long()
        left[to] = False
        assert torch.equal(out[0][to], q.codes[at >= 0])
        assert torch.equal(ref.scale_bytes(t)[to], ref.scale_bytes(q)[at >= 0])
    assert (out[0][left] == 0xAB).all() and (ref.scale_bytes(t)[left] == 0xCD).all()


@pytest.mark.parametrize("act", ["gelu", "swiglu"])
def test_quantize_e4m3_activation(act):
    g = gen(4)
    X = rows_of(g, 130, 2 * 1536 // 2 if act == "gelu" else 2 * 1536, BF16)
    v, e = ref.post(X.double(), torch.zeros_like(X.double()), act)
    ref.check_codes(mx.quantize(X, "block32_e4m3", act=act), v, e)


@pytest.mark.parametrize("fmt", FORMATS)
def test_streams_and_graphs(fmt):
    """On another stream than the caller's, and captured once, replayed on new contents."""
    g = gen(5)
    X, R = rows_of(g, 64, 640, BF16), rows_of(g, 64, 640, BF16)
    want, s = mx.rms_norm(X, None, R, fmt=fmt)
    side = torch.cuda.Stream()
    got, t = mx.rms_norm(X, None, R, fmt=fmt, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got.codes, want.codes) and torch.equal(t, s)
    x, r = torch.zeros_like(X), torch.zeros_like(R)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, o = mx.rms_norm(x, None, r, fmt=fmt)
    for _ in range(2):
        x.copy_(X), r.copy_(R)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q.codes, want.codes) and torch.equal(o, s)
        assert torch.equal(ref.scale_bytes(q), ref.scale_bytes(want))
        x.zero_()


def test_empty():
    q = mx.rms_norm(torch.zeros((0, 64), dtype=F16, device=DEV))
    assert q.codes.shape == (0, 64)
    q, s = mx.rms_norm(torch.zeros((0, 64), dtype=F16, device=DEV), None, torch.zeros((0, 64), dtype=F16, device=DEV))
    assert s.shape == (0, 64)


def test_sums_over_other_rows_are_refused():
    """Nothing is launched, and what lies there stays; a sum beside its inputs, in the same rows, is taken."""
    g = gen(21)
    M, K = 70, 640
    space = rows_of(g, M + 8, 3 * K, BF16)
    before = space.clone()
    X, R = space[:M, :K], space[:M, K:2 * K]
    for out in (space[1:M + 1, :K], space[8:, :K], space[3:M + 3, K:2 * K], space[:M, 8:K + 8], space[:M, K - 8:2 * K - 8],
                space.view(-1)[K:K + M * (K + 8)].view(M, K + 8)[:, :K]):
        with pytest.raises(clq.ClqError):
            mx.rms_norm(X, None, R, out=out)
    torch.cuda.synchronize()
    assert torch.equal(space, before)
    want, s = mx.rms_norm(X.contiguous(), None, R.contiguous())
    for out in (space[8:, 2 * K:], space[:M, 2 * K:], space[:M, K:2 * K]):
        q, h = mx.rms_norm(X, None, R, out=out)
        assert h is out and torch.equal(h, s) and torch.equal(q.codes, want.codes)
        space.copy_(before)


def same(a, b):
    """The same numbers, NaN in the same places."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0, 1e30, -1e30), b.nan_to_num(0, 1e30, -1e30))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,K,b", [(2, 32, 32), (7, 96, 16), (65, 1152, 64), (9, 512, 256), (3, 16384, 256), (12, 160, 1), (200, 4608, 8),
                                   (2000, 576, 64)] + MANY)
@pytest.mark.parametrize("place", ["new", "residual", "input"])
def test_swapped_sums(fmt, dtype, M, K, b, place):
    """The stored sum beside a swap, by its definition, with infinities and NaN in it; rows that are alone in a block, of
    whole warps, and that share warps."""
    g = gen(M + K + b)
    X, R = rows_of(g, M, K, dtype), rows_of(g, M, K, dtype, 3.0)
    X[M // 2, 3], X[M // 3, K - 1], R[M - 1, K // 2] = float("nan"), float("inf"), float("-inf")
    R[M // 3, K - 1] = float("-inf")
    want = (X.float() + R.float()).to(dtype)
    out = {"new": None, "residual": R, "input": X}[place]
    q, s = mx.rms_norm(X, None, R, fmt=fmt, perm=perm_of(g, K), b=b, out=out)
    assert out is None or s is out
    assert same(s, want) and want.isnan().any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,K", [(1, 32), (33, 96), (300, 512), (700, 1152), (2, 16384), (470, 8224)])
def test_sums(fmt, M, K):
    """The same without a swap."""
    g = gen(M + K)
    X, R = rows_of(g, M, K, F16), rows_of(g, M, K, F16, 3.0)
    X[M // 2, 3], R[M - 1, K // 2] = float("nan"), float("inf")
    assert same(mx.rms_norm(X, None, R, fmt=fmt)[1], (X.float() + R.float()).to(F16))


@pytest.mark.parametrize("fmt", FORMATS)
def test_on_another_stream(fmt):
    """On another stream, which has waited for the inputs, beside work on the first."""
    g = gen(25)
    X, R = rows_of(g, 300, 640, BF16), rows_of(g, 300, 640, BF16)
    perm = perm_of(g, 640)
    want, s = mx.rms_norm(X, None, R, fmt=fmt, perm=perm, b=64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [mx.rms_norm(X, None, R, fmt=fmt, perm=perm, b=64, stream=side) for _ in range(8)]
    torch.cuda.current_stream().wait_stream(side)
    for q, t in got:
        assert torch.equal(q.codes, want.codes) and torch.equal(ref.scale_bytes(q), ref.scale_bytes(want)) and torch.equal(t, s)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-36, 1e-30])
def test_rows_of_small_values(fmt, eps):
    """Squares around and below the smallest numbers of fp32, beside the smallest eps; a smaller one is refused."""
    g = gen(27)
    sizes = 10.0 ** torch.arange(-38, -12, 0.5, device=DEV, dtype=torch.float64)
    X = (torch.randn((len(sizes), 1152), generator=g, device=DEV).double() * sizes[:, None]).to(BF16)
    v = ref.norm(X, None, None, eps, BF16)[1]
    # a square below 2^-126 is off by 2^-150, so is their mean, of which the root counts half: 2^-25 beside eps
    ref.check_codes(mx.rms_norm(X, eps=eps, fmt=fmt), v, v.abs() * (NORM_OFF + 2.0 ** -24))
    with pytest.raises(clq.ClqError):
        mx.rms_norm(X, eps=2.0 ** -127, fmt=fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,K,swap", [(1, 32, False), (70, 96, False), (70, 96, True), (129, 1184, True), (6601, 1152, True)])
def test_codes_fill_their_bytes(fmt, M, K, swap):
    """The C calls write the sizes that their header states, all of the codes and nothing behind any array."""
    g = gen(M + K)
    X, R = rows_of(g, M, K, F16), rows_of(g, M, K, F16)
    perm = perm_of(g, K) if swap else None
    f, b = mx.FORMATS[fmt], 32 if swap else 1
    P = lambda t: None if t is None else t.data_ptr()
    code_bytes, scale_bytes = M * (K if fmt == "block32_e4m3" else K // 2), mx.load().clq_mx_scale_bytes(M, K, f)
    stream = torch.cuda.current_stream().cuda_stream
    for call in ("quantize", "norm"):
        got = []
        for fill in (0x11, 0xEE):
            codes = torch.full((code_bytes + 256,), fill, dtype=torch.uint8, device=DEV)
            scales = torch.full((scale_bytes + 256,), fill, dtype=torch.uint8, device=DEV)
            rows = torch.full((M + 64,), float(fill), device=DEV) if fmt == "block16" else None
            total = torch.full((M * K + 64,), float(fill), dtype=F16, device=DEV)
            if call == "quantize":
                assert mx.clq_mx_quantize(P(X), 0, M, K, K, P(perm), b, 0, f, P(codes), P(scales), P(rows), None, 0, M, stream) == 0
            else:
                assert mx.clq_mx_rms_norm(P(X), 0, M, K, K, P(R), K, None, 1e-6, P(perm), b, f, P(codes), P(scales), P(rows), P(total), K,
                                          stream) == 0
                assert (total[M * K:] == fill).all()
            assert (codes[code_bytes:] == fill).all() and (scales[scale_bytes:] == fill).all()
            assert rows is None or (rows[M:] == fill).all()
            got.append((codes[:code_bytes], rows[:M] if rows is not None else codes[:0], total[:M * K] if call == "norm" else codes[:0]))
        for a, c in zip(*got):
            assert torch.equal(a, c)
