"""The microscaled product with an activation and a residual behind it, and the 8-bit product, on the GPU against
their definitions in 64 bits (block_utils), in every tile; and the layer that runs norm, product and positions."""
import pytest
import torch

import block_utils as ref
import block_tiles as tiles
from paper_2509_24416_gb300 import clq, mx, rope

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
FORMATS = ["block32_e4m3", "block32", "block16"]
DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows_of(g, M, K, dtype, size=1.0):
    s = torch.full((K,), size, device=DEV)
    s[torch.randperm(K, generator=g, device=DEV)[:max(1, K // 50)]] *= 20
    return (torch.randn((M, K), generator=g, device=DEV) * s).to(dtype)


@pytest.fixture(autouse=True)
def no_device_error():
    yield
    assert clq.device_status() == 0


@pytest.fixture(scope="module")
def picks(tmp_path_factory):
    return tiles.library(tmp_path_factory.mktemp("tiles"))


def operands(g, M, K, N, fmt, dtype, bias):
    x = mx.quantize(rows_of(g, M, K, dtype), fmt)
    w = mx.quantize(rows_of(g, N, K, BF16, 0.1), fmt)
    return x, w, (torch.randn(N, generator=g, device=DEV).to(dtype) if bias else None)


def check(Y, x, w, bias, b, post, residual):
    want, room = ref.product(x, w, bias, b, post, residual, Y.dtype)
    off = (Y.double() - want).abs()
    # what is past the type's largest number and half a step (fp16: 65504 + 16) rounds to an infinity
    top = torch.finfo(Y.dtype).max * (1 + torch.finfo(Y.dtype).eps / 4)
    infinite = Y.isinf() & (Y.sign() == want.sign()) & (want.abs() + room >= top)
    assert ((off <= room) | infinite).all(), float((off - room)[~infinite].max())


# M, K, N, tile.  Among them, for the tiles of 192 and 256 rows: last tiles of 64, 128 and 192 columns, tiles that
# begin in the middle of a scale block, one and several a pair, outputs whose rows are 16-byte aligned and not.
FEW = [(1, 512, 64, (32, 1, 1)), (20, 1024, 144, (32, 1, 1)), (20, 1024, 140, (32, 1, 1)), (600, 160, 144, (64, 1, 1)), (600, 288, 129, (64, 1, 1))]
STORED = FEW + [
    (5017, 64, 131, (128, 1, 1)), (3822, 64, 272, (128, 1, 1)), (5042, 1184, 148, (128, 2, 1)), (2702, 1184, 400, (128, 2, 1)),
    (6939, 160, 267, (192, 2, 1)), (2664, 160, 944, (192, 2, 1)), (8192, 4608, 1152, (192, 2, 1)), (3424, 64, 2049, (256, 1, 1)),
    (3423, 64, 2064, (256, 1, 1)), (8107, 64, 2057, (256, 2, 1)), (2752, 160, 2592, (256, 2, 1))]
POST8 = FEW + [
    (7399, 64, 401, (128, 1, 1)), (3369, 64, 1088, (128, 1, 1)), (5061, 288, 133, (128, 2, 1)), (3442, 288, 320, (128, 2, 1)),
    (7285, 288, 257, (192, 2, 1)), (4011, 64, 2480, (192, 2, 1)), (8192, 4608, 1152, (192, 2, 1)), (3014, 64, 3988, (256, 1, 1)),
    (3666, 64, 3600, (256, 1, 1)), (7364, 1184, 262, (256, 2, 1)), (8166, 1184, 352, (256, 2, 1))]
POST4 = FEW + [
    (4369, 64, 774, (128, 1, 1)), (7482, 64, 608, (128, 1, 1)), (5230, 544, 129, (128, 2, 1)), (4891, 544, 160, (128, 2, 1)),
    (3944, 64, 533, (192, 2, 1)), (1929, 64, 1392, (192, 2, 1)), (6466, 64, 1066, (256, 1, 1)), (4743, 64, 1616, (256, 1, 1)),
    (2726, 544, 2580, (256, 2, 1)), (3017, 544, 2480, (256, 2, 1))]
# Tiles whose K steps several CTAs share, evenly and not, with last steps cut short.
SHARED8 = [
    (5, 4640, 9008, (32, 1, 2)), (1, 4608, 1152, (32, 1, 4)), (17, 4640, 300, (32, 1, 4)), (3, 2208, 1003, (32, 1, 4)),
    (1, 12288, 144, (32, 1, 8)), (32, 16384, 1151, (32, 1, 8)), (256, 4096, 1024, (64, 1, 2)), (1000, 4608, 259, (64, 1, 2)),
    (33, 4640, 259, (64, 1, 4)), (130, 16384, 144, (64, 1, 4))]
SHARED4 = [
    (5, 9120, 9008, (32, 1, 2)), (1, 4160, 1008, (32, 1, 4)), (31, 4640, 1000, (32, 1, 4)), (9, 9120, 137, (32, 1, 4)),
    (640, 9120, 384, (64, 1, 2)), (600, 9184, 401, (64, 1, 2)), (200, 8160, 144, (64, 1, 4)), (77, 9120, 257, (64, 1, 4))]


@pytest.mark.parametrize("M,K,N,tile", STORED + SHARED8)
def test_every_tile_stored(picks, M, K, N, tile):
    assert tiles.tile(picks, M, N, K, "block32_e4m3", False) == tile
    dtype = BF16 if (M + N) % 2 else F16
    x, w, bias = operands(gen(M + N + K), M, K, N, "block32_e4m3", dtype, M % 3 != 0)
    check(mx.linear(x, w, bias, dtype=dtype), x, w, bias, 1, None, None)


@pytest.mark.parametrize("fmt,M,K,N,tile", [("block32_e4m3",) + s for s in POST8 + SHARED8] + [
    (f,) + s for f in ("block32", "block16") for s in POST4 + SHARED4])
@pytest.mark.parametrize("post,residual", [(None, True), ("gelu", False), ("gelu", True), ("swiglu", False), ("swiglu", True)])
def test_every_tile(picks, fmt, M, K, N, tile, post, residual):
    if post == "swiglu" and N % 16:
        pytest.skip("a gated product has a multiple of 16 channels")
    assert tiles.tile(picks, M, N, K, fmt, True) == tile
    dtype = BF16 if (M + N) % 2 else F16
    g = gen(M + N + K)
    x, w, bias = operands(g, M, K, N, fmt, dtype, M % 3 != 0)
    columns = N // 2 if post == "swiglu" else N
    R = rows_of(g, M, columns, dtype, 3.0) if residual else None
    check(mx.linear(x, w, bias, dtype=dtype, post=post, residual=R), x, w, bias, 1, post, R)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K", [32, 64, 96, 128, 160, 192, 224, 256, 288, 2080, 16384])
def test_lengths_of_a_row(fmt, K):
    g = gen(K)
    for M, N in ((1, 8), (130, 200)):
        x, w, bias = operands(g, M, K, N, fmt, F16, True)
        R = rows_of(g, M, N, F16)
        check(mx.linear(x, w, bias, dtype=F16), x, w, bias, 1, None, None)
        check(mx.linear(x, w, bias, dtype=F16, post="gelu", residual=R), x, w, bias, 1, "gelu", R)


@pytest.mark.parametrize("post", [None, "gelu", "swiglu"])
@pytest.mark.parametrize("M,N", [(1, 16), (5, 48), (33, 80), (64, 1040), (129, 16), (257, 496), (2, 16400)])
def test_few_rows_and_columns(post, M, N):
    g = gen(M * N)
    x, w, bias = operands(g, M, 256, N, "block32_e4m3", BF16, True)
    R = rows_of(g, M, N // 2 if post == "swiglu" else N, BF16)
    check(mx.linear(x, w, bias, post=post, residual=R), x, w, bias, 1, post, R)


@pytest.mark.parametrize("post", [None, "swiglu"])
@pytest.mark.parametrize("M,N", [(20, 144), (600, 144), (6000, 272), (4011, 2480)])
@pytest.mark.parametrize("lead,stride", [(0, 0), (8, 8), (1, 0), (0, 1), (3, 5), (2, 4), (4, 8)])
def test_residuals_of_any_stride(post, M, N, lead, stride):
    g = gen(M + stride)
    x, w, bias = operands(g, M, 96, N, "block32_e4m3", F16, True)
    columns = N // 2 if post == "swiglu" else N
    flat = torch.randn(lead + M * (columns + stride), generator=g, device=DEV).to(F16)
    R = flat[lead:].view(M, columns + stride)[:, :columns]
    Y = mx.linear(x, w, bias, dtype=F16, post=post, residual=R)
    assert torch.equal(Y, mx.linear(x, w, bias, dtype=F16, post=post, residual=R.contiguous()))
    check(Y, x, w, bias, 1, post, R)


@pytest.mark.parametrize("post", [None, "gelu", "swiglu"])
@pytest.mark.parametrize("M,N", [(20, 144), (600, 129), (6000, 272), (8023, 1003), (8023, 2064)])
def test_onto_the_residual(post, M, N):
    """Y in the residual's place, and rows around both that stay."""
    if post == "swiglu":
        N = N // 16 * 16
    g = gen(M + N)
    x, w, bias = operands(g, M, 160, N, "block32_e4m3", BF16, True)
    columns = N // 2 if post == "swiglu" else N
    space = torch.randn((M + 64, columns), generator=g, device=DEV).to(BF16)
    before = space.clone()
    lead = 8  # 8 rows keep the address a multiple of 16 bytes
    want = mx.linear(x, w, bias, post=post, residual=before[lead:lead + M])
    Y = space[lead:lead + M]
    assert mx.linear(x, w, bias, Y=Y, post=post, residual=Y) is Y
    assert torch.equal(Y, want)
    assert torch.equal(space[:lead], before[:lead]) and torch.equal(space[lead + M:], before[lead + M:])


def test_rotated_layer():
    """A layer with swap and rotation, an activation in front and one behind: as its steps one by one."""
    g = gen(1)
    for fmt in FORMATS:
        W = rows_of(g, 320, 640, BF16, 0.05)
        perm = torch.randperm(640, generator=g, device=DEV).to(torch.int32)
        bias = torch.randn(320, generator=g, device=DEV).to(BF16)
        layer = mx.MXLinear.from_weight(W, fmt, perm, 64, bias)
        X, R = rows_of(g, 77, 640, BF16), rows_of(g, 77, 320, BF16)
        Y = layer(X, act="gelu", post="gelu", residual=R)
        q = mx.quantize(X, fmt, perm, 64, "gelu")
        assert torch.equal(Y, mx.linear(q, layer.w, bias, 64, post="gelu", residual=R))
        check(Y, q, layer.w, bias, 64, "gelu", R)
        assert torch.equal(layer(X), mx.linear(mx.quantize(X, fmt, perm, 64), layer.w, bias, 64))


@pytest.mark.parametrize("fmt", FORMATS)
def test_not_finite(fmt):
    """Rows and channels of infinities and NaN are NaN by themselves; a residual's own come through."""
    g = gen(2)
    X = rows_of(g, 200, 256, F16)
    X[7, 3], X[150, 200] = float("inf"), float("nan")
    w = mx.quantize(rows_of(g, 80, 256, BF16, 0.1), fmt)
    R = rows_of(g, 200, 80, F16)
    R[20, 5], R[21, 6], R[22, 7] = float("inf"), float("-inf"), float("nan")
    x = mx.quantize(X, fmt)
    for post in (None, "gelu"):
        Y = mx.linear(x, w, dtype=F16, post=post, residual=R)
        bad = Y.isnan()
        assert bad[7].all() and bad[150].all() and bad.sum() == 161 and bad[22, 7]
        assert Y[20, 5] == float("inf") and Y[21, 6] == float("-inf")
        assert torch.isfinite(Y).sum() == 200 * 80 - 163


def test_activation_of_large_accumulators():
    """GELU and SwiGLU where the product is far outside the output's range, and where fp32 has run out."""
    x = mx.quantize(torch.full((1, 32), 3e38, dtype=BF16, device=DEV), "block32_e4m3")
    W = torch.zeros((64, 32), dtype=BF16, device=DEV)
    W[0], W[1], W[2], W[3, 0], W[4, 0] = 1.0, -1e-3, 1e30, 1e-3, -1.0
    w = mx.quantize(W, "block32_e4m3")
    Y = mx.linear(x, w, post="gelu")
    assert Y[0, 2] == float("inf") and Y[0, 0] == float("inf") and Y[0, 1] == 0 and Y[0, 4] == 0 and (Y[0, 5:] == 0).all()
    assert abs(float(Y[0, 3]) / 3e35 - 1) < 0.1
    G = mx.linear(x, w, post="swiglu")
    assert (G[0, 8:] == 0).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_gelu_over_its_range(fmt):
    """Accumulators through GELU's whole range, one nonzero weight a channel so that they are exact."""
    K = 32
    X = torch.zeros((4097, K), dtype=F16, device=DEV)
    X[:, 0] = torch.linspace(-1.5, 1.5, 4097, device=DEV).to(F16)
    x = mx.quantize(X, fmt)
    W = torch.zeros((16, K), dtype=BF16, device=DEV)
    W[:, 0] = 2.0 ** torch.arange(-8, 8, device=DEV)
    w = mx.quantize(W, fmt)
    check(mx.linear(x, w, dtype=F16, post="gelu"), x, w, None, 1, "gelu", None)
    check(mx.linear(x, w, dtype=BF16, post="swiglu"), x, w, None, 1, "swiglu", None)


def test_streams_graphs_and_two_graphs():
    """On another stream; captured twice, replayed in turn on new contents."""
    g = gen(3)
    layer = mx.MXLinear.from_weight(rows_of(g, 1152, 640, BF16, 0.1), "block32_e4m3")
    sets = [(rows_of(g, 3000, 640, BF16), rows_of(g, 3000, 1152, BF16)) for _ in range(2)]
    want = [layer(X, post="gelu", residual=R) for X, R in sets]
    side = torch.cuda.Stream()
    got = layer(sets[0][0], post="gelu", residual=sets[0][1], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want[0])
    graphs = []
    for _ in range(2):
        x, r = torch.zeros_like(sets[0][0]), torch.zeros_like(sets[0][1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = layer(x, post="gelu", residual=r)
        graphs.append((graph, x, r, y))
    for turn in range(3):
        for i, (graph, x, r, y) in enumerate(graphs):
            x.copy_(sets[(i + turn) % 2][0]), r.copy_(sets[(i + turn) % 2][1])
            graph.replay()
        torch.cuda.synchronize()
        for i, (graph, x, r, y) in enumerate(graphs):
            assert torch.equal(y, want[(i + turn) % 2])


def test_same_bits_every_time():
    g = gen(4)
    x, w, bias = operands(g, 4000, 2304, 1152, "block32_e4m3", BF16, True)
    R = rows_of(g, 4000, 1152, BF16)
    first = mx.linear(x, w, bias, post="gelu", residual=R)
    for _ in range(20):
        assert torch.equal(mx.linear(x, w, bias, post="gelu", residual=R), first)


@pytest.mark.parametrize("M,K,N,tile", SHARED8)
def test_shared_tiles_again_and_in_place(M, K, N, tile):
    """The same bits every time, beside other products, and in the residual's place, with rows around it that stay."""
    g = gen(M + K)
    x, w, bias = operands(g, M, K, N, "block32_e4m3", BF16, True)
    space = torch.randn((M + 64, N), generator=g, device=DEV).to(BF16)
    before = space.clone()
    R = before[8:8 + M]
    first, plain = mx.linear(x, w, bias, post="gelu", residual=R), mx.linear(x, w, bias)
    sides = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [(mx.linear(x, w, bias, post="gelu", residual=R, stream=s), mx.linear(x, w, bias, stream=s)) for _ in range(20) for s in sides]
    torch.cuda.synchronize()
    assert all(torch.equal(a, first) and torch.equal(b, plain) for a, b in got)
    Y = space[8:8 + M]
    assert mx.linear(x, w, bias, Y=Y, post="gelu", residual=Y) is Y
    assert torch.equal(Y, first) and torch.equal(space[:8], before[:8]) and torch.equal(space[8 + M:], before[8 + M:])


@pytest.mark.parametrize("at", [0, 1023, 2048, 4607])
def test_shared_tiles_not_finite(at):
    """A value that is not finite reaches its row and no other, whichever CTA meets it."""
    g = gen(at)
    X = rows_of(g, 9, 4608, BF16)
    X[5, at] = float("inf")
    x, w = mx.quantize(X, "block32_e4m3"), mx.quantize(rows_of(g, 300, 4608, BF16, 0.1), "block32_e4m3")
    Y = mx.linear(x, w, post="gelu")
    assert Y[5].isnan().all() and Y.isnan().sum() == 300


SHARED = [("block32_e4m3",) + s for s in SHARED8] + [(f,) + s for f in ("block32", "block16") for s in SHARED4]


@pytest.mark.parametrize("fmt,M,K,N,tile", SHARED)
def test_shared_tiles_of_every_format(fmt, M, K, N, tile):
    """The same bits every time, beside other products, alone in a graph, and in the residual's place."""
    g = gen(M + K)
    x, w, bias = operands(g, M, K, N, fmt, F16, True)
    R = rows_of(g, M, N, F16)
    call = lambda **to: mx.linear(x, w, bias, dtype=F16, post="gelu", residual=R, **to)
    first = call()
    check(first, x, w, bias, 1, "gelu", R)
    sides = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [call(stream=s) for _ in range(20) for s in sides]
    torch.cuda.synchronize()
    assert all(torch.equal(y, first) for y in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ys = [call() for _ in range(8)]  # each begins while the one before it ends
    for _ in range(5):
        for y in ys:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, first) for y in ys)
    Y = R.clone()
    assert mx.linear(x, w, bias, dtype=F16, Y=Y, post="gelu", residual=Y) is Y
    assert torch.equal(Y, first)


@pytest.mark.parametrize("fmt,M,K,N,tile", SHARED)
def test_shared_tiles_not_finite_in_every_format(fmt, M, K, N, tile):
    """A value that is not finite, met by the first CTA, one in between or the last, is its row's alone."""
    g = gen(N)
    w = mx.quantize(rows_of(g, N, K, BF16, 0.1), fmt)
    for at in (0, K // 2, K - 1):
        X = rows_of(g, M, K, BF16)
        X[M // 2, at] = float("inf")
        Y = mx.linear(mx.quantize(X, fmt), w, post="gelu")
        assert Y[M // 2].isnan().all() and Y.isnan().sum() == N



def test_residuals_over_other_rows_are_refused():
    g = gen(22)
    x, w, bias = operands(g, 100, 160, 144, "block32_e4m3", BF16, True)
    space = torch.randn((109, 144), generator=g, device=DEV).to(BF16)
    before = space.clone()
    Y = space[:100]
    for R in (space[1:101], space[8:108], space.view(-1)[1:1 + 100 * 144].view(100, 144), space.view(-1)[8:8 + 100 * 152].view(100, 152)[:, :144]):
        with pytest.raises(clq.ClqError):
            mx.linear(x, w, bias, Y=Y, residual=R)
    torch.cuda.synchronize()
    assert torch.equal(space, before)
    wide = torch.cat((space, space), 1)[:100]
    assert torch.equal(mx.linear(x, w, bias, Y=Y, residual=wide[:, 144:]), mx.linear(x, w, bias, residual=before[:100]))


@pytest.mark.parametrize("M", [1, 40])
@pytest.mark.parametrize("post", [None, "gelu", "swiglu"])
def test_many_channels(M, post):
    """More than 2^27 channels: the columns of parts of them."""
    N, K = 2 ** 27 + 160, 32
    g = gen(31)
    codes = torch.randint(0, 0x70, (N, K), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.randint(118, 122, mx.scale_shape(N, K, "block32_e4m3"), generator=g, device=DEV, dtype=torch.uint8)
    w = mx.MXTensor(codes, scales, None, "block32_e4m3")
    x = mx.quantize(rows_of(g, M, K, BF16), "block32_e4m3")
    columns = N // 2 if post == "swiglu" else N
    R = torch.empty((M, columns), dtype=BF16, device=DEV).random_(-100, 100, generator=g)
    Y = mx.linear(x, w, post=post, residual=R)
    for n0 in (0, 2 ** 26 - 1024, 2 ** 26, 2 ** 27 - 1024, 2 ** 27):
        n1 = min(n0 + 2048, N)
        part = mx.MXTensor(codes[n0:n1], scales[n0 // 128:-(-n1 // 128)], None, "block32_e4m3")
        c0, c1 = (n0 // 2, n1 // 2) if post == "swiglu" else (n0, n1)
        want = mx.linear(x, part, post=post, residual=R[:, c0:c1])
        assert torch.equal(Y[:, c0:c1], want)
        check(want, x, part, None, 1, post, R[:, c0:c1])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("fmt", FORMATS)
def test_gelu_of_every_value(fmt, dtype):
    """Every finite value of the type as a channel's bias beside a product of 0: relative to itself wherever the type
    holds it, on the far negative side too."""
    v = torch.arange(-32768, 32768, device=DEV, dtype=torch.int16).view(dtype)
    v = v[torch.isfinite(v)]
    v = torch.cat((v, v[:-v.numel() % 16]))
    x = mx.quantize(torch.zeros((3, 32), dtype=dtype, device=DEV), fmt)
    w = mx.quantize(torch.zeros((v.numel(), 32), dtype=dtype, device=DEV), fmt)
    Y = mx.linear(x, w, v, dtype=dtype, post="gelu")
    d = v.double()
    want = d * 0.5 * torch.special.erfc(-d / 2 ** 0.5)
    # of GELU 2^-13 of itself to -6, 2^-10 behind it, nothing below 2^-122; then half a step
    own = torch.where(d >= -6, 2.0 ** -13, 2.0 ** -10)
    room = (ref.HALF_STEP[dtype] * (1 + 2.0 ** -8) + own) * want.abs() + ref.TINY[dtype] + 2.0 ** -122
    assert ((Y.double() - want).abs() <= room).all()
    near = (d >= -3) & (d <= 3)
    room = (ref.HALF_STEP[dtype] * (1 + 2.0 ** -10) + 2.0 ** -18) * want.abs() + ref.TINY[dtype] + 2.0 ** -22 * d.abs()
    assert ((Y.double() - want).abs() <= room)[:, near].all()


def test_gelu_in_front_and_behind():
    """The same activation behind a product and in front of the next one's quantization."""
    v = torch.linspace(-14, 6, 4096, device=DEV).to(BF16)
    x = mx.quantize(torch.zeros((32, 32), dtype=BF16, device=DEV), "block32_e4m3")
    w = mx.quantize(torch.zeros((4096, 32), dtype=BF16, device=DEV), "block32_e4m3")
    Y = mx.linear(x, w, v, post="gelu")
    behind = mx.quantize(Y, "block32_e4m3")
    ahead = mx.quantize(v[None].expand(32, 4096).contiguous(), "block32_e4m3", act="gelu")
    a, b = ref.values(behind), ref.values(ahead)
    # each half a step of E4M3 (2^-4) from the same value, one of them behind bf16's rounding (2^-8) and within 2^-10
    # of itself and 2^-122; steps of a block's smallest numbers are 2^-9 of its scale
    scale = torch.maximum(ref.scales(behind), ref.scales(ahead)).repeat_interleave(32, 1)
    assert ((a - b).abs() <= (2 * 2.0 ** -4 + 2.0 ** -7) * torch.maximum(a.abs(), b.abs()) + 2.0 ** -9 * scale + 2.0 ** -122).all()


def test_gelu_of_infinities():
    """Biases of infinities and NaN: the first its own value, minus infinity 0, NaN NaN; with a residual its own."""
    v = torch.tensor([float("inf"), float("-inf"), float("nan"), 1.0] * 4, device=DEV)
    for fmt in FORMATS:
        for dtype in (F16, BF16):
            x = mx.quantize(torch.zeros((5, 64), dtype=dtype, device=DEV), fmt)
            w = mx.quantize(torch.zeros((16, 64), dtype=dtype, device=DEV), fmt)
            Y = mx.linear(x, w, v.to(dtype), dtype=dtype, post="gelu").float()
            assert (Y[:, 0] == float("inf")).all() and (Y[:, 1] == 0).all() and Y[:, 2].isnan().all() and (Y[:, 3] > 0.8).all()
            R = torch.full((5, 16), 2.0, dtype=dtype, device=DEV)
            Y = mx.linear(x, w, v.to(dtype), dtype=dtype, post="gelu", residual=R).float()
            assert (Y[:, 0] == float("inf")).all() and (Y[:, 1] == 2).all() and Y[:, 2].isnan().all()


def test_on_another_stream():
    """A layer on another stream, which has waited for the inputs."""
    g = gen(26)
    layer = mx.MXLinear.from_weight(rows_of(g, 1152, 640, BF16, 0.1), "block32_e4m3")
    X, R = rows_of(g, 3000, 640, BF16), rows_of(g, 3000, 1152, BF16)
    want = layer(X, post="gelu", residual=R)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [layer(X, post="gelu", residual=R, stream=side) for _ in range(8)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(y, want) for y in got)


# ------------------------------------------------------------- the three in a row --
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,residual", [(1, True), (70, False), (1500, True)])
def test_norm_linear(fmt, dtype, M, residual):
    """h, the norm's codes, the product of them, q and k turned and v as it was, each from the step before."""
    g = gen(M)
    K, D, heads = 576, 72, 8
    W = rows_of(g, 3 * K, K, BF16, 0.05)
    perm = torch.randperm(K, generator=g, device=DEV).to(torch.int32)
    bias = torch.randn(3 * K, generator=g, device=DEV).to(dtype)
    weight = (1 + 0.3 * torch.randn(K, generator=g, device=DEV)).to(dtype)
    turn = rope.Rope(D, (36, 36), pairs="halves")
    layer = mx.MXNormLinear(mx.MXLinear.from_weight(W, fmt, perm, 64, bias), weight, 1e-5, rope=turn, heads=2 * heads)
    X, R = rows_of(g, M, K, dtype), rows_of(g, M, K, dtype) if residual else None
    positions = torch.randint(0, 1 << 20, (M, 2), generator=g, device=DEV).to(torch.int32)
    Y, h = layer(X, R, positions)
    q = mx.rms_norm(X, weight, R, 1e-5, fmt, perm, 64)
    if residual:
        q, s = q
        assert torch.equal(h, s)
    else:
        assert h is X
    y = mx.linear(q, layer.linear.w, bias, 64, dtype)
    check(y, q, layer.linear.w, bias, 64, None, None)
    n = 2 * heads * D
    assert torch.equal(Y[:, n:], y[:, n:])
    x = y[:, :n].reshape(M, 2 * heads, D)
    want = ref.turned(x, positions, turn.freqs, turn.sections, "halves")
    off = (Y[:, :n].reshape(M, 2 * heads, D).double() - want).abs()
    assert (off <= ref.turned_bound(x, want, turn.freqs, "halves", positions, dtype)).all()


def test_feed_forward_of_a_block():
    """norm -> up product with its activation -> down product onto the residual stream, against full precision."""
    g = gen(8)
    M, K, F = 300, 512, 1536
    X, R = rows_of(g, M, K, BF16), rows_of(g, M, K, BF16)
    W1, W2 = rows_of(g, F, K, BF16, 0.02), rows_of(g, K, F, BF16, 0.02)
    up = mx.MXNormLinear(mx.MXLinear.from_weight(W1, "block32_e4m3"), post="gelu")
    down = mx.MXLinear.from_weight(W2, "block32_e4m3")
    Y, h = up(X, R)
    out = down(Y, residual=h)
    hd = h.double()
    a = hd / torch.sqrt(hd.square().mean(1, keepdim=True) + 1e-6) @ W1.double().t()
    want = a * 0.5 * torch.special.erfc(-a / 2 ** 0.5) @ W2.double().t()
    got = out.double() - hd
    # 8 bits: each operand of each product within 2^-4 of itself at most, 2^-5 / sqrt 3 of it rms; four operands
    assert (got - want).norm() <= 2 * 2.0 ** -4 * want.norm()


def test_layer_on_another_stream():
    g = gen(9)
    turn = rope.Rope(64, (32, 32))
    layer = mx.MXNormLinear(mx.MXLinear.from_weight(rows_of(g, 384, 128, BF16, 0.1), "block32_e4m3"), rope=turn, heads=4)
    X, R = rows_of(g, 40, 128, BF16), rows_of(g, 40, 128, BF16)
    positions = torch.randint(0, 99, (40, 2), generator=g, device=DEV).to(torch.int32)
    want = layer(X, R, positions)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = layer(X, R, positions, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    x, r, p = torch.zeros_like(X), torch.zeros_like(R), torch.zeros_like(positions)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, h = layer(x, r, p)
    x.copy_(X), r.copy_(R), p.copy_(positions)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(h, want[1])
