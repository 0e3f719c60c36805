"""Microscaled operators on the GPU: paths, tiles and orders of calls that the shapes of
test_gpu_mx.py do not reach, against their definitions in 64 bits (mx_utils)."""
import pytest
import torch

import mx_tiles as tiles
import mx_utils as ref
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


# ------------------------------------------------------- every tile of the product --
@pytest.fixture(scope="module")
def picks(tmp_path_factory):
    return tiles.library(tmp_path_factory.mktemp("tiles"))


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def exact_tensor(g, rows, K, fmt, stack=(), low=0):
    """Random codes; block scales of 2^low and twice that, row scales of 0.5, 1 and 2, so that sums
    of products are exact in fp32.  The scales of rows past the last one, which nothing may use,
    are NaN; those of blocks past the last one 0."""
    lead = tuple(stack)
    codes = torch.randint(0, 256, lead + (rows, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    one, step, nan = (127 + low, 1, 255) if fmt == "block32" else (56 + 8 * low, 8, 127)
    shape = mx.scale_shape(rows, K, fmt)
    scales = (one + step * torch.randint(0, 2, lead + shape, generator=g, device=DEV)).to(torch.uint8)
    i, c, r, j, q = (torch.arange(n, device=DEV) for n in shape)
    row = 128 * i[:, None, None, None, None] + 32 * j[None, None, None, :, None] + r[None, None, :, None, None]
    scales = torch.where(row < rows, scales, nan)
    block = 4 * c[None, :, None, None, None] + q
    scales = torch.where(block < K // ref.BLOCK[fmt], scales, 0).to(torch.uint8).contiguous()
    rs = 2.0 ** torch.randint(-1, 2, lead + (rows,), generator=g, device=DEV) if fmt == "block16" else None
    return mx.MXTensor(codes, scales, rs, fmt)


def part(q, i):
    """Matrix i of a stack."""
    return mx.MXTensor(q.codes[i], q.scales[i], None if q.row_scale is None else q.row_scale[i], q.fmt)


def values64(q):
    grid = torch.tensor(list(ref.GRID) + list(-ref.GRID), dtype=torch.float64, device=DEV)
    v = grid[torch.stack((q.codes & 15, q.codes >> 4), 2).view(q.rows, q.K).long()]
    r, blk = torch.arange(q.rows, device=DEV)[:, None], torch.arange(q.K // ref.BLOCK[q.fmt], device=DEV)[None, :]
    byte = q.scales[r // 128, blk // 4, r % 32, r % 128 // 32, blk % 4]
    s = torch.exp2(byte.double() - 127) if q.fmt == "block32" else byte.view(torch.float8_e4m3fn).double()
    if q.row_scale is not None:
        s = s * q.row_scale.double()[:, None]
    return v * s.repeat_interleave(ref.BLOCK[q.fmt], 1)


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("M,K,N,tile", tiles.DENSE)
def test_linear_exact_in_every_tile(picks, fmt, M, K, N, tile):
    """Sums that fp32 holds: at most 36 * 4 * 8192 of multiples of 1 / 4, and powers of two and a bias of
    quarters on top."""
    if sms() == 152:
        assert tiles.dense(picks, M, N, K) == tile
    g = gen(M + N)
    dtype = F16 if (M + K) % 3 else BF16
    x, w = exact_tensor(g, M, K, fmt), exact_tensor(g, N, K, fmt)
    bias = (torch.randint(-64, 65, (N,), generator=g, device=DEV) / 4).to(dtype)
    want = values64(x) @ values64(w).t() / 4 + bias.double()
    assert torch.equal(want.float().double(), want)
    want = want.float().to(dtype)
    for _ in range(3):
        assert torch.equal(mx.linear(x, w, bias, 4, dtype), want)


def uneven_routing(g, T, k, E):
    """Experts that get from few tokens to nearly all of them; some places without an expert."""
    keys = torch.rand((T, E), generator=g, device=DEV) * torch.linspace(0.4, 1, E, device=DEV)
    experts = keys.argsort(1, descending=True)[:, :k].to(torch.int32)
    experts[torch.rand((T, k), generator=g, device=DEV) < 0.02] = -1
    return mx.Routing(experts.contiguous(), torch.ones((T, k), device=DEV), E)


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("T,k,E,N,K,tile", tiles.GROUPED)
def test_grouped_product_exact_in_every_tile(picks, fmt, T, k, E, N, K, tile):
    if sms() == 152:
        assert tiles.grouped(picks, T, k, E, N, K) == tile
    g = gen(T + N)
    dtype = F16 if T % 3 else BF16
    r = uneven_routing(g, T, k, E)
    rows, space, R = mx.plan(r)
    x, w = exact_tensor(g, R, K, fmt), exact_tensor(g, N, K, fmt, (E,))
    bias = (torch.randint(-64, 65, (E, N), generator=g, device=DEV) / 4).to(dtype)
    for turn in range(3):
        Y = torch.full((R, N), 7.0, dtype=dtype, device=DEV)
        assert mx.clq_mx_grouped_linear(P(x.codes), P(x.scales), P(x.row_scale), P(space), P(w.codes), P(w.scales),
                                        P(w.row_scale), P(bias), T, k, E, N, K, 4, mx.FORMATS[fmt], mx.DTYPES[dtype], P(Y),
                                        stream()) == 0
        xv = values64(x) if turn == 0 else xv
        for e in range(E):
            mine = rows[r.experts == e].long()  # none, for some of 20 tokens' experts
            want = xv[mine] @ values64(part(w, e)).t() / 4 + bias[e].double()
            assert torch.equal(Y[mine], want.float().to(dtype)), (turn, e)


@pytest.mark.parametrize("act", ["swiglu", "gelu", None])
@pytest.mark.parametrize("T,k,E,N,K,tile", tiles.GROUPED)
def test_fused_activation_in_every_tile(picks, act, T, k, E, N, K, tile):
    """The product that quantizes its output against the product (exact, above), then the
    quantization: one activation function serves both, so the bytes are the same."""
    N = N // 64 * 64 if act == "swiglu" else N
    if sms() == 152:
        assert tiles.grouped(picks, T, k, E, N, K) == tile
    F = N // 2 if act == "swiglu" else N
    g = gen(T + N)
    dtype = F16 if T % 3 else BF16
    r = uneven_routing(g, T, k, E)
    rows, space, R = mx.plan(r)
    # sums of the order of 1
    x, w = exact_tensor(g, R, K, "block32", low=-4), exact_tensor(g, N, K, "block32", (E,), low=-5)
    bias = (torch.randint(-8, 9, (E, N), generator=g, device=DEV) / 4).to(dtype)
    dt = mx.DTYPES[dtype]
    Y = torch.zeros((R, N), dtype=dtype, device=DEV)
    assert mx.clq_mx_grouped_linear(P(x.codes), P(x.scales), None, P(space), P(w.codes), P(w.scales), None, P(bias), T, k, E, N,
                                    K, 1, 0, dt, P(Y), stream()) == 0
    a = [torch.zeros_like(t) for t in mx._empty(R, F, "block32", DEV)[:2]]
    assert mx.clq_mx_quantize_rows(P(Y), dt, P(space), T, k, E, F, N, mx.ACTS[act], 0, P(a[0]), P(a[1]), None, stream()) == 0
    used = rows[rows >= 0].long()
    want = values64(mx.MXTensor(*a))[used]
    assert 0.01 < want.abs().mean() < 100
    for _ in range(3):
        f = [torch.full_like(t, 99) for t in a]
        assert mx.clq_mx_grouped_linear_act(P(x.codes), P(x.scales), P(space), P(w.codes), P(w.scales), P(bias), T, k, E, N, K,
                                            1, dt, mx.ACTS[act], P(f[0]), P(f[1]), stream()) == 0
        assert torch.equal(f[0][used], a[0][used])
        blocks = 4 * -(-F // 128)
        at = used.cpu().numpy()
        assert (ref.scale_bytes(f[1], R, blocks)[at] == ref.scale_bytes(a[1], R, blocks)[at]).all()


# ------------------------------------------------------------------------ routing --
# E, groups: groups of a power of two from 32 on, of another multiple of 32, of a power of two
# below 32, of any other size
GROUPS = [(64, 2), (128, 2), (256, 4), (256, 2), (512, 2), (512, 4), (512, 16), (320, 5), (256, 8),
          (192, 2), (384, 4), (320, 2), (448, 2), (288, 3),
          (32, 32), (64, 32), (64, 16), (256, 32), (256, 16), (60, 15), (24, 3),
          (300, 3), (96, 2), (144, 3), (45, 15), (288, 32), (33, 3), (500, 20)]


@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("E,groups", GROUPS)
def test_route_groups_of_every_size(E, groups, group_top):
    g = gen(E + groups)
    T, size = 96, E // groups
    for turn, (scoring, k) in enumerate((("softmax", 1), ("sigmoid", 4), ("softmax", 6), ("sigmoid", 8), ("softmax", 9), ("sigmoid", 32))):
        k = min(k, E)
        top_groups = max(1, groups // 2) if turn % 2 else max(1, groups - 1)
        L = torch.randn((T, E), generator=g, device=DEV)
        if turn >= 4:  # many equal scores
            L = L.round()
        L[:16] = torch.where(torch.rand((16, E), generator=g, device=DEV) < 0.5, L[:16], -float("inf"))
        by = L.view(T, groups, size)
        by[16:24, 0] = -float("inf")  # no expert of a group
        by[24:32, -1, 1:] = -float("inf")  # one
        L[32:36] = -float("inf")
        bal = 0.1 * torch.randn(E, generator=g, device=DEV) if turn in (1, 2) else None
        r = mx.route(L, k, scoring, bal, groups, top_groups, group_top)
        experts, weights, margin = ref.routing(L.cpu().double().numpy(), None if bal is None else bal.cpu().double().numpy(), k, scoring,
                                               groups, top_groups, group_top)
        # as in test_gpu_mx.py: fp32 scores are within 2^-20 of the exact ones, equal ones tie
        clear = (margin > 2.0 ** -20) | (margin == 0)
        assert clear.mean() > 0.9
        assert (r.experts.cpu().numpy()[clear] == experts[clear]).all(), turn
        assert abs(r.weights.cpu().double().numpy()[clear] - weights[clear]).max() <= 1e-5


# -------------------------------------------------- quantization into chosen rows --
def offset(t, nbytes):
    """A copy of t that starts `nbytes` behind a 256-byte boundary."""
    raw = torch.empty(t.numel() * t.element_size() + 256, dtype=torch.uint8, device=DEV)
    at = -raw.data_ptr() % 256 + nbytes
    out = raw[at:at + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
    out.copy_(t)
    return out


def quantize_to(X, fmt, perm, b, rows, R, codes_at=0):
    """clq_mx_quantize into R rows, those of `rows` [M, k]; every byte elsewhere is 0xAB."""
    M, K = X.shape
    out = [None if t is None else t.view(torch.uint8).fill_(0xAB).view(t.dtype) for t in mx._empty(R, K, fmt, DEV)]
    if codes_at:
        out[0] = offset(out[0], codes_at)
    assert mx.clq_mx_quantize(P(X), mx.DTYPES[X.dtype], M, K, X.stride(0), P(perm), b, 0, mx.FORMATS[fmt], *map(P, out), P(rows),
                              rows.shape[1], R, stream()) == 0
    return out


def check_rows(out, want, to, R, fmt):
    """Row to[i] of `out` is row i of the MXTensor `want`, and no other row was written."""
    to = to.long()
    blocks = want.K // ref.BLOCK[fmt]
    padded = 4 * -(-blocks // 4)
    assert torch.equal(out[0][to], want.codes)
    got, expect = ref.scale_bytes(out[1], R, padded), ref.scale_bytes(want.scales, want.rows, padded)
    assert (got[to.cpu().numpy()] == expect).all()
    rest = torch.ones(R, dtype=torch.bool, device=DEV)
    rest[to] = False
    assert (out[0][rest] == 0xAB).all() and (got[rest.cpu().numpy()] == 0xAB).all()
    if fmt == "block16":
        bits = out[2].view(torch.int32)
        assert torch.equal(out[2][to].nan_to_num(-1), want.row_scale.nan_to_num(-1))
        assert (bits[rest] == bits.new_tensor([-0x54545455])).all()


# the last one of each group is far below the threshold of the kernel for many rows
INTO_ROWS = [(6601, 1152, 64), (6601, 1152, 128), (14007, 512, 64), (12001, 704, 64), (9001, 640, 128), (2500, 4608, 128), (120, 1152, 64)]


@pytest.mark.parametrize("fmt", ["block32", "block16"])
@pytest.mark.parametrize("M,K,b", INTO_ROWS)
def test_quantize_into_rows(fmt, M, K, b):
    """Codes, scales and row scales of rows that go to one, two or no other rows, in both kernels,
    with a swap vector off a 16-byte and codes off a 32-byte boundary."""
    g = gen(M + K)
    X = torch.randn((M, K), generator=g, device=DEV).to(BF16)
    X[M // 3, 5], X[M // 2, 3], X[M // 5] = float("inf"), float("nan"), 0
    perm = torch.randperm(K, generator=g, device=DEV).to(torch.int32)
    step = 128 * max(1, 60000 // K // 128)  # parts that take the kernel for few rows
    parts = [mx.quantize(X[i:i + step], fmt, perm, b) for i in range(0, M, step)]
    blocks = K // ref.BLOCK[fmt]
    # the parts are whole blocks of 128 rows, so their scale arrays go end to end
    want = mx.MXTensor(torch.cat([p.codes for p in parts]), torch.cat([p.scales for p in parts]),
                       torch.cat([p.row_scale for p in parts]) if fmt == "block16" else None, fmt)
    R = 2 * M + 5
    places = torch.randperm(R, generator=g, device=DEV)[:2 * M].to(torch.int32).view(M, 2).contiguous()
    places[1::3, 0] = -1
    places[2::5, 1] = -1
    at, which = places.flatten(), torch.arange(M, device=DEV).repeat_interleave(2)
    live = at >= 0
    picked = which[live]
    scales = torch.from_numpy(ref.scale_bytes(want.scales, M, 4 * -(-blocks // 4))).to(DEV)[picked]
    tiled = torch.zeros((-(-len(picked) // 128) * 128, scales.shape[1]), dtype=torch.uint8, device=DEV)
    tiled[:len(picked)] = scales
    tiled = tiled.view(-1, 4, 32, scales.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()
    rows = mx.MXTensor(want.codes[picked].contiguous(), tiled, want.row_scale[picked] if fmt == "block16" else None, fmt)
    for codes_at, perm_at in ((0, 0), (16, 4)):
        out = quantize_to(X, fmt, offset(perm, perm_at), b, places, R, codes_at)
        check_rows(out, rows, at[live], R, fmt)


@pytest.mark.parametrize("M,K,b", [(6601, 1152, 64), (6601, 1152, 128), (40, 1152, 64)])
def test_quantize_reports_indices_out_of_range(M, K, b):
    """A row index past the last one is not written, an element of the swap vector that is none reads
    element 0; both are reported."""
    g = gen(M)
    X = torch.randn((M, K), generator=g, device=DEV).to(F16)
    perm = torch.randperm(K, generator=g, device=DEV).to(torch.int32)
    rows = torch.arange(M, device=DEV).to(torch.int32)[:, None].contiguous()
    want = quantize_to(X, "block16", perm, b, rows, M)
    torch.cuda.synchronize()
    assert clq.device_status() == 0
    bad = rows.clone()
    bad[M // 2], bad[M - 1] = M, 2 ** 31 - 1
    out = quantize_to(X, "block16", perm, b, bad, M)
    torch.cuda.synchronize()
    assert clq.device_status() == 7
    keep = torch.ones(M, dtype=torch.bool, device=DEV)
    keep[M // 2] = keep[M - 1] = False
    for o, w in zip((out[0], out[2]), (want[0], want[2])):
        assert torch.equal(o[keep], w[keep])
    assert (out[0][~keep] == 0xAB).all()
    for value in (K, -1, 2 ** 31 - 1, -2 ** 31):
        broken, zero = perm.clone(), perm.clone()
        broken[K // 2 + 1], zero[K // 2 + 1] = value, 0
        got = quantize_to(X, "block16", broken, b, rows, M)
        torch.cuda.synchronize()
        assert clq.device_status() == 7
        expect = quantize_to(X, "block16", zero, b, rows, M)
        assert torch.equal(got[0], expect[0]) and torch.equal(got[2], expect[2])


def test_combine_reports_rows_out_of_range():
    """A row past the last one adds nothing and is reported; one below 0 is a place without a row."""
    g = gen(7)
    Y = torch.randn((64, 48), generator=g, device=DEV).to(BF16)
    rows = torch.randint(0, 64, (33, 3), generator=g, device=DEV).to(torch.int32)
    w = torch.rand((33, 3), generator=g, device=DEV)
    out = torch.empty((33, 48), dtype=BF16, device=DEV)
    call = lambda r: mx.clq_mx_combine(P(Y), 1, P(r), P(w), 33, 3, 48, 64, P(out), stream())
    none = rows.clone()
    none[4, 1], none[20, 0], none[32, 2] = -1, -5, -1
    assert call(none) == 0
    want = out.clone()
    assert clq.device_status() == 0
    bad = none.clone()
    bad[4, 1], bad[20, 0], bad[32, 2] = 64, 2 ** 31 - 1, 65
    assert call(bad) == 0
    torch.cuda.synchronize()
    assert clq.device_status() == 7
    assert torch.equal(out, want)


@pytest.mark.parametrize("T,k,E", [(16385, 2, 8), (16897, 3, 40), (40000, 8, 256), (70001, 2, 512)])
def test_plan_of_many_tokens(T, k, E):
    """More blocks of tokens than one turn of the prefix takes (128 of 128 tokens)."""
    g = gen(T)
    r = uneven_routing(g, T, k, E)
    rows, space, R = mx.plan(r)
    at = r.experts.long()
    flat = at.flatten()
    order = torch.sort(torch.where(flat < 0, E, flat), stable=True)
    count = torch.bincount(flat[flat >= 0], minlength=E)
    blocks = (count + 127) // 128 * 128
    start = torch.cumsum(blocks, 0) - blocks
    before = torch.cumsum(count, 0) - count
    n = int(count.sum())
    want = torch.full_like(flat, -1)
    e = order.values[:n]
    want[order.indices[:n]] = start[e] + torch.arange(n, device=DEV) - before[e]
    assert torch.equal(rows.flatten().long(), want)
    assert int(start[-1] + blocks[-1]) <= R


def test_wider_codes_under_capture():
    """Codes in a wider type are narrowed under stream capture too, where nothing can be read back."""
    g = gen(11)
    w = exact_tensor(g, 64, 128, "block32")
    x = exact_tensor(g, 3, 128, "block32")
    wide = w.codes.long()
    want = mx.linear(x, w, dtype=F16)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = mx.linear(x, mx.MXTensor(wide, w.scales), dtype=F16)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    wide[5, 7] = -3
    with pytest.raises(ValueError, match="0 to 255"):
        mx.MXTensor(wide, w.scales)
