"""CPU-only checks of norm, product with what is behind it and rotary positions: declarations, refusals before any
launch, the argument checks of the tensor helpers, streams, and the 64-bit fractions of a turn."""
import copy
import ctypes
import gc
import os
import pickle
import random
import re
import struct
import subprocess
from fractions import Fraction

import pytest
import torch

import block_tiles as tiles
import test_gpu_post as shapes_of
from paper_2509_24416_gb300 import build, clq, mx, rope
from test_streams_cpu import FakeStream, HERE, SIDE, fake  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # a 16-byte aligned "device" address that nothing reads
E4M3 = mx.FORMATS["block32_e4m3"]


@pytest.fixture(scope="module")
def lib():
    build.build()
    mx.load()
    return rope.load()


def test_header_matches_binding(lib):
    text = open(os.path.join(ROOT, "include", "clq_rope.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(clq_rope[a-z0-9_]*)\s*\(", text))) == sorted(rope.EXPORTS)
    header = open(os.path.join(ROOT, "include", "clq_mx.h")).read()
    assert int(re.search(r"#define CLQ_MX_BLOCK32_E4M3 (\d+)", header).group(1)) == E4M3


def norm(X=P, dtype=0, M=4, K=64, ldx=64, residual=None, ldr=0, weight=None, eps=1e-6, perm=None, b=1, fmt=E4M3, codes=P,
         scales=P, row_scale=None, sum=None, lds=0):
    return mx.clq_mx_rms_norm(X, dtype, M, K, ldx, residual, ldr, weight, eps, perm, b, fmt, codes, scales, row_scale, sum, lds,
                              None)


BOTH = dict(residual=P, ldr=64, sum=P, lds=64)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), 1), (dict(fmt=2), 1), (dict(fmt=-1), 1), (dict(M=-1), 1), (dict(eps=0.0), 1), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(eps=1e-60), 1), (dict(residual=P, ldr=64), 1),
    (dict(sum=P, lds=64), 1), (dict(X=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(fmt=1), 1),
    (dict(residual=2 * P, ldr=64, sum=P, lds=72), 1), (dict(residual=2 * P, ldr=64, sum=2 * P, lds=72), 1),
    (dict(M=1 << 30), 2), (dict(K=48), 2), (dict(K=0), 2), (dict(K=16416, ldx=16416), 2), (dict(b=3), 2), (dict(b=128), 2),
    (dict(b=512), 2), (dict(ldx=56), 2), (dict(BOTH, ldr=56), 2), (dict(BOTH, lds=56), 2),
    (dict(ldx=68), 3), (dict(BOTH, ldr=68), 3), (dict(BOTH, lds=68), 3), (dict(X=P + 8), 3), (dict(BOTH, residual=P + 8), 3),
    (dict(BOTH, sum=P + 8), 3), (dict(weight=P + 8), 3), (dict(codes=P + 8), 3), (dict(scales=P + 4), 3), (dict(perm=P + 2), 3),
    (dict(fmt=1, row_scale=P + 2), 3), (dict(M=0, X=None, codes=None, scales=None), 0)])
def test_norm_refuses(lib, change, code):
    assert norm(**change) == code


def post(Xq=P, Xs=P, s_x=None, Wq=P, Ws=P, s_w=None, bias=None, M=4, N=32, K=64, b=1, fmt=E4M3, dtype=0, act=1, residual=None,
         ldr=0, Y=P):
    return mx.clq_mx_linear_post(Xq, Xs, s_x, Wq, Ws, s_w, bias, M, N, K, b, fmt, dtype, act, residual, ldr, Y, None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), 1), (dict(fmt=3), 1), (dict(act=-1), 1), (dict(act=3), 1), (dict(M=-1), 1), (dict(N=-1), 1),
    (dict(Xq=None), 1), (dict(Ws=None), 1), (dict(Y=None), 1), (dict(fmt=1), 1), (dict(residual=P, ldr=40), 1),
    (dict(act=2, residual=P, ldr=24), 1),
    (dict(M=1 << 30), 2), (dict(N=1 << 30), 2), (dict(K=80), 2), (dict(b=128), 2), (dict(act=2, N=24), 2),
    (dict(residual=P, ldr=31), 2), (dict(act=2, residual=P, ldr=15), 2),
    (dict(residual=P + 1, ldr=32), 3), (dict(Y=P + 8), 3), (dict(bias=P + 1), 3), (dict(Xs=P + 8), 3), (dict(Wq=P + 4), 3),
    (dict(M=0, Y=None), 0), (dict(N=0, Wq=None), 0)])
def test_product_refuses(lib, change, code):
    assert post(**change) == code


def test_experts_take_four_bits(lib):
    assert mx.clq_mx_grouped_linear(P, P, None, P, P, P, None, None, 4, 2, 8, 64, 64, 1, E4M3, 0, P, None) == 1
    assert mx.clq_mx_quantize_rows(P, 0, P, 4, 2, 8, 64, 64, 0, E4M3, P, P, None, None) == 1
    w1, w2 = tensor(128, 64, lead=(3,)), tensor(64, 64, lead=(3,))
    with pytest.raises(ValueError, match="4-bit"):
        mx.MXExperts(w1, w2)


def turn(x=P, dtype=0, T=4, H=2, D=64, ts=128, hs=64, positions=P, ld=3, axes=3, sections=(8, 12, 12), turns=P, pairs=0,
         inverse=0, out=P, ots=128, ohs=64):
    s = None if sections is None else (ctypes.c_int32 * len(sections))(*sections)
    return rope.clq_rope(x, dtype, T, H, D, ts, hs, positions, ld, axes, s, turns, pairs, inverse, out, ots, ohs, None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), 1), (dict(T=-1), 1), (dict(H=-1), 1), (dict(pairs=2), 1), (dict(pairs=-1), 1), (dict(axes=0), 1),
    (dict(axes=5, sections=(1,) * 5), 1), (dict(sections=None), 1), (dict(sections=(8, -1, 12)), 1), (dict(x=None), 1),
    (dict(out=None), 1), (dict(positions=None), 1), (dict(turns=None), 1), (dict(ots=192), 1), (dict(ohs=640, ots=72, T=2), 1),
    (dict(ohs=63), 2), (dict(ots=127), 2), (dict(ots=64, ohs=255), 2), (dict(ots=32, T=2, H=1), 2), (dict(ohs=32, T=1), 2),
    (dict(D=62), 2), (dict(T=1 << 30), 2), (dict(sections=(0, 0, 0)), 2), (dict(D=4098), 2), (dict(D=1), 2), (dict(H=65536), 2), (dict(ts=-1), 2),
    (dict(ohs=-8), 2), (dict(ots=0), 2), (dict(ohs=0), 2), (dict(ld=-1), 2), (dict(sections=(2 ** 31 - 1, 2 ** 31 - 1, 4)), 2),
    (dict(x=P + 1), 3), (dict(out=P + 1), 3), (dict(positions=P + 2), 3), (dict(turns=P + 4), 3),
    (dict(T=0, x=None), 0), (dict(H=0, x=None), 0)])
def test_rope_refuses(lib, change, code):
    assert turn(**change) == code


def tensor(rows, K, fmt="block32_e4m3", lead=()):
    return mx.MXTensor(torch.zeros(lead + (rows, K // (1 if fmt == "block32_e4m3" else 2)), dtype=torch.uint8),
                       torch.zeros(lead + mx.scale_shape(rows, K, fmt), dtype=torch.uint8),
                       torch.zeros(lead + (rows,)) if fmt == "block16" else None, fmt)


H = torch.float16


def test_helpers_refuse_host_tensors():
    X, q = torch.zeros((4, 64), dtype=H), tensor(4, 64)
    r = rope.Rope(64, (64,), device="cpu")
    for call in (lambda: mx.rms_norm(X), lambda: mx.rms_norm(X, None, X), lambda: mx.quantize(X, "block32_e4m3"),
                 lambda: mx.linear(q, tensor(8, 64), post="gelu"), lambda: mx.MXLinear(tensor(8, 64))(X, post="gelu"),
                 lambda: mx.MXNormLinear(mx.MXLinear(tensor(8, 64)))(X), lambda: mx.dequantize(q),
                 lambda: r(X.view(4, 1, 64), torch.zeros((4, 1), dtype=torch.int32))):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_other_devices_are_refused(monkeypatch):
    """Tensors of another device than the current one, on which the call would launch."""
    class There:
        is_cuda, device = True, torch.device("cuda:1")
        get_device = staticmethod(lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        mx._on_gpu(There(), None, There())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    mx._on_gpu(There(), There())


def test_helpers_refuse(monkeypatch):
    monkeypatch.setattr(mx, "_on_gpu", lambda *t: None)
    X, q, w = torch.zeros((4, 64), dtype=H), tensor(4, 64), tensor(32, 64)
    half = lambda *shape: torch.zeros(shape, dtype=H)
    layer = mx.MXLinear(w)
    r = rope.Rope(16, (16,), device="cpu")
    for bad in (
            lambda: mx.rms_norm(X, fmt="block8"), lambda: mx.rms_norm(X, half(32)), lambda: mx.rms_norm(X, half(64).float()),
            lambda: mx.rms_norm(X, None, half(4, 96)), lambda: mx.rms_norm(X, None, half(5, 64)),
            lambda: mx.rms_norm(X, None, X.float()), lambda: mx.rms_norm(X, None, half(64, 4).t()),
            lambda: mx.rms_norm(X, out=X), lambda: mx.rms_norm(X, None, X, out=half(4, 65)),
            lambda: mx.rms_norm(X, perm=torch.zeros(32, dtype=torch.int32)),
            lambda: mx.linear(q, w, dtype=H, post="relu"), lambda: mx.linear(q, tensor(24, 64), dtype=H, post="swiglu"),
            lambda: mx.linear(q, w, dtype=H, residual=half(4, 31)), lambda: mx.linear(q, w, dtype=H, residual=half(4, 32).float()),
            lambda: mx.linear(q, w, dtype=H, post="swiglu", residual=half(4, 32)),
            lambda: mx.linear(q, w, dtype=H, post="swiglu", Y=half(4, 32)), lambda: mx.linear(q, tensor(32, 64, "block32")),
            lambda: mx.MXNormLinear(layer, half(32)), lambda: mx.MXNormLinear(layer, post="relu"),
            lambda: mx.MXNormLinear(layer, rope=r), lambda: mx.MXNormLinear(layer, heads=1),
            lambda: mx.MXNormLinear(layer, rope=r, heads=3), lambda: mx.MXNormLinear(layer, rope=r, heads=-1),
            lambda: mx.MXNormLinear(layer, post="swiglu", rope=r, heads=2),
            lambda: mx.MXNormLinear(layer)(X, positions=torch.zeros((4, 1), dtype=torch.int32)),
            lambda: mx.MXNormLinear(layer, rope=r, heads=2)(X),
            lambda: rope.Rope(16, ()), lambda: rope.Rope(16, (2,) * 5), lambda: rope.Rope(16, (3,)), lambda: rope.Rope(16, (18,)),
            lambda: rope.Rope(16, (-2, 4)), lambda: rope.Rope(16, (0,)), lambda: rope.Rope(8192, (16,)),
            lambda: rope.Rope(16, (16,), theta=0), lambda: rope.Rope(16, (16,), pairs="thirds"),
            lambda: rope.Rope(16, (16,), freqs=[1.0]), lambda: rope.Rope(4, (4,), freqs=[1.0, float("inf")]),
            lambda: r(half(4, 2, 8), torch.zeros((4, 1), dtype=torch.int32)), lambda: r(half(4, 16), torch.zeros((4, 1), dtype=torch.int32)),
            lambda: r(half(4, 2, 16), torch.zeros((4, 1))), lambda: r(half(4, 2, 16), torch.zeros((3, 1), dtype=torch.int32)),
            lambda: r(half(4, 2, 16), torch.zeros((4, 2), dtype=torch.int32)),
            lambda: r(half(4, 2, 16), torch.zeros((4, 1), dtype=torch.int32), out=half(4, 2, 8)),
            lambda: r(half(4, 2, 16), torch.zeros((4, 1), dtype=torch.int32), out=half(1, 2, 16).expand(4, 2, 16)),
            lambda: r(half(4, 2, 16), torch.zeros((4, 1), dtype=torch.int32), out=half(4, 1, 16).expand(4, 2, 16))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        mx.rms_norm(X.float())


def test_fractions_of_a_turn():
    """Each within half of 2^-64 of f / 2 pi, by a series for pi of its own (Machin's)."""
    def arctan_inverse(n, terms=60):
        return sum(Fraction((-1) ** i, (2 * i + 1) * n ** (2 * i + 1)) for i in range(terms))
    pi = 16 * arctan_inverse(5) - 4 * arctan_inverse(239)
    r = rope.Rope(64, (16, 24, 24), device="cpu")
    for f, t in zip(r.freqs, r.turns.tolist()):
        want = Fraction(f) / (2 * pi) * 2 ** 64
        assert abs((t % 2 ** 64) - want) <= Fraction(1, 2) + Fraction(1, 2 ** 20)
    # more than a turn a position, and backwards
    r = rope.Rope(4, (4,), freqs=[100.0, -0.25], device="cpu")
    for f, t in zip(r.freqs, r.turns.tolist()):
        want = Fraction(f) / (2 * pi)
        off = Fraction(t, 2 ** 64) - want
        assert abs(off - round(off)) <= Fraction(1, 2 ** 64)


def test_shapes_of_the_tests_take_every_tile(tmp_path):
    lib = tiles.library(tmp_path)
    whole = {(32, 1, 1), (64, 1, 1), (128, 1, 1), (128, 2, 1), (192, 2, 1), (256, 1, 1), (256, 2, 1)}
    shared = {(32, 1, 2), (32, 1, 4), (64, 1, 2), (64, 1, 4)}
    shared8 = shared | {(32, 1, 8)}  # (4-bit rows have half the steps)
    for fmt, post, shapes, every in (("block32_e4m3", False, shapes_of.STORED + shapes_of.SHARED8, whole | shared8),
                                     ("block32_e4m3", True, shapes_of.POST8 + shapes_of.SHARED8, whole | shared8),
                                     ("block32", True, shapes_of.POST4 + shapes_of.SHARED4, whole | shared)):
        for M, K, N, tile in shapes:
            assert tiles.tile(lib, M, N, K, fmt, post) == tile, (M, K, N)
        assert {s[-1] for s in shapes} == every
        rng = random.Random(5)
        log = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
        seen = set()
        for _ in range(20000):
            M, N, K = log(1, 40000), log(1, 20000), 32 * log(1, 512)
            tile = tiles.tile(lib, M, N, K, fmt, post)
            seen.add(tile)
            if tile[2] > 1:  # at one CTA a SM, each with steps of its own
                bytes_ = K if fmt == "block32_e4m3" else K // 2
                assert -(-M // tile[0]) * -(-N // 128) * tile[2] <= 152 and tile[2] <= -(-bytes_ // 128)
        assert seen == every


X4 = torch.zeros((4, 64), dtype=torch.bfloat16)
POS = torch.zeros((4, 1), dtype=torch.int32)
CALLS = {
    "norm": (lambda s: mx.rms_norm(X4, stream=s), lambda q: [q.codes, q.scales]),
    "norm_residual": (lambda s: mx.rms_norm(X4, None, X4, fmt="block16", stream=s),
                      lambda r: [r[0].codes, r[0].scales, r[0].row_scale, r[1]]),
    "norm_in_place": (lambda s, x=X4.clone(): mx.rms_norm(X4, None, x, out=x, stream=s), lambda r: [r[0].codes, r[0].scales]),
    "linear": (lambda s: mx.linear(tensor(4, 64), tensor(8, 64), post="gelu", stream=s), lambda y: [y]),
    "layer": (lambda s: mx.MXLinear(tensor(8, 64))(X4, post="gelu", residual=X4[:, :8], stream=s), lambda y: [y]),
    "norm_linear": (lambda s: mx.MXNormLinear(mx.MXLinear(tensor(8, 64)))(X4, X4, stream=s), lambda r: list(r)),
    "norm_linear_alone": (lambda s: mx.MXNormLinear(mx.MXLinear(tensor(8, 64)))(X4, stream=s), lambda r: [r[0]]),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_streams_of_buffers_and_results(fake, monkeypatch, name):  # noqa: F811
    """Kernels go to the call's stream, and every new tensor of the result is recorded on the caller's."""
    log, seen = fake.log, []
    monkeypatch.setattr(mx, "_on_gpu", lambda *t: None)
    for f in mx.EXPORTS:
        monkeypatch.setattr(mx, f, lambda *a, f=f: log.append((f, a[-1])) or 0)
    monkeypatch.setattr(clq, "_record", lambda ts, s: seen.extend(
        (t.data_ptr(), s.cuda_stream) for t in ts if isinstance(t, torch.Tensor)))
    call, parts = CALLS[name]
    out = call(fake.side)
    work = [e for e in log if e[0] != "wait"]
    assert any(e[0].startswith("clq_mx") for e in work) and all(e[-1] == SIDE for e in work), log
    assert sorted(seen) == sorted((t.data_ptr(), HERE) for t in parts(out))
    for s in (None, FakeStream(HERE, log)):
        log.clear(), seen.clear()
        call(s)
        assert log and all(e[-1] == HERE for e in log) and not seen, log


@pytest.mark.parametrize("how", ["deepcopy", "copy", "pickle"])
def test_copies_of_positions(monkeypatch, lib, how):
    """A copy whose original is gone hands over its own pairs of each axis, alone and in a layer."""
    duplicate = {"deepcopy": copy.deepcopy, "copy": copy.copy, "pickle": lambda o: pickle.loads(pickle.dumps(o))}[how]
    seen = []

    class Host:
        rope = staticmethod(lambda *a: seen.append((a[2], a[3], a[4])) or a[0])
        mx_norm_linear = staticmethod(lambda *a: seen.append((a[13], a[14], a[15])) or (a[0], None))
    monkeypatch.setattr(clq, "_host", Host)
    first = mx.MXNormLinear(mx.MXLinear(tensor(128, 64)), rope=rope.Rope(64, (16, 24, 24), device="cpu"), heads=2)
    turns = first.rope.turns.clone()
    second = duplicate(first)
    first = None
    gc.collect()
    spoil = [(ctypes.c_int32 * 3)(7, 7, 7) for _ in range(1000)]
    X, positions = torch.zeros((4, 64), dtype=H), torch.zeros((4, 3), dtype=torch.int32)
    second(X, positions=positions)
    second.rope(X.view(4, 1, 64), positions)
    third = rope.Rope(64, (16, 24, 24), device="cpu")
    third = duplicate(third)
    third(X.view(4, 1, 64), positions)
    assert len(spoil) == 1000 and len(seen) == 3
    for t, pairs, axes in seen:
        assert axes == 3 and struct.unpack("=3i", pairs) == (8, 12, 12) and torch.equal(t, turns)
    # and without the native form
    monkeypatch.setattr(clq, "_host", None)
    monkeypatch.setattr(clq, "_find_host", lambda: None)
    monkeypatch.setattr(rope, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(rope, "_stream", lambda s: None)
    monkeypatch.setattr(rope, "clq_rope", lambda *a: seen.append(list(a[10])) or 0)
    third(X.view(4, 1, 64), positions)
    assert seen[-1] == [8, 12, 12]


@pytest.mark.parametrize("turns", [torch.zeros(31, dtype=torch.int64), torch.zeros(33, dtype=torch.int64),
                                   torch.zeros(32, dtype=torch.int32), torch.zeros(64, dtype=torch.int64)[::2]])
def test_frequencies_of_other_pairs_are_refused(monkeypatch, turns):
    monkeypatch.setattr(rope, "_on_gpu", lambda *t: None)
    r = rope.Rope(64, (16, 24, 24), device="cpu")
    r.turns = turns
    with pytest.raises(ValueError, match="turns"):
        r(torch.zeros((4, 1, 64), dtype=H), torch.zeros((4, 3), dtype=torch.int32))


OVERLAP = """
#include "overlap.h"
extern "C" int overlap(int64_t out, const int64_t* so, int64_t in, const int64_t* si, const int64_t* n, int64_t D) {
  const int64_t a[2] = {so[0], so[1]}, b[2] = {si[0], si[1]}, c[2] = {n[0], n[1]};
  return clq::overlaps(reinterpret_cast<void*>(out), a, reinterpret_cast<void*>(in), b, c, D);
}
"""


def test_overlap_against_sets(tmp_path):
    """The check of outputs against inputs, place by place."""
    so = str(tmp_path / "overlap.so")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build.CSRC, "-x", "c++", "-", "-o", so],
                       input=OVERLAP, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    fn = ctypes.CDLL(so).overlap
    two = ctypes.c_int64 * 2
    fn.argtypes = [ctypes.c_int64, two, ctypes.c_int64, two, two, ctypes.c_int64]
    rng = random.Random(3)
    places = lambda at, s, n, D: {at + i * s[0] + j * s[1] + c for i in range(n[0]) for j in range(n[1]) for c in range(D)}
    seen = {(a, b): 0 for a in (True, False) for b in (True, False)}
    for _ in range(60000):
        n, D = [rng.randint(1, 4), rng.randint(1, 4)], rng.randint(1, 5)
        inner = D + rng.randint(0, 4)
        outer = (n[1] - 1) * inner + D + rng.randint(0, 6)
        out_s, dims = [outer, inner], n
        if rng.random() < 0.3:
            out_s, dims = out_s[::-1], n[::-1]
        in_s = [rng.choice([s, s, s, 0, rng.randint(0, 30)]) for s in out_s]
        at = 200 + rng.randint(-outer * n[0] - 8, outer * n[0] + 8) if rng.random() < 0.9 else 200
        exact = all(k == 1 or a in (0, b) for k, a, b in zip(dims, in_s, out_s))
        same = at == 200 and all(k == 1 or a == b for k, a, b in zip(dims, in_s, out_s))
        A, B = places(200, out_s, dims, D), places(at, in_s, dims, D)
        want = not same and (bool(A & B) if exact else max(A) >= min(B) and max(B) >= min(A))
        got = bool(fn(400, two(*out_s), 2 * at, two(*in_s), two(*dims), D))
        assert got == want, (out_s, in_s, dims, D, at)
        assert got or same or not A & B
        seen[got, exact] += 1
    assert min(seen.values()) > 1000
    far = two(2 ** 62, 2 ** 62)  # extents beyond 64 bits
    assert fn(400, far, 2 ** 62, two(0, 1), two(9, 9), 8) == 1 and fn(400, far, 200, two(0, 1), two(9, 9), 8) == 0


ROW = 2 * 64  # bytes of a row of the calls below


@pytest.mark.parametrize("change", [
    dict(sum=P + ROW), dict(sum=P - ROW), dict(sum=P + 3 * ROW), dict(sum=P + 16), dict(ldx=72, ldr=64, sum=P + 16),
    dict(residual=2 * P, sum=2 * P + ROW), dict(X=4 * P, residual=2 * P, sum=2 * P + 3 * ROW - 16)])
def test_norm_refuses_a_sum_over_other_rows(lib, change):
    assert norm(**dict(BOTH, **change)) == 1


@pytest.mark.parametrize("change", [
    {}, dict(sum=P + 4 * ROW), dict(sum=P - 4 * ROW), dict(residual=8 * P, sum=8 * P),
    dict(ldx=128, ldr=128, lds=128, sum=P + ROW), dict(M=1, sum=P + ROW), dict(M=1, lds=128), dict(residual=P + ROW, sum=8 * P)])
def test_norm_takes_a_sum_beside_its_inputs(lib, change):
    assert norm(**dict(BOTH, **change)) not in (0, 1, 2, 3)  # (there is no device here)


@pytest.mark.parametrize("change,code", [
    (dict(residual=P + 64), 1), (dict(residual=P - 64), 1), (dict(residual=P + 2), 1), (dict(residual=P + 2, ldr=33), 1),
    (dict(residual=P + 32, act=2, ldr=16), 1), (dict(residual=P + 3 * 64 + 62), 1),
    (dict(residual=P), None), (dict(residual=P + 4 * 64), None), (dict(residual=P - 4 * 64), None),
    (dict(residual=P + 64, M=1), None), (dict(residual=P + 4 * 32, act=2, ldr=16), None)])
def test_product_refuses_a_residual_over_other_rows(lib, change, code):
    got = post(**dict(dict(ldr=32), **change))
    assert got == code if code else got not in (0, 1, 2, 3)


@pytest.mark.parametrize("change,code", [
    (dict(out=P + 256), 1), (dict(out=P + 128), 1), (dict(out=P - 2), 1), (dict(out=P + 2 * 512 - 2), 1), (dict(ts=0, hs=64, out=P + 128), 1),
    (dict(ts=64, hs=256, out=P + 256), 1), (dict(ts=136), 1),
    ({}, None), (dict(out=P + 2 * 512), None), (dict(ts=256, ots=256, out=P + 256), None), (dict(ts=256, ots=256, out=P + 128), 1),
    (dict(ts=256, ots=256, hs=0, out=P + 128), None), (dict(T=1, ts=8, out=P + 256), None)])
def test_rope_refuses_an_out_over_other_heads(lib, change, code):
    got = turn(**change)
    assert got == code if code else got not in (0, 1, 2, 3)


def test_columns_of_many_channels(tmp_path):
    """Exact for every number of channels that the calls take (an overflow would end the program)."""
    program = """
#include "mx_tiles.h"
#include <cstdio>
int main() {
  for (int n0 : {0, 32, 1 << 26, (1 << 27) + 32, (1 << 30) - 32})
    std::printf("%d %d ", clq::mx::first_column(n0, false), clq::mx::first_column(n0, true));
}
"""
    exe = str(tmp_path / "columns")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-I", build.CSRC, "-x", "c++", "-", "-o", exe], input=program,
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout
    assert [int(v) for v in out.split()] == [v for n in (0, 32, 2 ** 26, 2 ** 27 + 32, 2 ** 30 - 32) for v in (n, n // 2)]


def test_sizes_beyond_32_bits(monkeypatch):
    """Refused, where ctypes would cut them to what fits; a single row's stride does not count."""
    seen = []
    monkeypatch.setattr(mx, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(rope, "_on_gpu", lambda *t: None)
    for module, names in ((mx, mx.EXPORTS), (rope, rope.EXPORTS)):
        monkeypatch.setattr(module, "_stream", lambda s: None)
        for f in names:
            if f not in ("clq_mx_scale_bytes", "clq_mx_plan_bytes", "clq_mx_plan_rows"):
                monkeypatch.setattr(module, f, lambda *a, f=f: seen.append((f, a)) or 0)
    new = lambda *shape, dtype=H: torch.empty(shape, dtype=dtype, device="meta")
    far, wide = 2 ** 32 + 64, 2 ** 32 + 5
    rows = lambda n, stride: new(1).as_strided((n, 64), (stride, 1))
    long = new(1, 64).expand(wide, 64)
    r = rope.Rope(64, (16, 24, 24), device="meta")
    x, p = new(4, 2, 64), new(4, 3, dtype=torch.int32)
    for bad in (lambda: mx.quantize(rows(4, far)), lambda: mx.quantize(long), lambda: mx.rms_norm(rows(4, far)), lambda: mx.rms_norm(long),
                lambda: mx.rms_norm(new(4, 64), None, rows(4, far)), lambda: mx.rms_norm(new(4, 64), None, new(4, 64), out=rows(4, far)),
                lambda: mx.MXTensor(new(wide, 64, dtype=torch.uint8), new(*mx.scale_shape(wide, 64, "block32_e4m3"), dtype=torch.uint8), None,
                                    "block32_e4m3"),
                lambda: r(x, new(1, dtype=torch.int32).as_strided((4, 3), (far, 1))),
                lambda: r(new(1, 2, 64).expand(wide, 2, 64), new(1, 3, dtype=torch.int32).expand(wide, 3)),
                lambda: r(new(2, 1, 64).expand(2, wide, 64), new(2, 3, dtype=torch.int32))):
        with pytest.raises(ValueError, match="32-bit|must be"):
            bad()
    assert not seen
    mx.quantize(rows(1, far)), mx.rms_norm(rows(1, far), None, rows(1, far))
    r(x[:1], new(1, dtype=torch.int32).as_strided((1, 3), (far, 1)))
    ints = [[v for v in a if isinstance(v, int)] for _, a in seen]
    assert len(ints) == 3 and all(abs(v) <= 0x7FFFFFFF for call in ints for v in call)
    assert seen[0][1][4] == 64 and seen[1][1][4] == 64 and seen[1][1][6] == 64 and seen[2][1][8] == 3


@pytest.mark.parametrize("eps,taken", [(2.0 ** -149, False), (1e-40, False), (2.0 ** -126 - 2.0 ** -149, False), (2.0 ** -126, True),
                                       (1e-30, True), (3e38, True)])
def test_smallest_eps(lib, eps, taken):
    assert (norm(eps=eps) == 1) != taken
