"""CPU-only checks of the microscaled operators' C ABI and binding: declarations, refusals before
any launch, the argument checks of the tensor helpers, and the streams of their buffers."""
import os
import re

import pytest
import torch

from paper_2509_24416_gb300 import build, clq, mx
from test_streams_cpu import FakeStream, HERE, SIDE, fake  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # a 16-byte aligned "device" address that nothing reads


@pytest.fixture(scope="module")
def lib():
    build.build()
    return mx.load()


def test_header_matches_binding(lib):
    text = open(os.path.join(ROOT, "include", "clq_mx.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(clq_mx_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(mx.EXPORTS)
    for name in names:
        assert hasattr(lib, name) and hasattr(mx, name)


def quantize(X=P, dtype=0, M=4, K=64, ldx=64, perm=None, b=1, act=0, fmt=0, codes=P, scales=P, row_scale=None,
             out_rows=None, k=0, rows=4):
    return mx.clq_mx_quantize(X, dtype, M, K, ldx, perm, b, act, fmt, codes, scales, row_scale, out_rows, k, rows, None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), 1), (dict(fmt=2), 1), (dict(act=3), 1), (dict(act=-1), 1), (dict(M=-1), 1), (dict(rows=-1), 1),
    (dict(M=1 << 30, rows=1 << 30), 2), (dict(X=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(fmt=1), 1), (dict(out_rows=P, k=0), 1),
    (dict(K=48), 2), (dict(K=0), 2), (dict(K=16416, ldx=16416), 2), (dict(b=3), 2), (dict(b=512), 2), (dict(b=128), 2),
    (dict(ldx=32), 2), (dict(act=2), 2), (dict(rows=3), 2),
    (dict(ldx=68), 3), (dict(X=P + 8), 3), (dict(codes=P + 8), 3), (dict(scales=P + 4), 3), (dict(perm=P + 2), 3),
    (dict(fmt=1, row_scale=P + 2), 3), (dict(out_rows=P + 2, k=1), 3), (dict(M=0, X=None, codes=None, scales=None), 0)])
def test_quantize_refuses(lib, change, code):
    assert quantize(**change) == code


@pytest.mark.parametrize("args,code", [
    ((P, P, None, 4, 64, 0, 2, P), 1), ((P, P, None, 4, 64, 3, 0, P), 1), ((P, P, None, -1, 64, 0, 0, P), 1),
    ((P, P, None, 1 << 30, 64, 0, 0, P), 2), ((P, P, None, 4, 40, 0, 0, P), 2), ((P, P, None, 4, 64, 1, 0, P), 1), ((P, P, None, 4, 64, 0, 0, None), 1),
    ((P, P, None, 4, 64, 0, 0, P + 2), 3), ((P + 1, P, None, 4, 64, 0, 0, P), 3), ((None, None, None, 0, 64, 0, 0, None), 0)])
def test_dequantize_refuses(lib, args, code):
    assert mx.clq_mx_dequantize(*args, None) == code


def linear(Xq=P, Xs=P, s_x=None, Wq=P, Ws=P, s_w=None, bias=None, M=4, N=8, K=64, b=1, fmt=0, dtype=0, Y=P):
    return mx.clq_mx_linear(Xq, Xs, s_x, Wq, Ws, s_w, bias, M, N, K, b, fmt, dtype, Y, None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), 1), (dict(fmt=-1), 1), (dict(M=-1), 1), (dict(N=-1), 1), (dict(Xq=None), 1), (dict(Ws=None), 1),
    (dict(Y=None), 1), (dict(fmt=1, s_x=P), 1), (dict(fmt=1, s_w=P), 1), (dict(M=1 << 30), 2), (dict(N=1 << 30), 2), (dict(K=80), 2), (dict(b=128), 2), (dict(b=0), 2),
    (dict(Y=P + 8), 3), (dict(bias=P + 1), 3), (dict(Xs=P + 8), 3), (dict(Wq=P + 4), 3), (dict(fmt=1, s_x=P, s_w=P + 1), 3),
    (dict(M=0, Y=None), 0), (dict(N=0, Wq=None), 0)])
def test_linear_refuses(lib, change, code):
    assert linear(**change) == code


def route(logits=P, dtype=2, T=4, E=8, ld=8, balance=None, k=2, scoring=0, groups=1, top_groups=1, group_top=2, renorm=1,
          scale=1.0, experts=P, weights=P):
    return mx.clq_mx_route(logits, dtype, T, E, ld, balance, k, scoring, groups, top_groups, group_top, renorm, scale,
                           experts, weights, None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=3), 1), (dict(T=-1), 1), (dict(scoring=2), 1), (dict(group_top=3), 1), (dict(scale=float("nan")), 1),
    (dict(logits=None), 1), (dict(experts=None), 1), (dict(weights=None), 1), (dict(k=0), 2), (dict(k=9), 2), (dict(E=513, ld=513), 2),
    (dict(E=0), 2), (dict(ld=7), 2), (dict(groups=3), 2), (dict(groups=4, top_groups=5), 2), (dict(groups=0), 2),
    (dict(E=66, ld=66, groups=33), 2), (dict(logits=P + 2), 3), (dict(balance=P + 1), 3), (dict(weights=P + 2), 3),
    (dict(T=0, logits=None), 0)])
def test_route_refuses(lib, change, code):
    assert route(**change) == code


def test_plan_and_grouped_refuse(lib):
    assert mx.clq_mx_plan_rows(4, 9, 8) == 0 and mx.clq_mx_plan_bytes(4, 2, 513) == 0
    assert mx.clq_mx_plan_rows(1 << 28, 8, 8) == 0
    # every expert's rows rounded up to 128 fit
    for T, k, E in ((1, 1, 1), (5, 2, 4), (300, 8, 64), (4096, 6, 60)):
        rows = mx.clq_mx_plan_rows(T, k, E)
        most = min(E, T * k)
        assert rows % 128 == 0 and rows >= -(-(T * k - (most - 1)) // 128) * 128 + (most - 1) * 128
    nbytes = mx.clq_mx_plan_bytes(4, 2, 8)
    assert mx.clq_mx_plan(P, 4, 2, 8, P, P, nbytes - 1, None) == 2
    assert mx.clq_mx_plan(None, 4, 2, 8, P, P, nbytes, None) == 1
    assert mx.clq_mx_plan(P, 4, 2, 8, P + 2, P, nbytes, None) == 3
    assert mx.clq_mx_plan(P, 4, 9, 8, P, P, nbytes, None) == 2
    g = lambda **c: mx.clq_mx_grouped_linear(*(dict(Xq=P, Xs=P, s_x=None, plan=P, Wq=P, Ws=P, s_w=None, bias=None, T=4, k=2,
                                                    E=8, N=64, K=64, b=1, fmt=0, dtype=0, Y=P) | c).values(), None)
    assert g(plan=None) == 1 and g(Y=None) == 1 and g(fmt=1) == 1 and g(dtype=4) == 1 and g(N=-1) == 1
    assert g(k=9) == 2 and g(K=50) == 2 and g(N=1 << 30) == 2 and g(plan=P + 8) == 3 and g(T=0, Xq=None) == 0
    f = lambda **c: mx.clq_mx_grouped_linear_act(*(dict(Xq=P, Xs=P, plan=P, Wq=P, Ws=P, bias=None, T=4, k=2, E=8, N=64, K=64,
                                                        b=1, dtype=0, act=2, Yq=P, Ys=P) | c).values(), None)
    assert f(act=3) == 1 and f(Yq=None) == 1 and f(Ws=None) == 1 and f(N=96) == 2 and f(N=48, act=1) == 2 and f(K=40) == 2
    assert f(N=2 * 16416) == 2 and f(Ys=P + 8) == 3 and f(T=0, Xq=None) == 0
    q = lambda **c: mx.clq_mx_quantize_rows(*(dict(X=P, dtype=0, plan=P, T=4, k=2, E=8, K=64, ldx=128, act=2, fmt=0, codes=P,
                                                   scales=P, row_scale=None) | c).values(), None)
    assert q(act=-1) == 1 and q(X=None) == 1 and q(plan=None) == 1 and q(fmt=1) == 1 and q(k=9) == 2 and q(ldx=120) == 2
    assert q(K=48) == 2 and q(ldx=132) == 3 and q(plan=P + 4) == 3 and q(T=0, X=None) == 0
    c = lambda **c: mx.clq_mx_combine(*(dict(Y=P, dtype=0, rows=P, weights=P, T=4, k=2, D=64, R=128, out=P) | c).values(), None)
    assert c(Y=None) == 1 and c(k=0) == 1 and c(D=60) == 2 and c(D=1 << 25) == 2 and c(out=P + 8) == 3 and c(T=0, Y=None) == 0


def tensor(rows, K, fmt="block32", lead=()):
    return mx.MXTensor(torch.zeros(lead + (rows, K // 2), dtype=torch.uint8),
                       torch.zeros(lead + mx.scale_shape(rows, K, fmt), dtype=torch.uint8),
                       torch.zeros(lead + (rows,)) if fmt == "block16" else None, fmt)


def test_helpers_refuse_host_tensors():
    X, q = torch.zeros((4, 64), dtype=torch.float16), tensor(4, 64)
    for call in (lambda: mx.quantize(X), lambda: mx.dequantize(q), lambda: mx.linear(q, tensor(8, 64)),
                 lambda: mx.route(torch.zeros((4, 8)), 2), lambda: mx.MXLinear(tensor(8, 64))(X),
                 lambda: mx.plan(mx.Routing(torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)), 3))):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_helpers_refuse(monkeypatch):
    monkeypatch.setattr(mx, "_on_gpu", lambda *t: None)
    X = torch.zeros((4, 64), dtype=torch.float16)
    w = tensor(8, 64)
    with pytest.raises(ValueError):
        mx.quantize(X, "block8")
    with pytest.raises(ValueError):
        mx.quantize(X, act="relu")
    with pytest.raises(ValueError):
        mx.quantize(X, perm=torch.zeros(32, dtype=torch.int32))
    with pytest.raises(ValueError):
        mx.quantize(X.t())
    with pytest.raises(TypeError):
        mx.quantize(X.float())
    with pytest.raises(ValueError):
        mx.MXTensor(w.codes, w.scales[:, :0], None, "block32")
    with pytest.raises(ValueError):
        mx.MXTensor(w.codes, w.scales, torch.zeros(8), "block32")
    with pytest.raises(ValueError):
        mx.linear(tensor(4, 64, "block16"), w)
    with pytest.raises(ValueError):
        mx.linear(tensor(4, 96), w)
    with pytest.raises(ValueError):
        mx.linear(tensor(4, 64), w, torch.zeros(7, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        mx.linear(tensor(4, 64), w, Y=torch.zeros((4, 9), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        mx.dequantize(tensor(8, 64, lead=(2,)))
    with pytest.raises(ValueError):
        mx.route(torch.zeros((4, 8)), 2, "relu")
    with pytest.raises(ValueError):
        mx.route(torch.zeros((4, 8)), 2, balance=torch.zeros(7))
    w1, w2 = tensor(128, 64, lead=(3,)), tensor(64, 64, lead=(3,))
    layer = mx.MXExperts(w1, w2)
    for bad in (lambda: mx.MXExperts(w1, w2, act="gelu"), lambda: mx.MXExperts(w, w2),
                lambda: mx.MXExperts(w1, w2, bias1=torch.zeros((3, 64)))):
        with pytest.raises(ValueError):
            bad()
    r = mx.Routing(torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)), 3)
    for X, r in ((torch.zeros((5, 64), dtype=torch.float16), r), (torch.zeros((4, 96), dtype=torch.float16), r),
                 (torch.zeros((4, 64), dtype=torch.float16), mx.Routing(r.experts, r.weights, 4))):
        with pytest.raises(ValueError):
            layer(X, r)


def test_wider_code_bytes_are_narrowed():
    w = tensor(8, 64)
    codes = torch.arange(256).view(8, 32)
    q = mx.MXTensor(codes, w.scales)
    assert q.codes.dtype == torch.uint8 and torch.equal(q.codes.long(), codes)


X = torch.zeros((4, 64), dtype=torch.bfloat16)
CALLS = {
    "quantize": lambda s: mx.quantize(X, "block16", stream=s),
    "dequantize": lambda s: mx.dequantize(tensor(4, 64), stream=s),
    "linear": lambda s: mx.linear(tensor(4, 64), tensor(8, 64), stream=s),
    "layer": lambda s: mx.MXLinear(tensor(8, 64))(X, stream=s),
    "route": lambda s: mx.route(torch.zeros((4, 8)), 2, stream=s),
    "experts": lambda s: mx.MXExperts(tensor(128, 64, lead=(3,)), tensor(64, 64, lead=(3,)))(
        X, mx.Routing(torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)), 3), stream=s),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_buffers_belong_to_the_calls_stream(fake, monkeypatch, name):  # noqa: F811
    log = fake.log
    monkeypatch.setattr(mx, "_on_gpu", lambda *t: None)
    for f in mx.EXPORTS:
        if f not in ("clq_mx_plan_rows", "clq_mx_plan_bytes", "clq_mx_scale_bytes"):
            monkeypatch.setattr(mx, f, lambda *a, f=f: log.append((f, a[-1])) or 0)
    monkeypatch.setattr(mx, "clq_mx_plan_rows", lambda *a: 128)
    monkeypatch.setattr(mx, "clq_mx_plan_bytes", lambda *a: 256)
    CALLS[name](fake.side)
    work = [e for e in log if e[0] != "wait"]
    assert any(e[0].startswith("clq_mx") for e in work) and all(e[-1] == SIDE for e in work), log
    for s in (None, FakeStream(HERE, log)):
        log.clear()
        CALLS[name](s)
        assert log and all(e[-1] == HERE for e in log), log
