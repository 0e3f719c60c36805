"""Timed cases of the microscaled 4-bit operators: quantisation, product, routing to experts and the experts' products.

Each case runs in its plain form (elementary torch operations in 32 bits) or, with ``own`` set, through the public entry
points of ``paper_2509_24416_gb300.mx``.  Both take the same tensors, in the layouts those entry points document:

* codes: uint8 [rows, K / 2], code 2j in the low nibble of byte j; E2M1: sign, then 0 0.5 1 1.5 2 3 4 6;
* scales: uint8 [ceil(rows / 128), ceil(K / block / 4), 32, 4, 4]: the scale of row 128 i + 32 j + r, block 4 c + q of the row
  is at [i, c, r, j, q]; E8M0 bytes for blocks of 32, E4M3 bytes for blocks of 16, which have an fp32 scale a row besides;
* the rows of a gated up projection: 8 of the gate, 8 of the up half, and so on.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _quantize(name, M, K, fmt, dtype, b=1, act="none"):
    return dict(name=name, kind="quantize", M=M, K=K, fmt=fmt, dtype=dtype, b=b, act=act)


def _linear(name, M, K, N, fmt, dtype, b=1, bias=True):
    return dict(name=name, kind="linear", M=M, K=K, N=N, fmt=fmt, dtype=dtype, b=b, bias=bias)


def _route(name, T, E, k, scoring, dtype="f32", balance=False, groups=1, top_groups=1, masked=0.0):
    return dict(name=name, kind="route", T=T, E=E, k=k, scoring=scoring, dtype=dtype, balance=balance, groups=groups,
                top_groups=top_groups, masked=masked)


def _experts(name, T, D, F, E, k, fmt, dtype, act="swiglu", scoring="softmax", b=1, bias=False):
    return dict(name=name, kind="experts", T=T, D=D, F=F, E=E, k=k, fmt=fmt, dtype=dtype, act=act, scoring=scoring, b=b,
                bias=bias)


def listed():
    return [
        # The input of one attention projection of a small latent, rotated as the layer's weights are: a call of microseconds.
        _quantize("quantize_256", 256, 1152, "block32", "f16", b=64),
        # The input of a video block's down projection, with the activation in front of it and a scale a row.
        _quantize("quantize_gelu_16384", 16384, 4608, "block16", "bf16", act="gelu"),
        # One token of a served model through a wide layer: the weights' bytes are the work.
        _linear("linear_1", 1, 4096, 16384, "block32", "bf16", bias=False),
        # Ragged everywhere: rows, K and N that no tile divides.
        _linear("linear_ragged_1357", 1357, 1184, 1003, "block16", "f16"),
        # QKV of one block at 1024 px (batch 2 x 4096 tokens, hidden 1152), rotated.
        _linear("linear_qkv_8192", 8192, 1152, 3456, "block32", "f16", b=64),
        # The largest: a long batch through a wide layer.
        _linear("linear_32768", 32768, 4096, 8192, "block16", "bf16"),
        # The router of a few served tokens.
        _route("route_7", 7, 64, 6, "softmax", "bf16"),
        # The router of a long prompt: balance bias, groups, and some tokens masked out.
        _route("route_32768", 32768, 256, 8, "sigmoid", balance=True, groups=8, top_groups=4, masked=0.03),
        # One decoding step of eight sequences through the experts: few rows each, latency and the touched weights' bytes.
        _experts("experts_8", 8, 2048, 1024, 64, 6, "block32", "bf16"),
        # A short ragged prompt, block16, biases, ungated activation.
        _experts("experts_333", 333, 1152, 1536, 16, 2, "block16", "f16", act="gelu", scoring="sigmoid", bias=True),
        # A prompt of 8192 tokens.
        _experts("experts_8192", 8192, 2048, 1024, 64, 8, "block32", "bf16", b=64),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _block(rng, K):
    return rng.choice([b for b in (1, 1, 16, 32, 64, 128, 256) if K % b == 0])


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "route", "experts", "experts"])
    fmt, dtype = rng.choice(["block32", "block16"]), rng.choice(["f16", "bf16"])
    if kind == "quantize":
        K = _between(rng, 256, 12288) // 32 * 32
        M = _between(rng, 1, min(32768, 16384 * 4608 // K))
        act = rng.choice(["none", "none", "gelu", "swiglu"])
        case = _quantize("", M, K, fmt, dtype, b=_block(rng, K), act=act)
    elif kind == "linear":
        K, N, M = _between(rng, 256, 12288) // 32 * 32, _between(rng, 64, 16384), _between(rng, 1, 32768)
        if rng.random() < 0.7:
            N = max(64, N // 32 * 32)
        while M * N * K > 32768 * 4096 * 8192 or M * N > 32768 * 8192:
            M = M // 2
        case = _linear("", M, K, N, fmt, dtype, b=_block(rng, K), bias=rng.random() < 0.5)
    elif kind == "route":
        E = rng.choice([8, 16, 60, 64, 128, 160, 256, 384])
        groups = rng.choice([1, 1, 4]) if E % 4 == 0 else 1
        case = _route("", _between(rng, 1, 32768), E, rng.choice([1, 2, 4, 6, 8]), rng.choice(["softmax", "sigmoid"]),
                      rng.choice(["f32", "bf16", "f16"]), balance=rng.random() < 0.5, groups=groups,
                      top_groups=rng.choice([1, 2, 3]) if groups > 1 else 1, masked=rng.choice([0.0, 0.05]))
    else:
        E, D, F = rng.choice([4, 8, 16, 60, 64, 128]), _between(rng, 256, 4096) // 32 * 32, _between(rng, 128, 4096) // 32 * 32
        while E * D * F > 64 * 2048 * 2048:
            E = E // 2
        T, k = _between(rng, 1, 8192), rng.choice([1, 2, 4])
        while T * k * D * F > 8192 * 8 * 2048 * 1024:
            T = T // 2
        case = _experts("", T, D, F, E, k, fmt, dtype, act=rng.choice(["swiglu", "gelu"]),
                        scoring=rng.choice(["softmax", "sigmoid"]), b=_block(rng, D), bias=rng.random() < 0.3)
    del case["name"]
    return case


# ------------------------------------------------------------------- inputs --
def _inputs(g, M, K, dtype):
    """N(0, 1) rows with one channel in a hundred scaled, as transformer activations have."""
    scale = torch.ones(K, device="cuda")
    at = torch.randperm(K, generator=g, device="cuda")[:max(1, K // 100)]
    scale[at] = 20 + 40 * torch.rand(at.numel(), generator=g, device="cuda")
    return (torch.randn((M, K), generator=g, device="cuda") * scale).to(DTYPES[dtype])


def _weights(g, N, K, perm, b, fmt):
    """Codes and scales of N(0, 0.02^2) weights with the layer's swap and rotation in them, as a checkpoint holds them."""
    W = (0.02 * torch.randn((N, K), generator=g, device="cuda")).bfloat16().float()
    return _codes(_rotate(W, perm, b), fmt)


def _logits(g, case):
    T, E = case["T"], case["E"]
    logits = torch.randn((T, E), generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
    if case.get("masked"):
        logits[torch.rand(T, generator=g, device="cuda") < case["masked"]] = -math.inf
    return logits.to(DTYPES[case["dtype"] if case["kind"] == "route" else "f32"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, state = case["kind"], dict(case=case)
    if kind == "route":
        state["logits"] = _logits(g, case)
        state["balance"] = 0.1 * torch.randn(case["E"], generator=g, device="cuda") if case["balance"] else None
        return state
    K = case["D"] if kind == "experts" else case["K"]
    # the swap vector goes with the rotation
    perm = torch.randperm(K, generator=g, device="cuda").to(torch.int32) if case["b"] > 1 else None
    state["perm"] = perm
    if kind == "quantize":
        state["X"] = _inputs(g, case["M"], 2 * K if case["act"] == "swiglu" else K, case["dtype"])
        return state
    if kind == "linear":
        state["X"] = _inputs(g, case["M"], K, case["dtype"])
        state["W"] = _weights(g, case["N"], K, perm, case["b"], case["fmt"])
        state["bias"] = (0.01 * torch.randn(case["N"], generator=g, device="cuda")).to(DTYPES[case["dtype"]]) if case["bias"] else None
        return state
    E, F = case["E"], case["F"]
    N1 = 2 * F if case["act"] == "swiglu" else F
    state["X"] = _inputs(g, case["T"], K, case["dtype"])
    state["logits"] = _logits(g, case)
    state["W1"] = [torch.stack(t) if t[0] is not None else None for t in zip(*(_weights(g, N1, K, perm, case["b"], case["fmt"]) for _ in range(E)))]
    state["W2"] = [torch.stack(t) if t[0] is not None else None for t in zip(*(_weights(g, K, F, None, 1, case["fmt"]) for _ in range(E)))]
    for name, n in (("bias1", N1), ("bias2", K)):
        state[name] = (0.01 * torch.randn((E, n), generator=g, device="cuda")).to(DTYPES[case["dtype"]]) if case["bias"] else None
    return state


# -------------------------------------------------------------- plain forms --
def _rotate(v, perm, b):
    """v[:, perm] H, H block diagonal of Sylvester's Hadamard matrices of order b, in the order of the fast transform."""
    if perm is not None:
        v = v[:, perm.long()]
    h = 1
    while h < b:
        v = v.view(v.shape[0], -1, 2, h)
        v = torch.stack((v[:, :, 0] + v[:, :, 1], v[:, :, 0] - v[:, :, 1]), 2).view(v.shape[0], -1)
        h *= 2
    return v


def _act(v, act):
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if act == "swiglu":
        v = v.view(v.shape[0], -1, 2, 8)
        gate, up = v[:, :, 0], v[:, :, 1]
        return (gate / (1 + torch.exp(-gate)) * up).reshape(v.shape[0], -1)
    return v


def _tiled(scales):
    R, B = scales.shape
    full = torch.zeros((-(-R // 128) * 128, -(-B // 4) * 4), dtype=torch.uint8, device=scales.device)
    full[:R, :B] = scales
    return full.view(-1, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


def _codes(v, fmt):
    """(codes, scales, row scales or None) of fp32 rows, in the layouts above."""
    R, K = v.shape
    block = 32 if fmt == "block32" else 16
    v = v.view(R, K // block, block)
    most = v.abs().amax(2)
    if fmt == "block32":
        bits = most.view(torch.int32)
        byte = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x400000)).clamp(min=0)
        inv = ((254 - byte) << 23).view(torch.float32)
        rows, scales = None, byte.to(torch.uint8)
    else:
        rows = (most.amax(1) / 2688).clamp(min=2.0 ** -100)
        sf = (most / (6 * rows[:, None])).to(torch.float8_e4m3fn)
        scales = sf.view(torch.uint8)
        inv = torch.where(scales > 0, 1 / (sf.float() * rows[:, None]), 0.0)
    x = v * inv[:, :, None]
    a = x.abs()
    i = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    i = (i + 8 * torch.signbit(x)).view(R, K)
    return i[:, 0::2] | (i[:, 1::2] << 4), _tiled(scales), rows


def _values(codes, scales, rows, fmt):
    """The fp32 values that codes and scales stand for (without the scale a row)."""
    R, K = codes.shape[0], 2 * codes.shape[1]
    i = torch.stack((codes & 15, codes >> 4), 2).view(R, K).to(torch.int32)
    m = i & 7
    mag = torch.where(m < 2, 2 * m, (2 + (m & 1)) << (m >> 1)).float() * 0.25
    v = torch.where(i > 7, -mag, mag)
    s = scales.permute(0, 3, 2, 1, 4).reshape(128 * scales.shape[0], -1)
    block = 32 if fmt == "block32" else 16
    s = s[:R, :K // block]
    if fmt == "block32":
        e = s.to(torch.int32)
        f = torch.where(e > 0, e << 23, 1 << 22).view(torch.float32)
    else:
        f = s.contiguous().view(torch.float8_e4m3fn).float()
    return (v.view(R, -1, block) * f[:, :, None]).view(R, K)


def _product(x, W, fmt, b, bias):
    """x: codes, scales and row scales of the rows; W: of the weights; fp32."""
    acc = _values(*x, fmt) @ _values(*W, fmt).t()
    if x[2] is not None:
        acc = acc * (x[2][:, None] * W[2][None, :])
    y = acc / b
    return y if bias is None else y + bias.float()


def _halves(v):
    """Sums of the rows by halves: the order is part of the definition, since the scores are compared."""
    n = 1 << (v.shape[1] - 1).bit_length()
    v = torch.nn.functional.pad(v, (0, n - v.shape[1]))
    while v.shape[1] > 1:
        v = v[:, :v.shape[1] // 2] + v[:, v.shape[1] // 2:]
    return v


def _top(c, k):
    """Indices of the k largest, ties to the lowest index."""
    return torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k]


def _routing(logits, balance, k, scoring, groups, top_groups):
    x = logits.float()
    masked = (x == -math.inf) | x.isnan()
    x = x.clamp(max=torch.finfo(torch.float32).max)
    if scoring == "softmax":
        most = x.masked_fill(masked, -math.inf).amax(1, keepdim=True)
        e = torch.exp(x - most).masked_fill(masked, 0)
        p = e / _halves(e)
    else:
        p = 1 / (1 + torch.exp(-x))
    c = p if balance is None else p + balance
    c = c.masked_fill(masked, -math.inf)
    if groups > 1:
        by = c.view(c.shape[0], groups, -1)
        two = torch.sort(by, dim=2, descending=True).values[:, :, :2]
        best = _top(two.sum(2), top_groups)
        inside = torch.zeros((c.shape[0], groups), dtype=torch.bool, device=c.device).scatter_(1, best, True)
        c = by.masked_fill(~inside[:, :, None], -math.inf).view(c.shape)
    at = _top(c, k)
    none = c.gather(1, at) == -math.inf
    w = p.gather(1, at).masked_fill(none, 0)
    total = w.sum(1, keepdim=True)
    w = torch.where(total > 0, w / total, 0.0)
    return at.masked_fill(none, -1).to(torch.int32), w


def _route_plain(state):
    case = state["case"]
    return _routing(state["logits"], state.get("balance"), case["k"], case["scoring"], case.get("groups", 1), case.get("top_groups", 1))


def _experts_plain(state):
    case, X = state["case"], state["X"]
    fmt, E, k = case["fmt"], case["E"], case["k"]
    at, w = _route_plain(state)
    slot = torch.sort(at.view(-1), stable=True)
    counts = torch.bincount(slot.values[slot.values >= 0], minlength=E).tolist()
    rows = slot.indices[at.numel() - sum(counts):]
    x = _codes(_rotate(X.float(), state["perm"], case["b"]), fmt)
    plain_scales = x[1].permute(0, 3, 2, 1, 4).reshape(128 * x[1].shape[0], -1)
    y = torch.zeros((at.numel(), X.shape[1]), device=X.device)
    begin = 0
    for e, n in enumerate(counts):
        if n == 0:
            continue
        mine = rows[begin:begin + n]
        begin += n
        token = mine // k
        xe = (x[0][token], _tiled(plain_scales[token]), None if x[2] is None else x[2][token])
        W1, W2 = ([t[e] if t is not None else None for t in state[m]] for m in ("W1", "W2"))
        b1, b2 = (state[m][e] if state[m] is not None else None for m in ("bias1", "bias2"))
        h = _product(xe, W1, fmt, case["b"], b1).to(X.dtype).float()
        y[mine] = _product(_codes(_act(h, case["act"]), fmt), W2, fmt, 1, b2).to(X.dtype).float()
    return (y.view(-1, k, X.shape[1]) * w[:, :, None]).sum(1).to(X.dtype), at


def _plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind == "route":
        return _route_plain(state)
    if kind == "experts":
        return _experts_plain(state)
    act = case.get("act", "none")
    q = _codes(_rotate(_act(state["X"].float(), act), state["perm"], case["b"]), case["fmt"])
    if kind == "quantize":
        v = _values(*q, case["fmt"])
        return (v if q[2] is None else v * q[2][:, None]).to(state["X"].dtype)
    return _product(q, state["W"], case["fmt"], case["b"], state["bias"]).to(state["X"].dtype)


# ------------------------------------------------------------ the framework --
def _handle(state):
    """The layer that a program keeps: a wrapper of the tensors in `state`."""
    from paper_2509_24416_gb300 import mx

    case = state["case"]
    if case["kind"] == "linear":
        return mx, mx.MXLinear(mx.MXTensor(*state["W"], case["fmt"]), perm=state["perm"], b=case["b"], bias=state["bias"])
    if case["kind"] == "experts":
        return mx, mx.MXExperts(mx.MXTensor(*state["W1"], case["fmt"]), mx.MXTensor(*state["W2"], case["fmt"]), act=case["act"],
                                perm=state["perm"], b=case["b"], bias1=state["bias1"], bias2=state["bias2"])
    return mx, None


def _own(state):
    case, kind = state["case"], state["case"]["kind"]
    if "handle" not in state:
        state["handle"] = _handle(state)
    mx, layer = state["handle"]
    if kind == "linear":
        return layer(state["X"])
    if kind == "quantize":
        q = mx.quantize(state["X"], case["fmt"], perm=state["perm"], b=case["b"], act=case["act"])
        return mx.dequantize(q, state["X"].dtype)
    r = mx.route(state["logits"], case["k"], scoring=case["scoring"], balance=state.get("balance"), groups=case.get("groups", 1),
                 top_groups=case.get("top_groups", 1))
    return (r.experts, r.weights) if kind == "route" else (layer(state["X"], r), r.experts)


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------------------- work --
def work(case):
    kind = case["kind"]
    if kind == "route":
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": case["T"] * (case["E"] * size + 8 * case["k"]), "flops": 8 * case["T"] * case["E"]}
    per = 0.5 + (1 / 32 if case["fmt"] == "block32" else 1 / 16)  # bytes a code
    if kind == "quantize":
        n = case["M"] * case["K"]
        stages = max(0, case["b"].bit_length() - 1)
        return {"bytes": n * ((4 if case["act"] == "swiglu" else 2) + per + 2), "flops": n * (stages + 4)}
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": 2 * M * K + N * K * per + 2 * M * N, "flops": 2 * M * K * N}
    T, D, F, E, k = (case[m] for m in ("T", "D", "F", "E", "k"))
    N1 = 2 * F if case["act"] == "swiglu" else F
    touched = E * (1 - (1 - min(k, E) / E) ** T)
    return {"bytes": 4 * T * D + 4 * T * E + touched * (N1 + F) * D * per, "flops": 2 * T * min(k, E) * (N1 + F) * D}


# ----------------------------------------------------------------- 64 bits --
def _exact_hadamard(v, perm, b):
    if perm is not None:
        v = v[:, perm.long()]
    i = torch.arange(b, device=v.device)
    both = i[:, None] & i[None, :]
    odd = sum(((both >> s) & 1) for s in range(max(1, b.bit_length()))) % 2
    return (v.view(-1, b) @ (1 - 2 * odd).double()).view(v.shape)


def _exact_quantized(v, fmt):
    """The values nearest to v in the format, by distance to every representable one."""
    block = 32 if fmt == "block32" else 16
    w = v.view(v.shape[0], -1, block)
    most = w.abs().amax(2, keepdim=True)
    if fmt == "block32":
        step = torch.exp2(torch.ceil(torch.log2(most / 6)).clamp(min=-127))
    else:
        row = (most.amax(1, keepdim=True) / 2688).clamp(min=2.0 ** -100)
        step = row * (most / (6 * row)).float().to(torch.float8_e4m3fn).double()
    x = torch.where(step > 0, w / step, 0.0)
    a = x.abs().clamp(max=6)
    unit = torch.exp2(torch.floor(torch.log2(a.clamp(min=1))) - 1)
    return (torch.sign(x) * torch.round(a / unit) * unit * step).view(v.shape)


def _exact_stored(W, fmt):
    codes, scales, rows = W
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=codes.device)
    table = torch.cat((table, -table))
    v = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
    v[:, 0::2], v[:, 1::2] = table[(codes & 15).long()], table[(codes >> 4).long()]
    R, block = codes.shape[0], 32 if fmt == "block32" else 16
    r, q = torch.arange(R, device=codes.device)[:, None], torch.arange(v.shape[1] // block, device=codes.device)[None, :]
    s = scales[r // 128, q // 4, r % 32, r % 128 // 32, q % 4]
    f = torch.exp2(s.double() - 127) if fmt == "block32" else s.view(torch.float8_e4m3fn).double() * rows.double()[:, None]
    return v * f.repeat_interleave(block, 1)


def _exact_act(v, act):
    if act == "gelu":
        return v * 0.5 * torch.special.erfc(-v / math.sqrt(2))
    if act == "swiglu":
        v = v.view(v.shape[0], -1, 16)
        return (v[..., :8] * torch.sigmoid(v[..., :8]) * v[..., 8:]).reshape(v.shape[0], -1)
    return v


def _exact_weights(state, at):
    """The weights of the chosen experts `at`: the choice itself is one of whole numbers."""
    x = state["logits"].double()
    p = torch.softmax(x, 1) if state["case"]["scoring"] == "softmax" else torch.sigmoid(x)
    w = torch.where(at >= 0, p.gather(1, at.clamp(min=0).long()).nan_to_num(0), 0.0)
    total = w.sum(1, keepdim=True)
    return torch.where(total > 0, w / total, 0.0)


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "route":
        return None, _exact_weights(state, _route_plain(state)[0])
    if work(case)["flops"] > 6e12:
        return None
    fmt, perm, b = case["fmt"], state["perm"], case["b"]
    if kind != "experts":
        q = _exact_quantized(_exact_hadamard(_exact_act(state["X"].double(), case.get("act", "none")), perm, b), fmt)
        if kind == "quantize":
            return q
        y = q @ _exact_stored(state["W"], fmt).t() / b
        return y if state["bias"] is None else y + state["bias"].double()
    at = _route_plain(state)[0]
    w = _exact_weights(state, at)
    q = _exact_quantized(_exact_hadamard(state["X"].double(), perm, b), fmt)
    y = torch.zeros_like(q)
    for e in range(case["E"]):
        token, slot = torch.nonzero(at == e, as_tuple=True)
        if token.numel() == 0:
            continue
        h = q[token] @ _exact_stored([t if t is None else t[e] for t in state["W1"]], fmt).t() / b
        h = h if state["bias1"] is None else h + state["bias1"][e].double()
        # the up projection's output is held in the layer's 16 bits
        a = _exact_quantized(_exact_act(h.to(state["X"].dtype).double(), case["act"]), fmt)
        v = a @ _exact_stored([t if t is None else t[e] for t in state["W2"]], fmt).t()
        v = v if state["bias2"] is None else v + state["bias2"][e].double()
        y[token] += v * w[token, slot][:, None]
    return y, None
