"""Microscaled 4-bit layers and experts (include/clq_mx.h) on torch tensors.

As ``clq``: ``clq_mx_*`` functions with the C names and arguments, tensor helpers that
allocate their outputs with torch on the call's stream and raise ``clq.ClqError`` on a
non-zero status, and the layers made of them.  Every step runs in libclq.so.

* ``quantize`` / ``dequantize``: rows <-> ``MXTensor`` (E2M1 codes, block scales), with
  the layer's swap and rotation or an activation in front;
* ``linear``: the product of two of them; ``MXLinear``: a layer;
* ``route``: tokens to experts; ``MXExperts``: a feed-forward of experts.
"""
import ctypes

import torch

from . import clq
from .clq import _buffer, _check, _dt, _elsewhere, _ptr, _row_major, _stream, _with_stream

BLOCK32, BLOCK16 = 0, 1
FORMATS = {"block32": BLOCK32, "block16": BLOCK16}
ACTS = {"none": 0, None: 0, "gelu": 1, "swiglu": 2}
SCORING = {"softmax": 0, "sigmoid": 1}
DTYPES = {torch.float16: clq.CLQ_F16, torch.bfloat16: clq.CLQ_BF16}
CLQ_F32 = 2

_P, _I, _Z, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
_SIGS = {
    "clq_mx_scale_bytes": (_Z, [_I, _I, _I]),
    "clq_mx_quantize": (_I, [_P, _I, _I, _I, _I, _P, _I, _I, _I, _P, _P, _P, _P, _I, _I, _P]),
    "clq_mx_dequantize": (_I, [_P, _P, _P, _I, _I, _I, _I, _P, _P]),
    "clq_mx_linear": (_I, [_P] * 7 + [_I] * 6 + [_P, _P]),
    "clq_mx_route": (_I, [_P, _I, _I, _I, _I, _P, _I, _I, _I, _I, _I, _I, _F, _P, _P, _P]),
    "clq_mx_plan_rows": (_I, [_I, _I, _I]),
    "clq_mx_plan_bytes": (_Z, [_I, _I, _I]),
    "clq_mx_plan": (_I, [_P, _I, _I, _I, _P, _P, _Z, _P]),
    "clq_mx_grouped_linear": (_I, [_P] * 8 + [_I] * 8 + [_P, _P]),
    "clq_mx_grouped_linear_act": (_I, [_P] * 6 + [_I] * 8 + [_P, _P, _P]),
    "clq_mx_quantize_rows": (_I, [_P, _I, _P] + [_I] * 7 + [_P, _P, _P, _P]),
    "clq_mx_combine": (_I, [_P, _I, _P, _P, _I, _I, _I, _I, _P, _P]),
}
EXPORTS = tuple(_SIGS)
_lib = None


def load():
    """libclq.so with the microscaled entry points."""
    global _lib
    if _lib is None:
        lib = clq.load()
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


# ------------------------------------------------- C-named raw entry points --
def clq_mx_scale_bytes(rows, K, fmt):
    return load().clq_mx_scale_bytes(rows, K, fmt)


def clq_mx_quantize(X, dtype, M, K, ldx, perm, b, act, fmt, codes, scales, row_scale, out_rows, k,
                    rows, stream):
    return load().clq_mx_quantize(X, dtype, M, K, ldx, perm, b, act, fmt, codes, scales, row_scale,
                                  out_rows, k, rows, stream)


def clq_mx_dequantize(codes, scales, row_scale, M, K, fmt, dtype, out, stream):
    return load().clq_mx_dequantize(codes, scales, row_scale, M, K, fmt, dtype, out, stream)


def clq_mx_linear(Xq, Xs, s_x, Wq, Ws, s_w, bias, M, N, K, b, fmt, dtype, Y, stream):
    return load().clq_mx_linear(Xq, Xs, s_x, Wq, Ws, s_w, bias, M, N, K, b, fmt, dtype, Y, stream)


def clq_mx_route(logits, dtype, T, E, ld, balance, k, scoring, groups, top_groups, group_top,
                 renormalize, scale, experts, weights, stream):
    return load().clq_mx_route(logits, dtype, T, E, ld, balance, k, scoring, groups, top_groups,
                               group_top, renormalize, scale, experts, weights, stream)


def clq_mx_plan_rows(T, k, E):
    return load().clq_mx_plan_rows(T, k, E)


def clq_mx_plan_bytes(T, k, E):
    return load().clq_mx_plan_bytes(T, k, E)


def clq_mx_plan(experts, T, k, E, out_rows, plan, plan_bytes, stream):
    return load().clq_mx_plan(experts, T, k, E, out_rows, plan, plan_bytes, stream)


def clq_mx_grouped_linear(Xq, Xs, s_x, plan, Wq, Ws, s_w, bias, T, k, E, N, K, b, fmt, dtype, Y,
                          stream):
    return load().clq_mx_grouped_linear(Xq, Xs, s_x, plan, Wq, Ws, s_w, bias, T, k, E, N, K, b,
                                        fmt, dtype, Y, stream)


def clq_mx_grouped_linear_act(Xq, Xs, plan, Wq, Ws, bias, T, k, E, N, K, b, dtype, act, Yq, Ys,
                              stream):
    return load().clq_mx_grouped_linear_act(Xq, Xs, plan, Wq, Ws, bias, T, k, E, N, K, b, dtype,
                                            act, Yq, Ys, stream)


def clq_mx_quantize_rows(X, dtype, plan, T, k, E, K, ldx, act, fmt, codes, scales, row_scale,
                         stream):
    return load().clq_mx_quantize_rows(X, dtype, plan, T, k, E, K, ldx, act, fmt, codes, scales,
                                       row_scale, stream)


def clq_mx_combine(Y, dtype, rows, weights, T, k, D, R, out, stream):
    return load().clq_mx_combine(Y, dtype, rows, weights, T, k, D, R, out, stream)


# ----------------------------------------------------------- tensor helpers --
def _format(fmt):
    if fmt not in FORMATS:
        raise ValueError("format must be one of %s, got %r" % (sorted(FORMATS), fmt))
    return FORMATS[fmt]


def scale_shape(rows, K, fmt):
    """Shape of the scale array of `rows` x K codes: the scale of row 128 i + 32 j + r, block
    4 c + q is at [i, c, r, j, q]."""
    block = 16 if _format(fmt) == BLOCK16 else 32
    return (-(-rows // 128), -(-K // (4 * block)), 32, 4, 4)


def _on(t, dtype, device, name):
    if t is not None and (t.dtype != dtype or t.device != device or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s tensor on %s" % (name, dtype, device))


def _on_gpu(*tensors):
    """The C calls take addresses: what they are of is checked here."""
    tensors = [t for t in tensors if t is not None]
    if not all(t.is_cuda and t.device == tensors[0].device for t in tensors):
        raise ValueError("expected tensors on one GPU, got %s" % [str(t.device) for t in tensors])


class MXTensor:
    """Rows of E2M1 codes: ``codes`` uint8 [.., rows, K / 2], ``scales`` uint8 [.., *scale_shape]
    and, for "block16", ``row_scale`` fp32 [.., rows]; a leading dimension is a stack (of experts'
    weights).  Code bytes that come in a wider integer type are narrowed here, once, after a look
    at them (the device is waited for; under stream capture, which cannot wait, without)."""

    def __init__(self, codes, scales, row_scale=None, fmt="block32"):
        lead, rows, K = codes.shape[:-2], codes.shape[-2], 2 * codes.shape[-1]
        if len(lead) > 1 or tuple(scales.shape) != tuple(lead) + scale_shape(rows, K, fmt):
            raise ValueError("scales of shape %s do not belong to codes of shape %s"
                             % (tuple(scales.shape), tuple(codes.shape)))
        if (row_scale is not None) != (fmt == "block16") or (
                row_scale is not None and row_scale.shape != codes.shape[:-1]):
            raise ValueError("block16 has one scale a row, block32 none")
        if codes.dtype in (torch.int16, torch.int32, torch.int64):
            if codes.numel() and not (codes.is_cuda and torch.cuda.is_current_stream_capturing()):
                lo, hi = torch.stack(torch.aminmax(codes)).tolist()
                if lo < 0 or hi > 255:
                    raise ValueError("code bytes are 0 to 255, got %d to %d" % (lo, hi))
            codes = codes.to(torch.uint8).contiguous()
        _on(codes, torch.uint8, codes.device, "codes")
        _on(scales, torch.uint8, codes.device, "scales")
        _on(row_scale, torch.float32, codes.device, "row_scale")
        self.codes, self.scales, self.row_scale, self.fmt = codes, scales, row_scale, fmt
        self.rows, self.K = rows, K

    @classmethod
    def _made(cls, codes, scales, row_scale, fmt):
        """Around arrays that a call of this module has just made."""
        t = cls.__new__(cls)
        t.codes, t.scales, t.row_scale, t.fmt = codes, scales, row_scale, fmt
        t.rows, t.K = codes.shape[0], 2 * codes.shape[1]
        return t

    def _tensors(self):
        return self.codes, self.scales, self.row_scale


def _empty(rows, K, fmt, device):
    return (torch.empty((rows, K // 2), dtype=torch.uint8, device=device),
            torch.empty(scale_shape(rows, K, fmt), dtype=torch.uint8, device=device),
            torch.empty(rows, dtype=torch.float32, device=device) if fmt == "block16" else None)


def _native(name, *args, where):
    """The native form of a call (module _clq_host): its result, or None where it does not take
    these arguments or the module is missing.  `where`: the C calls its status may be of."""
    host = clq._host or clq._find_host()
    fn = getattr(host, name, None) if host else None
    r = fn(*args) if fn is not None else None
    if type(r) is int:
        raise clq.ClqError(r & 255, where[r >> 8])
    return r


def _row_input(X, act, perm):
    """K of an input whose rows are to be quantized."""
    _row_major(X, "X")
    if act not in ACTS:
        raise ValueError("activation must be one of none, gelu, swiglu, got %r" % (act,))
    K = X.shape[1]
    if ACTS[act] == 2:
        if K % 2:
            raise ValueError("a gated input has an even number of columns")
        K //= 2
    _on(perm, torch.int32, X.device, "perm")
    if perm is not None and perm.numel() != K:
        raise ValueError("perm must have %d entries" % K)
    return K


def quantize(X, fmt="block32", perm=None, b=1, act=None, stream=None):
    """X [M, K] fp16 / bf16 ([M, 2K] for act "swiglu": 8 columns of the gate, 8 of the up half,
    and so on) -> MXTensor of act(X)[:, perm] H_b."""
    if stream is not None and _elsewhere(stream):
        return _with_stream(stream, quantize, X, fmt, perm, b, act)
    f = _format(fmt)
    r = _native("mx_quantize", X, f, perm, b, ACTS.get(act, -1), where=("clq_mx_quantize",))
    if r is not None:
        return MXTensor._made(*r, fmt)
    K = _row_input(X, act, perm)
    _on_gpu(X)
    M = X.shape[0]
    codes, scales, rows = _empty(M, K, fmt, X.device)
    _check(clq_mx_quantize(_ptr(X), _dt(X), M, K, X.stride(0), _ptr(perm), b, ACTS[act], f,
                           _ptr(codes), _ptr(scales), _ptr(rows), None, 0, M, _stream(stream)),
           "clq_mx_quantize")
    return MXTensor._made(codes, scales, rows, fmt)


def dequantize(q, dtype=torch.bfloat16, stream=None):
    """The values of an MXTensor's rows, [rows, K]."""
    if stream is not None and _elsewhere(stream):
        return _with_stream(stream, dequantize, q, dtype)
    if q.codes.dim() != 2:
        raise ValueError("expected one array of rows, got a stack")
    if dtype in DTYPES:
        r = _native("mx_dequantize", q.codes, q.scales, q.row_scale, FORMATS[q.fmt], DTYPES[dtype],
                    where=("clq_mx_dequantize",))
        if r is not None:
            return r
    _on_gpu(q.codes)
    out = torch.empty((q.rows, q.K), dtype=dtype, device=q.codes.device)
    _check(clq_mx_dequantize(_ptr(q.codes), _ptr(q.scales), _ptr(q.row_scale), q.rows, q.K,
                             _format(q.fmt), _dt(out), _ptr(out), _stream(stream)),
           "clq_mx_dequantize")
    return out


def _pair(x, w):
    if x.fmt != w.fmt or x.K != w.K:
        raise ValueError("operands differ: %s with %d codes a row, %s with %d"
                         % (x.fmt, x.K, w.fmt, w.K))


def linear(x, w, bias=None, b=1, dtype=torch.bfloat16, Y=None, stream=None):
    """x (MXTensor of M rows), w (of N rows) -> Y [M, N] = x w^T / b + bias."""
    if stream is not None and _elsewhere(stream):
        return _with_stream(stream, linear, x, w, bias, b, dtype, Y)
    _pair(x, w)
    if x.codes.dim() != 2 or w.codes.dim() != 2:
        raise ValueError("expected arrays of rows, got a stack")
    dev = x.codes.device
    _on_gpu(x.codes, w.codes)
    if Y is None:
        Y = torch.empty((x.rows, w.rows), dtype=dtype, device=dev)
    else:
        _buffer(Y, (x.rows, w.rows), dtype, dev, "Y")
    _on(bias, dtype, dev, "bias")
    if bias is not None and tuple(bias.shape) != (w.rows,):
        raise ValueError("bias must have shape (%d,)" % w.rows)
    _check(clq_mx_linear(_ptr(x.codes), _ptr(x.scales), _ptr(x.row_scale), _ptr(w.codes),
                         _ptr(w.scales), _ptr(w.row_scale), _ptr(bias), x.rows, w.rows, x.K, b,
                         _format(x.fmt), _dt(Y), _ptr(Y), _stream(stream)), "clq_mx_linear")
    return Y


class MXLinear:
    """A linear layer with microscaled 4-bit weights and activations: ``w`` holds the weights
    with the layer's swap and rotation in them."""

    def __init__(self, w, perm=None, b=1, bias=None):
        self.w, self.perm, self.b, self.bias = w, perm, b, bias

    @classmethod
    def from_weight(cls, W, fmt="block32", perm=None, b=1, bias=None):
        """From full-precision weights W [N, K]."""
        return cls(quantize(W, fmt, perm, b), perm, b, bias)

    def __call__(self, X, act=None, Y=None, stream=None):
        """Y = act(X) W^T + bias, X [M, K] (or [M, 2K], see quantize)."""
        if stream is not None and _elsewhere(stream):
            return _with_stream(stream, self, X, act, Y)
        w = self.w
        if Y is None:
            r = _native("mx_layer", X, FORMATS[w.fmt], self.perm, self.b, ACTS.get(act, -1), w.codes,
                        w.scales, w.row_scale, self.bias, where=("clq_mx_quantize", "clq_mx_linear"))
            if r is not None:
                return r
        q = quantize(X, self.w.fmt, self.perm, self.b, act)
        return linear(q, self.w, self.bias, self.b, X.dtype, Y)


class Routing:
    """``experts`` int32 [T, k] (-1: none) and ``weights`` fp32 [T, k] of E experts."""

    def __init__(self, experts, weights, E):
        if experts.dim() != 2 or weights.shape != experts.shape:
            raise ValueError("experts and weights are [T, k]")
        _on(experts, torch.int32, experts.device, "experts")
        _on(weights, torch.float32, experts.device, "weights")
        self.experts, self.weights, self.E = experts, weights, E

    @classmethod
    def _made(cls, experts, weights, E):
        r = cls.__new__(cls)
        r.experts, r.weights, r.E = experts, weights, E
        return r

    def _tensors(self):
        return self.experts, self.weights


def route(logits, k, scoring="softmax", balance=None, groups=1, top_groups=1, group_top=2,
          renormalize=True, scale=1.0, stream=None):
    """logits [T, E] (fp16, bf16 or fp32) -> Routing to k experts; see clq_mx_route for the
    scores, the groups and what a masked (-inf) logit does."""
    if stream is not None and _elsewhere(stream):
        return _with_stream(stream, route, logits, k, scoring, balance, groups, top_groups,
                            group_top, renormalize, scale)
    if scoring not in SCORING:
        raise ValueError("scoring must be one of %s, got %r" % (sorted(SCORING), scoring))
    r = _native("mx_route", logits, k, SCORING[scoring], balance, groups, top_groups, group_top,
                int(renormalize), scale, where=("clq_mx_route",))
    if r is not None:
        return Routing._made(*r, logits.shape[1])
    _row_major(logits, "logits")
    T, E = logits.shape
    _on(balance, torch.float32, logits.device, "balance")
    if balance is not None and tuple(balance.shape) != (E,):
        raise ValueError("balance must have shape (%d,)" % E)
    _on_gpu(logits)
    experts = torch.empty((T, k), dtype=torch.int32, device=logits.device)
    weights = torch.empty((T, k), dtype=torch.float32, device=logits.device)
    dtype = CLQ_F32 if logits.dtype == torch.float32 else _dt(logits)
    _check(clq_mx_route(_ptr(logits), dtype, T, E, logits.stride(0), _ptr(balance), k,
                        SCORING[scoring], groups, top_groups, group_top, int(renormalize), scale,
                        _ptr(experts), _ptr(weights), _stream(stream)), "clq_mx_route")
    return Routing._made(experts, weights, E)


def plan(routing, stream=None):
    """The rows that a routing gives its tokens -> (rows int32 [T, k], plan, how many rows there
    are at most); see clq_mx_plan."""
    if stream is not None and _elsewhere(stream):
        return _with_stream(stream, plan, routing)
    T, k = routing.experts.shape
    _on_gpu(routing.experts)
    nbytes = clq_mx_plan_bytes(T, k, routing.E)
    if nbytes == 0:
        raise clq.ClqError(2, "clq_mx_plan")
    dev = routing.experts.device
    rows = torch.empty((T, k), dtype=torch.int32, device=dev)
    space = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _check(clq_mx_plan(_ptr(routing.experts), T, k, routing.E, _ptr(rows), _ptr(space), nbytes,
                       _stream(stream)), "clq_mx_plan")
    return rows, space, clq_mx_plan_rows(T, k, routing.E)


class MXExperts:
    """A feed-forward of E experts in microscaled 4 bits: token t gets
    sum_j weight_tj (act(x W1_e^T + bias1_e) W2_e^T + bias2_e) over its experts e.

    ``w1``: stack [E, N1, K] with the swap and rotation of the input in it; act "swiglu" takes N1 =
    2 F rows, 8 of the gate, 8 of the up half, and so on, "gelu" or None N1 = F; ``w2``: stack
    [E, N, F].  The first product is rounded to the input's type; the activation is quantized."""

    def __init__(self, w1, w2, act="swiglu", perm=None, b=1, bias1=None, bias2=None):
        if w1.codes.dim() != 3 or w2.codes.dim() != 3 or w1.codes.shape[0] != w2.codes.shape[0]:
            raise ValueError("w1 and w2 are stacks of one matrix an expert")
        if act not in ACTS or w1.rows != w2.K * (2 if ACTS[act] == 2 else 1) or w1.fmt != w2.fmt:
            raise ValueError("w1's rows, w2's columns, their formats and the activation differ")
        self.E = w1.codes.shape[0]
        for bias, n, name in ((bias1, w1.rows, "bias1"), (bias2, w2.rows, "bias2")):
            if bias is not None and tuple(bias.shape) != (self.E, n):
                raise ValueError("%s must have shape (%d, %d)" % (name, self.E, n))
        self.w1, self.w2, self.act, self.perm, self.b = w1, w2, act, perm, b
        self.bias1, self.bias2 = bias1, bias2

    @classmethod
    def from_weights(cls, W1, W2, fmt="block32", act="swiglu", perm=None, b=1, bias1=None,
                     bias2=None):
        """From full-precision weights W1 [E, N1, K] (gated: its rows in the order that the class
        takes, eight of the gate, eight of the up half), W2 [E, N, F]."""
        def stack(W, perm, b):
            q = [quantize(w, fmt, perm, b) for w in W]
            return MXTensor(torch.stack([t.codes for t in q]), torch.stack([t.scales for t in q]),
                            torch.stack([t.row_scale for t in q]) if fmt == "block16" else None, fmt)
        return cls(stack(W1, perm, b), stack(W2, None, 1), act, perm, b, bias1, bias2)

    def _product(self, codes, scales, row_scale, space, w, bias, b, T, k, rows, dtype, st):
        Y = torch.empty((rows, w.rows), dtype=dtype, device=codes.device)
        _check(clq_mx_grouped_linear(_ptr(codes), _ptr(scales), _ptr(row_scale), _ptr(space),
                                     _ptr(w.codes), _ptr(w.scales), _ptr(w.row_scale), _ptr(bias),
                                     T, k, self.E, w.rows, w.K, b, _format(w.fmt), _dt(Y), _ptr(Y),
                                     st), "clq_mx_grouped_linear")
        return Y

    def __call__(self, X, routing, stream=None):
        """X [T, K], routing of its tokens -> [T, N] in X's type."""
        if stream is not None and _elsewhere(stream):
            return _with_stream(stream, self, X, routing)
        w1, w2 = self.w1, self.w2
        if routing.E == self.E:
            r = _native("mx_experts", X, routing.experts, routing.weights, FORMATS[w1.fmt], self.perm,
                        self.b, ACTS[self.act], w1.codes, w1.scales, w1.row_scale, self.bias1,
                        w2.codes, w2.scales, w2.row_scale, self.bias2,
                        where=("clq_mx_plan", "clq_mx_quantize", "clq_mx_grouped_linear",
                               "clq_mx_combine", "clq_mx_grouped_linear_act",
                               "clq_mx_quantize_rows"))
            if r is not None:
                return r
        K = _row_input(X, None, self.perm)
        T, k = routing.experts.shape
        if K != self.w1.K or X.shape[0] != T or routing.E != self.E:
            raise ValueError("X has %d rows of %d columns; the experts take %d columns, the "
                             "routing is of %d tokens to %d experts" % (X.shape[0], K, self.w1.K, T,
                                                                        routing.E))
        for bias in (self.bias1, self.bias2):
            _on(bias, X.dtype, X.device, "bias")
        _on_gpu(X, routing.experts, routing.weights, w1.codes, w2.codes)
        out = torch.empty((T, self.w2.rows), dtype=X.dtype, device=X.device)
        if T == 0:
            return out
        fmt, st, dt = self.w1.fmt, _stream(None), _dt(X)
        rows, space, R = plan(routing)
        q = _empty(R, K, fmt, X.device)
        _check(clq_mx_quantize(_ptr(X), dt, T, K, X.stride(0), _ptr(self.perm), self.b, 0,
                               _format(fmt), *map(_ptr, q), _ptr(rows), k, R, st),
               "clq_mx_quantize")
        a = _empty(R, w2.K, fmt, X.device)
        if fmt == "block32":
            _check(clq_mx_grouped_linear_act(_ptr(q[0]), _ptr(q[1]), _ptr(space), _ptr(w1.codes),
                                             _ptr(w1.scales), _ptr(self.bias1), T, k, self.E,
                                             w1.rows, K, self.b, dt, ACTS[self.act], _ptr(a[0]),
                                             _ptr(a[1]), st), "clq_mx_grouped_linear_act")
        else:  # a row's scale needs the whole row
            h = self._product(*q, space, w1, self.bias1, self.b, T, k, R, X.dtype, st)
            _check(clq_mx_quantize_rows(_ptr(h), dt, _ptr(space), T, k, self.E, w2.K, h.stride(0),
                                        ACTS[self.act], _format(fmt), *map(_ptr, a), st),
                   "clq_mx_quantize_rows")
        y = self._product(*a, space, w2, self.bias2, 1, T, k, R, X.dtype, st)
        _check(clq_mx_combine(_ptr(y), dt, _ptr(rows), _ptr(routing.weights), T, k,
                              self.w2.rows, R, _ptr(out), st), "clq_mx_combine")
        return out
