"""The microscaled formats and operators in 64 bits, from their definitions (numpy, CPU).

Shares no code with the library.  Products are exact sums of float64 terms; where a rounding of
the library's fp32 steps could fall on the other side of a tie, ``nearest_slack`` measures by how
much a code misses the nearest one instead of asking for the same code."""
import numpy as np
import torch

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
BLOCK = {"block32": 32, "block16": 16}


def e4m3(byte):
    e, m = (byte >> 3).astype(np.int64), (byte & 7).astype(np.float64)
    return np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))


def e8m0(byte):
    return np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))


def scale_bytes(scales, rows, blocks):
    """Bytes [rows, blocks] of a tiled scale array, place by place."""
    s = scales.cpu().numpy()
    r, q = np.arange(rows)[:, None], np.arange(blocks)[None, :]
    return s[r // 128, q // 4, r % 32, r % 128 // 32, q % 4]


def codes_of(codes):
    c = codes.cpu().numpy()
    out = np.empty((c.shape[0], 2 * c.shape[1]), dtype=np.uint8)
    out[:, 0::2], out[:, 1::2] = c & 15, c >> 4
    return out


def scales_of(q):
    """Float64 scale of each block (row scales included)."""
    byte = scale_bytes(q.scales, q.rows, q.K // BLOCK[q.fmt])
    if q.fmt == "block32":
        return e8m0(byte)
    return e4m3(byte) * q.row_scale.cpu().numpy().astype(np.float64)[:, None]


def values_of(q):
    c = codes_of(q.codes)
    v = np.where(c > 7, -GRID[c & 7], GRID[c & 7])
    return v * np.repeat(scales_of(q), BLOCK[q.fmt], axis=1)


def hadamard(v, perm, b):
    if perm is not None:
        v = v[:, perm.cpu().numpy()]
    H = np.array([[1.0]])
    while H.shape[0] < b:
        H = np.block([[H, H], [H, -H]])
    return (v.reshape(-1, b) @ H).reshape(v.shape)


def act(v, name):
    if name == "gelu":
        t = torch.from_numpy(v)
        return (0.5 * t * torch.special.erfc(-t / 2 ** 0.5)).numpy()
    if name == "swiglu":
        v = v.reshape(v.shape[0], -1, 16)
        g, u = v[..., :8], v[..., 8:]
        with np.errstate(over="ignore"):
            return (g / (1 + np.exp(-g)) * u).reshape(v.shape[0], -1)
    return v


def nearest_slack(x, code):
    """How much further each code (with its sign) is from x than the nearest value, |x| first cut
    to 6."""
    x = np.clip(x, -6, 6)
    val = np.where(code > 7, -GRID[code & 7], GRID[code & 7])
    best = np.abs(np.abs(x)[..., None] - GRID).min(-1)
    return np.abs(x - val) - best


def product_bound(x, w, ref, dtype, K):
    """|y - ref| of a product accumulated in fp32 (in steps of 64 terms, each step's sum and the
    running sum rounded or cut at 2^-22 of the largest term) and rounded once to `dtype`."""
    size = np.abs(x) @ np.abs(w).T
    eps = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -133
    return eps * np.abs(ref) + (K / 64 + 4) * 2.0 ** -22 * size + tiny


def routing(logits, balance, k, scoring, groups, top_groups, group_top, renormalize=True, scale=1.0):
    """Token by token, in the order of the definition; float64.  (experts, weights, margin): margin
    is how near the choice came to another one, against the size of the scores that it compared."""
    T, E = logits.shape
    experts, weights = np.full((T, k), -1, np.int64), np.zeros((T, k))
    margin = np.full(T, np.inf)
    for t in range(T):
        x = logits[t].astype(np.float64)
        masked = np.isnan(x) | (x == -np.inf)
        x = np.minimum(x, np.finfo(np.float32).max)
        p = np.zeros(E)
        if not masked.all():
            if scoring == "softmax":
                e = np.where(masked, 0, np.exp(np.where(masked, -np.inf, x) - x[~masked].max()))
                p = e / e.sum()
            else:
                with np.errstate(over="ignore"):
                    p = np.where(masked, 0, 1 / (1 + np.exp(-x)))
        c = np.where(masked, -np.inf, p + (0 if balance is None else balance))
        if groups > 1:
            by = c.reshape(groups, -1)
            top = -np.sort(-by, axis=1)[:, :group_top].sum(1)
            order = np.argsort(-top, kind="stable")
            keep = np.zeros(groups, bool)
            keep[order[:top_groups]] = True
            a, b = top[order[top_groups - 1]], top[order[top_groups]] if top_groups < groups else -np.inf
            if np.isfinite(a) and np.isfinite(b):
                margin[t] = min(margin[t], (a - b) / max(abs(a), 2 * p.max()))
            c = np.where(np.repeat(keep, E // groups), c, -np.inf)
        order = np.argsort(-c, kind="stable")
        picked = [e for e in order[:k] if c[e] != -np.inf]
        s = order[:k + 1]
        s = s[np.isfinite(c[s])]
        if s.size > 1:
            size = np.maximum(np.abs(c[s]), p[s])
            margin[t] = min(margin[t], (-np.diff(c[s]) / np.maximum(np.maximum(size[1:], size[:-1]), 1e-300)).min())
        w = p[picked]
        if renormalize:
            w = w / w.sum() if w.sum() > 0 else 0 * w
        experts[t, :len(picked)], weights[t, :len(picked)] = picked, w * scale
    return experts, weights, margin
