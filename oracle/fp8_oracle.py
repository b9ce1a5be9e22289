"""Plain fp64 references of the 8-bit linear layers and the experts.

TEST INFRASTRUCTURE ONLY: NumPy, written from the definitions in the headers
(include/echo_fp8.h, include/echo_moe.h); it shares no code with the library.
"""
from __future__ import annotations

import numpy as np

Q = 128


def _table() -> np.ndarray:
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(e == 15) & (m == 7)] = np.nan
    return np.where(c >> 7, -v, v)


TABLE = _table()
_MID = (TABLE[:126] + TABLE[1:127]) / 2   # between the magnitudes of codes i and i + 1


def encode(x) -> np.ndarray:
    """e4m3 codes of x: nearest, ties to the even code, saturating at 448."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    lo = np.searchsorted(_MID, a, side="left")     # a <= MID[lo]
    tie = (lo < 126) & (a == _MID[np.minimum(lo, 125)])
    c = np.where(tie & (lo % 2 == 1), lo + 1, lo).astype(np.uint8)
    c = np.where(np.signbit(x), c | 0x80, c)
    return np.where(np.isnan(x), 0x7F, c).astype(np.uint8)


def decode(codes) -> np.ndarray:
    return TABLE[np.asarray(codes, np.uint8)]


def spread(scales, rows, cols, block_rows) -> np.ndarray:
    """The scale of every value of a [rows][cols] matrix."""
    s = np.repeat(np.asarray(scales, np.float64), Q, axis=-1)[..., :cols]
    return s if block_rows == 1 else np.repeat(s, block_rows, axis=-2)[..., :rows, :]


def quantize(x, block_rows=1):
    """(codes, fp32 scales) of x, whose values are fp32 numbers."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape[-2:]
    p = np.zeros((*x.shape[:-2], -(-rows // block_rows) * block_rows, -(-cols // Q) * Q), np.float32)
    p[..., :rows, :cols] = x
    b = p.reshape(*x.shape[:-2], p.shape[-2] // block_rows, block_rows, p.shape[-1] // Q, Q)
    with np.errstate(all="ignore"):
        amax = np.nanmax(np.where(np.isnan(b), np.float32(0), np.abs(b)), axis=(-3, -1))
        s = (amax / np.float32(448)).astype(np.float32)
        s[s == 0] = 1
        q = (b / s[..., :, None, :, None]).astype(np.float32)
    codes = encode(q).reshape(p.shape)[..., :rows, :cols]
    return np.ascontiguousarray(codes), s


def values(codes, scales, block_rows):
    rows, cols = codes.shape[-2:]
    with np.errstate(all="ignore"):
        return decode(codes) * spread(scales, rows, cols, block_rows)


def gemm(x, xs, w, ws, residual=None):
    """(y, sum of magnitudes) in fp64."""
    a, b = values(x, xs, 1), values(w, ws, Q)
    with np.errstate(all="ignore"):
        y, m = a @ b.T, np.abs(a) @ np.abs(b).T
    return (y if residual is None else y + residual), m


def route(logits, top_k, score="softmax", num_groups=1, top_groups=1, group_top=1,
          renormalize=False, scale=1.0, bias=None):
    """(ids, weights in fp64), one token after the other."""
    T, E = logits.shape
    ids, weights = np.full((T, top_k), -1, np.int32), np.zeros((T, top_k))
    per = E // num_groups
    for t in range(T):
        z = np.asarray(logits[t], np.float64).copy()
        z[np.isnan(z)] = -np.inf
        z = np.minimum(z, np.finfo(np.float32).max)
        on = z > -np.inf
        sc = np.zeros(E)
        if on.any():
            if score == "softmax":
                sc[on] = np.exp(z[on] - z[on].max())
                sc /= sc.sum()
            else:
                with np.errstate(over="ignore"):
                    sc[on] = 1 / (1 + np.exp(-z[on]))
        key = z.copy()
        if bias is not None:
            key = np.where(on, sc + np.asarray(bias, np.float64), -np.inf)
            key[np.isnan(key)] = -np.inf
            key = np.minimum(key, np.finfo(np.float64).max)
        if num_groups > 1:
            by = np.where(key > -np.inf, sc, -np.inf) if group_top == 2 and bias is None else key
            g = -np.sort(-by.reshape(num_groups, per), axis=1)[:, :group_top].sum(1)
            g = np.minimum(g, np.finfo(np.float64).max)
            keep = np.argsort(-g, kind="stable")[:top_groups]
            out = np.ones(num_groups, bool)
            out[keep] = False
            key[np.repeat(out, per)] = -np.inf
        best = np.argsort(-key, kind="stable")[:top_k]
        best = best[key[best] > -np.inf]
        w = sc[best]
        if renormalize:
            w = w / w.sum() if w.sum() > 0 else 0 * w
        ids[t, :len(best)], weights[t, :len(best)] = best, w * float(np.float32(scale))
    return ids, weights


def experts(x, xs, ids, weights, w_gate_up, gate_up_scale, w_down, down_scale, residual=None):
    """(out, bound) in fp64: bound is how far a result may be off besides its own
    rounding, for an e4m3 step (2^-3 of the value at most) of single activation
    codes next to a border, and the rounding of an expert's output to 11 bits under
    the largest of its neighbours (here of its row)."""
    E, H, I = w_down.shape
    T = x.shape[0]
    a = values(x, xs, 1)
    out = np.zeros((T, H)) if residual is None else np.asarray(residual, np.float64).copy()
    bound = np.zeros((T, H))
    for e in range(E):
        t, j = np.nonzero(np.asarray(ids) == e)
        if not len(t):
            continue
        g = a[t] @ values(w_gate_up[e, :I], gate_up_scale[e, 0], Q).T
        u = a[t] @ values(w_gate_up[e, I:], gate_up_scale[e, 1], Q).T
        h = g / (1 + np.exp(-g)) * u
        hc, hs = np.zeros(h.shape, np.uint8), []
        for c in range(0, I, Q):
            b = h[:, c:c + Q]
            s = (np.abs(b).max(1) / 448).astype(np.float32)
            s[s == 0] = 1
            hs.append(s)
            hc[:, c:c + Q] = encode((b / s[:, None].astype(np.float64)).astype(np.float32))
        h = values(hc, np.stack(hs, 1), 1)
        d = values(w_down[e], down_scale[e], Q)
        y = h @ d.T
        wt = np.asarray(weights, np.float64)[t, j][:, None]
        np.add.at(out, t, wt * y)
        off = 2.0 ** -11 * np.abs(y) + 2.0 ** -39 * np.abs(y).max(1, keepdims=True)
        np.add.at(bound, t, np.abs(wt) * (off + 2.0 ** -3 * np.sqrt((h * h) @ (d * d).T)))
    return out, bound
