"""Plain fp64 references of int8 quantisation and products, rotary positions and the
norms between blocks.

TEST INFRASTRUCTURE ONLY: the test suite is its only caller.  NumPy in fp64, sharing no
code with the library.  Beside each result stands a bound on what an evaluation in fp32
may be off, by counting roundings of 2^-24.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24      # a rounding to fp32, relative
BF = 2.0 ** -8      # a rounding to bf16
TINY = 2.0 ** -148  # two roundings among fp32's subnormal numbers


def bf16(x) -> np.ndarray:
    """Rounded to bf16, to nearest even, as fp32 (finite values)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def scale_of(top) -> np.ndarray:
    with np.errstate(over="ignore"):
        s = (np.asarray(top, np.float64) / 127.0).astype(np.float32)
    s = np.where(s == 0, np.float32(1), s)
    return np.where(np.isfinite(s), s, np.float32(np.nan)).astype(np.float32)


def quantize(x):
    """(codes, scales) of the rows of x (fp32 values)."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        s = scale_of(np.abs(x.astype(np.float64)).max(-1))   # a NaN stays one
        q = np.rint((x.astype(np.float64) / s[..., None].astype(np.float64)).astype(np.float32))
    q = np.where(np.isnan(s)[..., None], 0, np.clip(q, -127, 127))
    return q.astype(np.int8), s


def gemm(x, xs, w, ws, bias=None, residual=None):
    """(y, bound): the sum's conversion and two products by scales, then the sums."""
    total = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T   # exact: below 2^53
    v = total * xs.astype(np.float64)[:, None] * ws.astype(np.float64)
    b = 3 * U * np.abs(v) + TINY
    for more in (None if bias is None else bias, residual):
        if more is not None:
            v = v + np.asarray(more, np.float64)
            b = b + U * np.abs(v) + TINY
    return v, b * (1 + 2.0 ** -20)


def frequencies(R, theta, scaling="none", factor=1.0, low=1.0, high=32.0, original_length=0):
    f, out, m = [theta ** (-2.0 * i / R) for i in range(R // 2)], [], 1.0
    base = theta * factor ** (R / (R - 2)) if scaling == "ntk" and R > 2 else theta
    for i in range(R // 2):
        if scaling == "linear":
            out.append(f[i] / factor)
        elif scaling == "ntk":
            out.append(base ** (-2.0 * i / R))
        elif scaling == "bands":
            u = original_length * f[i] / (2 * np.pi)
            k = 1.0 if u >= high else 0.0 if u <= low else (u - low) / (high - low)
            out.append(f[i] * (k + (1 - k) / factor))
        elif scaling == "yarn":
            d = [R * np.log(original_length / (2 * np.pi * u)) / (2 * np.log(theta)) for u in (high, low)]
            lo, hi = max(np.floor(d[0]), 0), min(np.ceil(d[1]), R - 1)
            k = 1 - min(max((i - lo) / max(hi - lo, 0.001), 0), 1)
            out.append(f[i] * (k + (1 - k) / factor))
        else:
            out.append(f[i])
    if scaling == "yarn":
        m = 0.1 * np.log(factor) + 1
    return np.array(out), m


def rotate(x, pos, freq, layout="half", magnitude=1.0, inverse=False):
    """(y, bound) of heads x [T][heads][D].

    Bound: the angle is 2^-22 off at most; cos and sin come by a function good to 2
    units in the last place (2^-22 of values of at most 1), are multiplied by the
    magnitude, and two products and a sum round."""
    x = np.asarray(x, np.float64)
    r = 2 * len(freq)
    # the turns in extended precision: fp64's own product is 2^-22 off at 2^31
    turns = np.asarray(pos, np.longdouble)[:, None] * np.asarray(freq, np.longdouble) / (2 * np.longdouble("3.14159265358979323846264338327950288"))
    angle = ((turns - np.rint(turns)).astype(np.float64) * 2 * np.pi)[:, None]
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle) * (-1 if inverse else 1)
    i = np.arange(r // 2)
    a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + r // 2)
    y = x.copy()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    bound = np.zeros_like(x)
    bound[..., a] = bound[..., b] = (2.0 ** -22 + 2.0 ** -22 + 3 * U) * abs(magnitude) * (
        np.abs(x[..., a]) + np.abs(x[..., b])) + TINY
    return y, bound


def _norm(x, dx, kind, w, b, eps, adds):
    """(norm, bound) of rows x that are dx off, sums of up to `adds` roundings."""
    if kind == "none":
        return x, dx
    if kind == "layer":
        m = x.mean(-1, keepdims=True)
        dm = dx.mean(-1, keepdims=True) + adds * U * np.abs(x).mean(-1, keepdims=True)
        x, dx = x - m, dx + dm + U * np.abs(x - m)
    ms = (x * x).mean(-1, keepdims=True)
    # mean of squares: what x is off, the squares' and sums' roundings; root and reciprocal
    dms = 2 * (np.abs(x) * dx).mean(-1, keepdims=True) + (dx * dx).mean(-1, keepdims=True) + adds * U * ms
    with np.errstate(all="ignore"):
        inv = 1.0 / np.sqrt(ms + eps)
        dinv = inv * (0.5 * dms / (ms + eps) + 4 * U)
        w = np.ones(x.shape[-1]) if w is None else w
        y = x * inv * w
        dy = np.abs(w) * (dx * (inv + dinv) + np.abs(x) * dinv) + 4 * U * np.abs(y)
    if b is not None:
        y = y + b
        dy = dy + U * np.abs(y)
    return y, dy


def join(block, residual, gate=None, post="none", pre="none", post_weight=None, post_bias=None,
         pre_weight=None, pre_bias=None, post_eps=1e-5, pre_eps=1e-5, residual_scale=1.0,
         block_scale=1.0, weight_offset=0.0, adds=96):
    """((sum, bound), (y, bound)); scales and eps are the fp32 numbers nearest to those given."""
    f32 = lambda v: np.float64(np.float32(v))   # noqa: E731
    off = lambda w: None if w is None else np.asarray(w, np.float64) + f32(weight_offset)   # noqa: E731
    wide = lambda b: None if b is None else np.asarray(b, np.float64)   # noqa: E731
    r = d = 0.0
    if block is not None:
        x = np.asarray(block, np.float64)
        v, d = _norm(x, np.zeros_like(x), post, off(post_weight), wide(post_bias), f32(post_eps), adds)
        if gate is not None:
            v, d = v * np.asarray(gate, np.float64), d * np.abs(gate)
        r = v * f32(block_scale)
        d = d * abs(f32(block_scale)) + 2 * U * np.abs(r)
    if residual is not None:
        a = f32(residual_scale) * np.asarray(residual, np.float64)
        r = r + a
        d = d + U * np.abs(a) + U * np.abs(r)
    y, dy = _norm(r, d, pre, off(pre_weight), wide(pre_bias), f32(pre_eps), adds)
    slack = 1 + 2.0 ** -12
    return (r, d * slack + TINY), (y, dy * slack + TINY)


def codes(y):
    """(codes, scales) of rows y in 64 bits."""
    with np.errstate(all="ignore"):
        s = scale_of(np.abs(y).max(-1))
        q = np.rint(y / s[:, None].astype(np.float64))
    q = np.where(np.isnan(s)[:, None], 0, np.clip(q, -127, 127))
    return q.astype(np.int8), s
