"""Inputs of the 8-bit tests, made on the host (no GPU work at import time)."""
from __future__ import annotations

import numpy as np

from oracle import fp8_oracle as FO


def bf16_round(x) -> np.ndarray:
    """fp32 values rounded to bf16 (round to nearest even), as fp32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r).astype(np.float32)


def activations(g, T, K):
    """Codes and scales of rows with strong and weak channels."""
    x = g.standard_normal((T, K)) * np.exp(g.standard_normal(K))
    return FO.quantize(bf16_round(x), 1)


def weights(g, *shape):
    """Codes and scales of N(0, 1 / fan_in) matrices with uneven rows."""
    w = g.standard_normal(shape) / np.sqrt(shape[-1]) * np.exp(0.5 * g.standard_normal((*shape[:-1], 1)))
    return FO.quantize(w.astype(np.float32), FO.Q)


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def experts_weights(g, E, H, I):
    """(w_gate_up, its scales, w_down, its scales) on the host."""
    gu, gus = weights(g, E, 2, I, H)
    return (gu.reshape(E, 2 * I, H), gus, *weights(g, E, H, I))
