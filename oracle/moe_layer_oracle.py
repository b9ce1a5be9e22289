"""Plain fp64 reference of the 8-bit decoder layer with experts.

TEST INFRASTRUCTURE ONLY: NumPy, on the layer reference's pieces
(layer_oracle.py), the 8-bit references (fp8_oracle.py) and the C oracle's
append and attention.  Activations are rounded to bf16 where the library's
tensors are bf16 and quantised where it quantises them.
"""
from __future__ import annotations

import numpy as np

import oracle
from oracle import fp8_oracle as FO
from oracle.layer_oracle import bf, bf16_bits, bf16_value, positions, rmsnorm, rope


def quantized_weights(lw):
    """(codes, scales) of the layer's projections and experts."""
    f = lambda a: bf16_value(a).astype(np.float32)   # noqa: E731
    E, H, I = lw.num_experts, lw.hidden, lw.intermediate
    gu, gus = FO.quantize(f(lw.w_gate_up).reshape(E, 2, I, H), FO.Q)
    return dict(qkv=FO.quantize(f(lw.w_qkv), FO.Q), o=FO.quantize(f(lw.w_o), FO.Q),
                experts=(gu.reshape(E, 2 * I, H), gus, *FO.quantize(f(lw.w_down), FO.Q)))


def forward(lw, router, pool, batch, hidden_bits):
    """One layer step.  router: keyword arguments of fp8_oracle.route; pool:
    oracle.Pool (receives the new K/V).  Returns the output's bf16 bits [T][H] and
    the intermediate tensors, the routing's distance among them: how far each
    token's last chosen key is ahead of the best one left (and its groups')."""
    Hq, Hkv, D = lw.num_q_heads, lw.num_kv_heads, lw.head_dim
    w = quantized_weights(lw)
    x = bf16_value(hidden_bits)
    T = x.shape[0]
    y = bf(rmsnorm(x, bf16_value(lw.attn_norm), lw.rms_eps))
    qkv = bf(FO.gemm(*FO.quantize(y), *w["qkv"])[0])
    q = qkv[:, :Hq * D].reshape(T, Hq, D)
    k = qkv[:, Hq * D:(Hq + Hkv) * D].reshape(T, Hkv, D)
    v = qkv[:, (Hq + Hkv) * D:].reshape(T, Hkv, D)
    pos = positions(batch)
    q, k = bf(rope(q, pos, lw.rope_theta)), bf(rope(k, pos, lw.rope_theta))
    oracle.kv_append(pool, batch, bf16_bits(k), bf16_bits(v))
    att = oracle.attention(pool, batch, bf16_bits(q), Hq, 1.0 / np.sqrt(D)).reshape(T, Hq * D)
    h = bf(FO.gemm(*FO.quantize(att), *w["o"], residual=x)[0])
    y2 = bf(rmsnorm(h, bf16_value(lw.mlp_norm), lw.rms_eps))
    logits = y2 @ bf16_value(lw.w_router).T
    ids, weights = FO.route(logits, bias=lw.router_bias, **router)
    one_more = FO.route(logits, bias=lw.router_bias, **{**router, "top_k": router["top_k"] + 1})[0]
    s = 1 / (1 + np.exp(-logits)) if router["score"] == "sigmoid" else \
        np.exp(logits - np.logaddexp.reduce(logits, 1)[:, None])
    key = np.take_along_axis(s + lw.router_bias, one_more, 1)
    distance = key[:, -2] - key[:, -1]
    n, top = router.get("num_groups", 1), router.get("top_groups", 1)
    if top < n:   # and the last kept group ahead of the best one left, for each of its keys
        per_group = -np.sort(-(s + lw.router_bias).reshape(T, n, -1), axis=2)[:, :, :router["group_top"]]
        group = -np.sort(-per_group.sum(2), axis=1)
        distance = np.minimum(distance, (group[:, top - 1] - group[:, top]) / router["group_top"])
    out, _ = FO.experts(*FO.quantize(y2), ids, weights, *w["experts"], residual=h)
    return bf16_bits(out), dict(k=k, v=v, h=h, y2=y2, logits=logits, ids=ids,
                                distance=distance)
