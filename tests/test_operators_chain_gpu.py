"""The stand-alone operators as a block uses them: packed documents, 8-bit
linear layers, norms before and after each sub-layer, against the same block
in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from operator_refs import attention as ref_attention, gelu
from test_operators_gpu import DT, i32, np64, quantized, rand

pytestmark = pytest.mark.gpu


def test_packed_block_with_8_bit_layers():
    lens, H, dh, F = [70, 1, 133], 4, 72, 576
    D, T, B = H * dh, sum(lens), len(lens)
    seed = iter(range(100))
    w = {n: rand(next(seed), *s, std=0.06) for n, s in (("qkv", (3 * D, D)), ("o", (D, D)), ("fc1", (F, D)), ("fc2", (D, F)))}
    bias = {n: rand(next(seed), v.shape[0], std=0.1, dtype=torch.bfloat16) for n, v in w.items()}
    q8 = {n: quantized(v, 128) for n, v in w.items()}
    x0, mod = rand(next(seed), T, D), rand(next(seed), B, 6 * D, std=0.3)
    w_post, w_pre = 1 + rand(next(seed), D, std=0.1), 1 + rand(next(seed), D, std=0.1)
    rb = [d for d, n in enumerate(lens) for _ in range(n)]
    start = i32(np.concatenate([[0], np.cumsum(lens)]))
    sh1, sc1, g1, sh2, sc2, g2 = (mod[:, i * D:(i + 1) * D] for i in range(6))

    def buf(*s, dt="bf16"):
        return torch.empty(*s, dtype=DT[dt], device="cuda")

    def linear(n, a, sa, act="none", dtype="bf16"):
        N, K = w[n].shape
        s = dm.linear_shape(T, K, N, act=act, dtype=dtype)
        out, osc = buf(T, N, dt=dtype), buf(T, -(-N // 128), dt="f32") if dtype == "e4m3" else None
        dm.linear_fp8(s, a, sa, *q8[n], out, dm.linear_fp8_workspace(s), bias=bias[n], out_scale=osc)
        return out if osc is None else (out, osc)

    x, h, hs = x0.clone(), buf(T, D, dt="e4m3"), buf(T, -(-D // 128), dt="f32")
    kw = dict(w_pre=w_pre, row_batch=i32(rb), h_scale=hs)
    dm.norm_residual(dm.norm_shape(T, D, batch=B, pre="rms", h_dtype="e4m3", mod_stride=6 * D), x, None, h, shift=sh1, scale=sc1, **kw)
    qkv = linear("qkv", h, hs).view(T, 3 * H, dh)
    o = buf(T, H, dh)
    s = dm.attn_shape(qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], o, docs=B, max_q=max(lens), max_k=max(lens), cap=20.0)
    dm.attention(s, qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], o, dm.attention_workspace(s), q_start=start, k_start=start)
    y = linear("o", *quantized(o.view(T, D), 1))
    ns = dm.norm_shape(T, D, batch=B, post="rms", pre="rms", y_dtype="bf16", h_dtype="e4m3", mod_stride=6 * D)
    dm.norm_residual(ns, x, x, h, y=y, w_post=w_post, gate=g1, shift=sh2, scale=sc2, **kw)
    y = linear("fc2", *linear("fc1", h, hs, act="gelu", dtype="e4m3"))
    dm.norm_residual(dm.norm_shape(T, D, batch=B, post="rms", y_dtype="bf16", mod_stride=6 * D), x, x, None, y=y, w_post=w_post,
                     gate=g2, row_batch=i32(rb))

    # the same in 64 bits, with the weights that the codes stand for
    def wt(n):
        c, sc = q8[n]
        return np64(c) * np.repeat(np.repeat(np64(sc), 128, 0)[:c.shape[0]], 128, 1)[:, :c.shape[1]]

    def rms(z):
        return z / np.sqrt((z * z).mean(-1, keepdims=True) + 1e-6)

    m = {n: np64(v)[rb] for n, v in (("sh1", sh1), ("sc1", sc1), ("g1", g1), ("sh2", sh2), ("sc2", sc2), ("g2", g2))}
    r = np64(x0)
    z = (rms(r) * np64(w_pre) * (1 + m["sc1"]) + m["sh1"]) @ wt("qkv").T + np64(bias["qkv"])
    z = z.reshape(T, 3, H, dh)
    at, parts = 0, []
    for n in lens:
        parts.append(ref_attention(z[at:at + n, 0], z[at:at + n, 1], z[at:at + n, 2], dh ** -0.5, cap=20.0)[0])
        at += n
    y1 = np.concatenate(parts).reshape(T, D) @ wt("o").T + np64(bias["o"])
    r1 = r + m["g1"] * rms(y1) * np64(w_post)
    y2 = gelu((rms(r1) * np64(w_pre) * (1 + m["sc2"]) + m["sh2"]) @ wt("fc1").T + np64(bias["fc1"])) @ wt("fc2").T + np64(bias["fc2"])
    r2 = r1 + m["g2"] * rms(y2) * np64(w_post)
    # Each 8-bit rounding is off by 2^-4 of a value at most and 2^-4 / sqrt(3) in the mean square over a binade's
    # values (0.026 measured over normal ones is lower).  A layer's output then carries 0.036 of its norm for each
    # such input before it; three of them in a row (h, o, and what q, k and v carry) stay below 0.036 * 3, the MLP's
    # two add below 0.036 * 2, and the norms after the layers and the gates' mean square (0.3) scale both.
    got = np64(x)
    err = np.linalg.norm(got - r2) / np.linalg.norm(r2 - r)
    assert err <= 0.036 * 5, err
