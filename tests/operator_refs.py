"""Plain 64-bit definitions of the stand-alone operators (numpy, CPU) with the
error bounds their tests use.  A rounding is off by at most half a step: 2^-8
of the value in bf16, 2^-24 in fp32, 2^-4 in e4m3 (2^-10 absolute below its
normal range)."""
from __future__ import annotations

import numpy as np

U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def row_limits(nq, nk, mask, prefix):
    """Keys visible to each query: j < limit."""
    if mask == "full":
        return np.full(nq, nk)
    lim = np.clip(np.arange(nq) + nk - nq + 1, 0, nk)
    return np.maximum(lim, min(max(prefix, 0), nk)) if mask == "prefix" else lim


def attention(q, k, v, scale, mask="full", prefix=0, cap=0.0, slopes=None, dtype="bf16"):
    """One document: q [nq, H, dh], k, v [nk, Hk, dh] (float64, finite where
    visible).  Returns (o, tol) [nq, H, dh]."""
    nq, H, dh = q.shape
    nk, Hk = k.shape[:2]
    o, tol = np.zeros(q.shape), np.zeros(q.shape)
    lim = row_limits(nq, nk, mask, prefix)
    u = U[dtype]
    seen = np.arange(nk)[None, :] < lim[:, None]
    some = lim > 0
    if not some.any():
        return o, tol
    for h in range(H):
        kh, vh = k[:, h * Hk // H], v[:, h * Hk // H]
        s = q[:, h] @ kh.T * scale
        # fp32 products and sums of a score, the tanh, the bias, the exp
        eps = (np.abs(q[:, h]) @ np.abs(kh).T * scale) * (dh + 16) * 2.0 ** -24 + np.abs(s) * 2.0 ** -22
        if cap > 0:
            s = cap * np.tanh(s / cap)
            eps += cap * 2.0 ** -20
        if slopes is not None:
            b = slopes[h] * np.abs(np.arange(nq)[:, None] + nk - nq - np.arange(nk))
            s = s - b
            eps += b * 2.0 ** -22
        s = np.where(seen, s, -np.inf)[some]
        at = s.argmax(1)[:, None]
        p = np.exp(s - np.take_along_axis(s, at, 1))
        # a probability's relative error: its score's, that of the running maximum, its rounding
        # (to bf16 for the product with v) and the fp32 sums' over the visible terms
        rel = np.expm1(eps[some] + np.take_along_axis(eps[some], at, 1)) + 2.0 ** -21 + (u if dtype == "bf16" else 0) \
            + lim[some, None] * 2.0 ** -24
        w = p / p.sum(1, keepdims=True)
        o[some, h] = w @ vh
        tol[some, h] = 2 * (w * rel) @ np.abs(vh) + ((w * rel).sum(1)[:, None] + u) * np.abs(o[some, h]) + 1e-30
    return o, tol


def gelu(y):
    return 0.5 * y * (1 + np.tanh(np.sqrt(2 / np.pi) * (y + 0.044715 * y ** 3)))


def spread(scale, rows, R, C):
    return np.repeat(np.repeat(scale, rows, 0)[:R], 128, 1)[:, :C]


def linear(a, a_scale, w, w_scale, bias, act):
    """(y, tol): tol for what fp32 sums may be off, before any final rounding."""
    A = a * spread(a_scale, 1, *a.shape)
    W = w * spread(w_scale, 128, *w.shape)
    y, mag = A @ W.T, np.abs(A) @ np.abs(W).T
    K = a.shape[1]
    # 128 products are added in fp32 (2^-23: the matrix pipe may truncate), scaled (two roundings) and added
    # to a sum over the blocks
    tol = mag * (128 + 2 * -(-K // 128) + 8) * 2.0 ** -23
    if bias is not None:
        y, tol = y + bias, tol + 2.0 ** -23 * (np.abs(y) + np.abs(bias))
    if act == "gelu":  # its slope is below 1.13; its own arithmetic within 2^-20 of the value, and of 2^-20 at most
        tol = 1.13 * tol + 2.0 ** -20 * np.abs(y)
        y = gelu(y)
    return y, tol


def e4m3_tol(y, scale):
    """Half a step of a code, in what it stands for."""
    return np.maximum(2.0 ** -4 * np.abs(y), scale * 2.0 ** -10) * (1 + 2.0 ** -20)


def norm_residual(x, y, w_post, gate, w_pre, shift, scale, post, pre, res_scale, eps):
    """Rows of x, y with their own gate, shift and scale rows ([R, D] or None).
    Returns (x_out, tol, h, tol)."""
    one = np.ones_like(x)
    D = x.shape[1]
    N = (D // 64 + 64) * 2.0 ** -24  # an fp32 sum over D by 64 lanes or more, and what is done with it

    def norm(z, dz, kind):
        mu = z.mean(-1, keepdims=True) if kind == "layer" else np.zeros((len(z), 1))
        sd = np.sqrt(((z - mu) ** 2).mean(-1, keepdims=True) + eps)
        size = np.abs(z) + np.abs(z).mean(-1, keepdims=True)
        # an error dz of the row moves mean and deviation by no more than its rms
        rms = np.sqrt((dz ** 2).mean(-1, keepdims=True))
        n = (z - mu) / sd
        return n, (dz + rms * (1 + np.abs(n)) + N * size * (1 + np.abs(n) * 0)) / sd + N * np.abs(n)

    if y is None:
        xo, dx = res_scale * x, 2.0 ** -24 * np.abs(res_scale * x)
    else:
        n, dn = norm(y, 0 * y, post) if post != "none" else (y, 0 * y)
        f = (one if w_post is None else w_post * one) * (one if gate is None else gate)
        xo = res_scale * x + f * n
        dx = np.abs(f) * (dn + 2.0 ** -23 * np.abs(n)) + 2.0 ** -24 * np.abs(res_scale * x) + 2.0 ** -23 * np.abs(xo)
    n, dn = norm(xo, dx, pre)
    f = (one if w_pre is None else w_pre * one) * (one if scale is None else 1 + scale)
    h = f * n + (0 if shift is None else shift)
    fmag = np.abs(one if w_pre is None else w_pre * one) * (one if scale is None else 1 + np.abs(scale))
    dh = np.abs(f) * dn + 2.0 ** -22 * fmag * np.abs(n) + 2.0 ** -23 * np.abs(h)
    return xo, dx, h, dh
