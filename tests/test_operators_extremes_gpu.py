"""Scores and values at the ends of their types, for each kernel of the
masked attention, against the 64-bit definitions of operator_refs.py."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from test_operators_gpu import DT, Attn, i32, rand

pytestmark = pytest.mark.gpu

# (type, query heads, key heads, queries, keys, room) of a call that the kernel takes
KERNELS = {"rows": ("bf16", 24, 24, [600, 333], [600, 333], 0),        # 256-row workgroups: whole and masked tiles
           "ranges": ("bf16", 24, 3, [700, 5], [6000, 900], 6000),     # ... that divide the keys
           "few": ("bf16", 4, 2, [150, 3], [150, 90], 200),            # 32-row workgroups
           "tokens": ("bf16", 4, 2, [1, 2], [2000, 700], 2000),        # ... that divide the keys
           "f32": ("f32", 6, 2, [150, 3], [150, 90], 200)}


def call(kernel, dh, **kw):
    dtype, H, Hk, ql, kl, room = KERNELS[kernel]
    return Attn(dtype, H, Hk, dh, ql, kl, room=room, fused=False, seed=dh, **kw)


@pytest.mark.parametrize("bias", [False, True], ids=["cap", "cap+bias"])
@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("kernel", KERNELS)
def test_capped_scores_of_infinite_products(kernel, dh, bias):
    """cap * tanh(-inf / cap) is -cap, a score like any other, wherever its key
    lies: in tiles that every row sees whole, on the diagonal, in the last."""
    a = call(kernel, dh, mask="causal", cap=1.0, bias=bias)
    a.q[:, :, 0] = 1.0
    a.k[:, :, 0] = 0.0
    # the definition's infinities: tanh(-40) is -1 within 2^-113
    far = float(torch.tensor(40 * dh ** 0.5, dtype=a.k.dtype))
    finite = a.k.clone()
    for d, n in enumerate(a.kl):
        rows, fin = a.k[a.k0[d]:a.k0[d] + n], finite[a.k0[d]:a.k0[d] + n]
        for at, sign in ((slice(0, 1), -1), (slice(3, None, 7), -1), (slice(5, None, 31), 1), (slice(n - 1, n), -1)):
            rows[at, :, 0], fin[at, :, 0] = sign * float("inf"), sign * far
    a.run()
    a.k = finite
    a.check()


@pytest.mark.parametrize("rise", [15, 40, 63])
@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("kernel", KERNELS)
def test_large_values_under_rising_scores(kernel, dh, rise):
    """Scores that rise by a factor of 2^rise from tile to tile, values of some
    2^100: their number times the largest is below 2^127, so that every result is
    finite, whichever maximum the probabilities are taken relative to."""
    a = call(kernel, dh, mask="causal")
    a.q[:, :, 0] = 1.0
    for d, n in enumerate(a.kl):
        a.k[a.k0[d]:a.k0[d] + n, :, 0] = (torch.arange(n, device="cuda") // 64 * (rise * dh ** 0.5 / 1.4427))[:, None]
    a.v.mul_(2.0 ** 100)
    a.run()
    assert a.o.isfinite().all()
    a.check()


@pytest.mark.parametrize("dtype,H,nq", [("bf16", 24, 700), ("bf16", 4, 3), ("f32", 4, 40), ("f32", 24, 700)])
@pytest.mark.parametrize("mask", ["full", "causal"])
def test_attention_without_any_key(dtype, H, nq, mask):
    """Empty k and v: every query gets zeros, rows outside the documents stay."""
    q = rand(1, nq + 2, H, 64, dtype=DT[dtype])
    kv = torch.empty(0, H, 64, dtype=DT[dtype], device="cuda")
    o = torch.full_like(q, 7.0)
    s = dm.attn_shape(q, kv, kv, o, docs=2, max_q=nq, max_k=0, mask=mask)
    dm.attention(s, q, kv, kv, o, dm.attention_workspace(s), q_start=i32([0, 1, nq]))
    assert (o[:nq] == 0).all() and (o[nq:] == 7.0).all()


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 72), ("bf16", 128), ("f32", 64)])
def test_attention_many_short_documents(dtype, dh):
    """Thousands of documents of none to four rows, single tokens and whole ones."""
    n = 3001
    a = Attn(dtype, 4, 2, dh, [d % 3 for d in range(n)], [d % 5 for d in range(n)], mask="causal", fused=False, seed=dh)
    a.run()
    a.check()


def test_keys_that_are_the_values():
    """One tensor as k and v (read only)."""
    a = Attn("bf16", 8, 2, 128, [300, 40], [300, 40], fused=False, seed=1)
    a.v = a.k
    a.run()
    a.check()


def test_norm_rows_of_no_batch():
    """A row_batch out of range is cut to the modulation's rows."""
    R, D, B = 9, 264, 3
    x, mod = rand(1, R, D), rand(2, B, 3 * D, std=0.5)
    at = [-1, 0, 1, 2, 3, 2 ** 31 - 1, -2 ** 31, 100, 1]
    out = []
    for rb in (at, np.clip(at, 0, B - 1).tolist()):
        xo, h = torch.empty_like(x), torch.empty_like(x)
        s = dm.norm_shape(R, D, batch=B, pre="rms", h_dtype="f32", mod_stride=3 * D)
        dm.norm_residual(s, x, xo, h, y=x, gate=mod[:, :D], shift=mod[:, D:2 * D], scale=mod[:, 2 * D:], row_batch=i32(rb))
        out.append((xo, h))
    assert all(torch.equal(u, v) for u, v in zip(*out))
