"""Queries and keys normed for each head and turned by their positions, against the
definition in 64 bits, element by element within derived bounds."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from test_operators_gpu import DT, close, i32, np64, rand

pytestmark = pytest.mark.gpu
U24 = 2.0 ** -24


def reference(x, w, norm, pairs, pairing, pos, freqs, dtype, eps=1e-6):
    """(result, tolerance) of heads x [R, H, dh] in 64 bits.

    fp32: a statistic over dh <= 256 values is a sum of 8 in a row and a tree of 5: off by 13 roundings, half of that
    under the root; root, division, the products with 1 / dh, the norm and the weight: 6 more.  A mean is off by 15
    roundings of the mean magnitude, and shifts all values.  cos and sin of an angle that is reduced in 64 bits and
    then rounded to fp32 (at most half a turn: 2^-24 pi) are off by that and 4 roundings, in bf16 (the hardware's
    functions) by 2^-18.  Products and sum: 2 roundings.  Last, half a step of bf16."""
    z, P = x.astype(np.float64), sum(pairs)
    mag = np.zeros(z.shape)
    if norm != "none":
        shift = np.abs(z).mean(-1, keepdims=True) if norm == "layer" else 0.0
        z = z - (z.mean(-1, keepdims=True) if norm == "layer" else 0.0)
        r = 1 / np.sqrt((z * z).mean(-1, keepdims=True) + eps)
        z = z * r * w
        # what an error of the mean does: to the values, and through them to the deviation
        mag = 16 * np.abs(r * w) * shift * (1 + np.abs(x).max(-1, keepdims=True) * r) + 16 * np.abs(z)
    axis = np.repeat(np.arange(len(pairs)), pairs)
    t = pos.astype(np.float64)[:, axis] * freqs if P else np.zeros((x.shape[0], 0))
    c, s = np.cos(t)[:, None], np.sin(t)[:, None]
    i, j = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if pairing == "interleaved" else (slice(0, P), slice(P, 2 * P))
    y, tol = z.copy(), mag.copy() * U24
    a, b = z[..., i], z[..., j]
    y[..., i], y[..., j] = a * c - b * s, a * s + b * c
    both = np.abs(a) + np.abs(b)
    more = (mag[..., i] + mag[..., j]) * U24 + both * (10 * U24 if dtype == "f32" else 2.0 ** -18)
    tol[..., i], tol[..., j] = more, more
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(y) + tol)
    return y, tol + 1e-37


class Qk:
    def __init__(self, R, H, Hk, dh, dtype="bf16", norm="rms", pairs=(), pairing="interleaved", far=1000, v=False, out_rows=None,
                 q_dst=None, k_dst=None, weights=True, seed=0, offset=0.0):
        dt = DT[dtype]
        self.a = (R, H, Hk, dh, dtype, norm, tuple(pairs), pairing)
        self.qkv = (rand(seed, R, H + 2 * Hk, dh, std=1.5) + offset).to(dt)
        self.q, self.k = (self.qkv[:, :H] if H else None), (self.qkv[:, H:H + Hk] if Hk else None)
        self.v = self.qkv[:, H + Hk:] if v else None
        self.w = [1 + rand(seed + n, dh, std=0.2) if weights and norm != "none" else None for n in (1, 2)]
        g = torch.Generator().manual_seed(seed + 3)
        self.pos = torch.randint(-far, far + 1, (R, len(pairs)), generator=g, dtype=torch.int64).to(torch.int32).cuda()
        self.freqs = dm.rope_freqs(pairs) if pairs else None
        n = out_rows or R
        self.q_dst, self.k_dst = (None if d is None else i32(d) for d in (q_dst, k_dst))

        def out(heads, on=True):
            return torch.full((n, heads, dh), 7.0, dtype=dt, device="cuda") if heads and on else None
        self.out = [out(H), out(Hk), out(Hk, v)]
        self.shape = dm.qk_shape(self.q, self.k, self.out[0], self.out[1], v=self.v, v_out=self.out[2], norm=norm, pairs=pairs,
                                 pairing=pairing)

    def run(self, stream=None):
        dm.qk_norm_rope(self.shape, self.q, self.k, self.out[0], self.out[1], v=self.v, v_out=self.out[2], w_q=self.w[0],
                        w_k=self.w[1], pos=self.pos if self.a[6] else None, freqs=self.freqs, q_dst=self.q_dst,
                        k_dst=self.k_dst, stream=stream)
        return self

    def check(self, q=None, k=None, v=None):
        R, H, Hk, dh, dtype, norm, pairs, pairing = self.a
        fr = np64(torch.zeros(0)) if self.freqs is None else self.freqs.cpu().numpy()
        ins = (self.q if q is None else q, self.k if k is None else k, self.v if v is None else v)
        for n, (x, w, out, dst) in enumerate(zip(ins, self.w + [None], self.out, (self.q_dst, self.k_dst, self.k_dst))):
            if x is None:
                continue
            if n == 2:
                y, tol = np64(x), np.zeros(x.shape)
            else:
                y, tol = reference(np64(x), 1.0 if w is None else np64(w), norm, pairs, pairing, self.pos.cpu().numpy(), fr, dtype)
            got, at = np64(out), np.arange(R) if dst is None else dst.cpu().numpy()
            here = (at >= 0) & (at < out.shape[0])
            close(got[at[here]], y[here], tol[here], "qkv"[n])
            rest = np.delete(got, at[here], 0)
            assert (rest == 7.0).all()


AXES = {64: (8, 12, 12), 72: (18, 18), 128: (22, 21, 21)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["rms", "layer", "none"])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
@pytest.mark.parametrize("R,H,Hk,dh", [(1, 24, 8, 128), (37, 4, 4, 72), (300, 12, 4, 64), (5, 3, 1, 128)])
def test_heads(dtype, norm, pairing, R, H, Hk, dh):
    Qk(R, H, Hk, dh, dtype, norm, AXES[dh], pairing, v=R % 2 == 1, seed=R).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["rms", "layer", "none"])
@pytest.mark.parametrize("dh,pairs,pairing", [
    (8, (4,), "halves"), (8, (1, 2), "interleaved"), (16, (3,), "interleaved"), (24, (4, 4, 4), "halves"), (40, (7, 5, 3, 1), "interleaved"),
    (128, (16, 16), "halves"), (128, (4,), "halves"), (128, (0, 33, 0), "interleaved"), (256, (64, 32, 32), "halves"),
    (200, (100,), "halves"), (256, (40, 44, 44), "interleaved"), (72, (12, 0, 12), "halves"), (72, (), "interleaved"), (64, (0, 0), "halves"), (8, (4,), "interleaved"), (16, (8,), "halves"),
    (16, (8,), "interleaved"), (32, (16,), "halves"), (24, (12,), "interleaved"), (64, (16,), "interleaved")])
def test_widths_and_parts_of_a_head(dtype, norm, dh, pairs, pairing):
    """Heads of every width, turned in part, with axes of no pair; nothing to turn at all."""
    Qk(11, 5, 2, dh, dtype, norm, pairs, pairing, v=True, seed=dh).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_positions_far_out(dtype):
    Qk(64, 4, 4, 64, dtype, "none", (16, 16), far=2 ** 31 - 1, seed=2).run().check()
    c = Qk(64, 4, 4, 64, dtype, "none", (16, 16), far=2 ** 20, seed=2)
    c.freqs = c.freqs * 1000.0  # scaled: several turns a step
    c.run().check()


@pytest.mark.parametrize("H,Hk,v", [(6, 0, False), (0, 6, False), (0, 5, True), (1, 1, True)])
def test_queries_or_keys_alone(H, Hk, v):
    Qk(19, H, Hk, 64, pairs=(32,), pairing="halves", v=v).run().check()


def test_without_weights_and_with_a_large_mean():
    Qk(9, 4, 4, 128, "f32", "layer", (64,), weights=False).run().check()
    Qk(9, 4, 4, 128, "f32", "layer", (64,), offset=100.0).run().check()
    c = Qk(9, 4, 4, 128, "bf16", "rms", (64,), seed=3)
    c.qkv.zero_()  # a head of zeros stays one
    c.run().check()
    assert not np64(c.out[0]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [4, 700])
def test_rows_that_go_elsewhere(dtype, R):
    """Into the rooms of a cache, queries in an order of their own; rows whose place is outside are not written."""
    rng = np.random.default_rng(R)
    k_dst, q_dst = rng.permutation(3 * R)[:R], rng.permutation(3 * R)[:R]
    k_dst[1], k_dst[2], q_dst[0], q_dst[3] = -1, 3 * R, -2 ** 31, 2 ** 31 - 1
    Qk(R, 8, 2, 128, dtype, "rms", (22, 21, 21), v=True, out_rows=3 * R, k_dst=k_dst.tolist(), q_dst=q_dst.tolist()).run().check()
    Qk(R, 8, 2, 128, dtype, "rms", (64,), "halves", v=True, out_rows=3 * R, k_dst=k_dst.tolist()).run().check()


def test_more_rows_than_outputs_hold():
    """Only the rows named inside the output are written."""
    Qk(10, 2, 2, 64, pairs=(32,), out_rows=3, k_dst=[5, 0, 9, 2, -1, 7, 8, 3, 4, 6], q_dst=[1, 5, 9, 7, -1, 4, 8, 3, 2, 6]).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_on_views_of_a_projection(dtype):
    c = Qk(333, 12, 4, 72, dtype, "rms", (18, 18), seed=5)
    q, k, before = c.q.clone(), c.k.clone(), c.qkv.clone()
    c.shape = dm.qk_shape(c.q, c.k, c.q, c.k, norm="rms", pairs=(18, 18))
    c.out = [c.q, c.k, None]
    c.run().check(q=q, k=k)
    assert torch.equal(c.qkv[:, 16:], before[:, 16:])


def test_outputs_by_heads_and_with_gaps():
    """Outputs laid out [heads, rows, head_dim], and rows with room behind them."""
    c = Qk(50, 6, 3, 64, pairs=(32,), v=True)
    by_head = [torch.full((h, 50, 64), 7.0, dtype=torch.bfloat16, device="cuda") for h in (6, 3)]
    wide = torch.full((50, 5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    c.out = [by_head[0].transpose(0, 1), by_head[1].transpose(0, 1), wide[:, 1:4]]
    c.shape = dm.qk_shape(c.q, c.k, *c.out[:2], v=c.v, v_out=c.out[2], pairs=(32,))
    c.run().check()
    assert (np64(wide)[:, [0, 4]] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite(dtype):
    """They stay in their head; what is not turned is not touched by angles; v is copied bit by bit."""
    c = Qk(6, 2, 2, 64, dtype, "none", (12,), v=True, seed=4)
    c.q[1, 0, 30], c.q[2, 1, 50], c.k[3, 0, 24] = float("nan"), float("inf"), float("-inf")
    raw = c.v.contiguous().view(torch.int16 if dtype == "bf16" else torch.int32)
    bits = (torch.arange(raw.numel(), device="cuda") * (97 if dtype == "bf16" else 6700417)).view(raw.shape).to(raw.dtype)
    c.v.copy_(bits.view(c.v.dtype))
    c.run()
    assert torch.equal(c.out[2].view(raw.dtype), bits)
    q, k = np64(c.out[0]), np64(c.out[1])
    for got, src in ((q, np64(c.q)), (k, np64(c.k))):
        assert np.array_equal(got[..., 24:], src[..., 24:], equal_nan=True)
        assert np.isfinite(got[..., :24]).all()
    c = Qk(6, 2, 2, 64, dtype, "rms", (12,), seed=4)
    c.run()
    clean = np64(c.out[0])
    c.q[1, 0, 30] = float("nan")
    c.run()
    got = np64(c.out[0])
    assert np.isnan(got[1, 0]).all()
    got[1, 0] = clean[1, 0]
    assert np.array_equal(got, clean)


def test_no_rows():
    Qk(0, 4, 4, 64, pairs=(32,)).run()


def test_streams_repeats_and_graphs():
    c = Qk(300, 8, 4, 128, pairs=(22, 21, 21), v=True, out_rows=500, k_dst=np.random.default_rng(0).permutation(500)[:300].tolist())
    c.run().check()
    first = [t.clone() for t in c.out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in c.out:
        t.fill_(7.0)
    side.wait_stream(torch.cuda.current_stream())
    c.run(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, c.out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for far in (10, 1000, 7):
        c.pos.copy_(c.pos.clone() + far)  # a replay reads what the positions are then
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in c.out]
        c.run().check()
        assert all(torch.equal(x, y) for x, y in zip(got, c.out))
