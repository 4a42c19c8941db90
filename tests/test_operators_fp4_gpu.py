"""MXFP4 quantisation and linear layers against their definitions in 64 bits: codes
and scales bit by bit, products within the bounds of fp32 sums."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from operator_refs import gelu
from test_operators_gpu import DT, close, np64, rand

pytestmark = pytest.mark.gpu
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
U24 = 2.0 ** -24


# ---------------------------------------------------------------- the definitions
def ref_scales(x):
    """Stored scales [R, C / 32] of finite or non-finite x in 64 bits, by trying every power of two."""
    amax = np.abs(x).reshape(x.shape[0], -1, 32).max(-1)
    s = np.zeros(amax.shape, dtype=np.int64)
    for e in range(-126, 128):
        s[amax >= 7.0 * 2.0 ** (e - 1)] = e + 127
    return np.where(np.isfinite(amax), s, 255)


def ref_codes(x, s):
    """Codes of x over its stored scales: to the nearest value, ties to the even code."""
    u = np.abs(x).reshape(*s.shape, 32) / 2.0 ** (s[..., None] - 127.0)
    code = np.zeros(u.shape, dtype=np.int64)
    for i in range(1, 8):
        mid = (GRID[i - 1] + GRID[i]) / 2
        code[(u > mid) | ((u == mid) & (i % 2 == 0))] = i
    code += 8 * np.signbit(x).reshape(code.shape)
    return np.where((s == 255)[..., None], 0, code).reshape(x.shape)


def values(codes, s):
    """Of nibble codes [R, C] and stored scales."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    p = np.where(s == 255, np.nan, 2.0 ** (s - 127.0))
    return (v.reshape(*s.shape, 32) * p[..., None]).reshape(codes.shape)


def nibbles(codes):
    c = codes.cpu().numpy().astype(np.int64)
    return np.stack([c & 15, c >> 4], -1).reshape(c.shape[0], -1)


def rows_of(scale, cols):
    """Panels [ceil(cols / 256), R, 8] to [R, cols / 32], the bytes behind them apart."""
    s = scale.cpu().numpy().astype(np.int64).transpose(1, 0, 2)
    s = s.reshape(s.shape[0], -1)
    return s[:, :cols // 32], s[:, cols // 32:]


def buffers(R, C):
    return (torch.full((R, C // 2), 0xAA, dtype=torch.uint8, device="cuda"),
            torch.full((-(-C // 256), R, 8), 0xAA, dtype=torch.uint8, device="cuda"))


def quantized(x):
    codes, scale = buffers(*x.shape)
    dm.quantize_fp4(x, codes, scale)
    return codes, scale


def known(x):
    codes, scale = quantized(x)
    return codes, scale, values(nibbles(codes), rows_of(scale, x.shape[1])[0])


# ---------------------------------------------------------------- quantisation
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(1, 32), (1, 256), (3, 64), (7, 288), (8, 1152), (9, 4608), (77, 544), (1030, 96)])
def test_codes_and_scales(dtype, R, C):
    x = (rand(R + C, R, C) * torch.exp2(rand(1, R, 1, std=8.0))).to(DT[dtype])
    codes, scale = quantized(x)
    s, behind = rows_of(scale, C)
    assert np.array_equal(s, ref_scales(np64(x)))
    assert np.array_equal(nibbles(codes), ref_codes(np64(x), s))
    assert not behind.any()
    for back in ("f32", "bf16"):
        y = torch.full((R, C), 7.0, dtype=DT[back], device="cuda")
        dm.dequantize_fp4(codes, scale, y)
        assert np.array_equal(np64(y), values(nibbles(codes), s))


def test_borders_and_ends_of_the_range():
    """Ties, largest values next to 7 2^e, subnormal numbers, zeros with signs, the largest number."""
    rows = []
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0, 0.0, -0.0]
    for e in (-127, -126, -125, -124, -60, 0, 1, 90, 120):
        for top in (7.0, np.nextafter(np.float32(7.0), np.float32(0)), 6.0, 4.0, 3.5, 3.4999):
            row = np.array(ties + [top] + [0.3] * (32 - len(ties) - 1), dtype=np.float64) * 2.0 ** e
            rows.append(row.astype(np.float32))
    rows.append(np.zeros(32, np.float32))
    rows.append(np.full(32, 1e-45, np.float32))
    rows.append(np.full(32, np.finfo(np.float32).max, np.float32))
    rows.append(np.full(32, 3.4e-38, np.float32))
    x = torch.from_numpy(np.stack(rows)).cuda()
    codes, scale = quantized(x)
    s, _ = rows_of(scale, 32)
    assert np.array_equal(s, ref_scales(np64(x)))
    assert np.array_equal(nibbles(codes), ref_codes(np64(x), s))
    want = values(nibbles(codes), s)
    y = torch.empty_like(x)
    dm.dequantize_fp4(codes, scale, y)
    assert np.array_equal(np64(y), np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want))
    b = torch.empty(x.shape, dtype=torch.bfloat16, device="cuda")
    dm.dequantize_fp4(codes, scale, b)
    assert np.array_equal(np64(b), np64(y))  # one and a half bits fit bf16, from 2^-128 on its subnormal ones too


def test_values_that_are_not_finite():
    """They make their own block not a number, and no other."""
    for dtype in ("f32", "bf16"):
        x = rand(3, 5, 320, dtype=DT[dtype])
        x[0, 3], x[1, 31], x[2, 32], x[3, 319] = float("nan"), float("inf"), float("-inf"), float("nan")
        codes, scale = quantized(x)
        s, behind = rows_of(scale, 320)
        want = ref_scales(np64(x))
        assert (want == 255).sum() == 4 and np.array_equal(s, want) and not behind.any()
        assert np.array_equal(nibbles(codes), ref_codes(np.nan_to_num(np64(x), nan=0.0, posinf=0.0, neginf=0.0), s))
        y = torch.empty_like(x)
        dm.dequantize_fp4(codes, scale, y)
        assert np.array_equal(np.isnan(np64(y)), np.repeat(want == 255, 32, 1))


def test_strided_rows_and_no_rows():
    full = rand(5, 40, 512, dtype=torch.bfloat16)
    x = full[::2, 64:352]
    codes, scale = quantized(x)
    assert np.array_equal(nibbles(codes), ref_codes(np64(x), rows_of(scale, 288)[0]))
    out = torch.full((40, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    dm.dequantize_fp4(codes, scale, out[::2, 64:352])
    got = np64(out)
    assert np.array_equal(got[::2, 64:352], values(nibbles(codes), rows_of(scale, 288)[0]))
    got[::2, 64:352] = 7.0
    assert (got == 7.0).all()
    codes, scale = buffers(0, 64)
    dm.quantize_fp4(full[:0, :64], codes, scale)
    dm.dequantize_fp4(codes, scale, full[:0, :64])


# ---------------------------------------------------------------- linear
class Linear:
    def __init__(self, M, K, N, act="none", dtype="bf16", bias=True, seed=0, spread=0.5):
        self.M, self.K, self.N, self.act, self.dtype = M, K, N, act, dtype
        self.a, self.a_scale, self.av = known(rand(seed, M, K) * torch.exp(rand(seed + 1, M, 1, std=spread)))
        self.w, self.w_scale, self.wv = known(rand(seed + 2, N, K, std=0.05))
        self.bias = rand(seed + 3, N, std=0.1, dtype=torch.float32 if dtype == "f32" else torch.bfloat16) if bias else None
        self.shape = dm.linear_shape(M, K, N, act=act, dtype=dtype)
        self.ws = dm.linear_fp4_workspace(self.shape)
        if self.ws is not None:
            self.ws.fill_(0xFF)  # what lies in a workspace is no input: NaN

    @classmethod
    def of(cls, a, a_scale, w, w_scale, bias, act="none", dtype="bf16"):
        """On operands that other operators made."""
        c = cls.__new__(cls)
        (c.M, K2), c.N, c.act, c.dtype, c.bias = a.shape, w.shape[0], act, dtype, bias
        c.K, c.a, c.a_scale, c.w, c.w_scale = 2 * K2, a, a_scale, w, w_scale
        c.av, c.wv = (values(nibbles(x), rows_of(s, c.K)[0]) for x, s in ((a, a_scale), (w, w_scale)))
        c.shape = dm.linear_shape(c.M, c.K, c.N, act=act, dtype=dtype)
        c.ws = dm.linear_fp4_workspace(c.shape)
        return c

    def run(self, stream=None):
        out_scale = None
        if self.dtype == "fp4":
            out, out_scale = buffers(self.M, self.N)
        else:
            out = torch.full((self.M, self.N), 7.0, dtype=DT[self.dtype], device="cuda")
        dm.linear_fp4(self.shape, self.a, self.a_scale, self.w, self.w_scale, out, self.ws, bias=self.bias, out_scale=out_scale,
                      stream=stream)
        return out if out_scale is None else (out, out_scale)

    def want(self):
        """The result in 64 bits, and how far fp32 sums may be off: products are exact, every addition rounds a
        partial sum by 2^-24 of it at most (2^-23 if it is cut off), there are at most K / 8 + 40 of them (groups of
        eight and more on the pipe, ranges of k, the bias); GELU's slope is below 1.13, and its own arithmetic is off
        by 8 roundings of its result and of the exponent, whose effect is below 2 |y| each."""
        y = self.av @ self.wv.T
        tol = (self.K / 8 + 40) * 2 * U24 * (np.abs(self.av) @ np.abs(self.wv).T)
        if self.bias is not None:
            y = y + np64(self.bias)
            tol = tol + U24 * np.abs(y)
        if self.act == "gelu":
            tol = 1.13 * tol + 24 * U24 * np.abs(y)
            y = gelu(y)
        return y, tol

    def check(self, got):
        y, tol = self.want()
        if self.dtype == "f32":
            close(np64(got), y, tol, "f32")
            assert np.linalg.norm(np64(got) - y) <= 2e-6 * np.linalg.norm(y)
        elif self.dtype == "bf16":
            close(np64(got), y, tol + 2.0 ** -8 * (np.abs(y) + tol), "bf16")
        else:
            codes, s = nibbles(got[0]), rows_of(got[1], self.N)
            assert not s[1].any()
            s = s[0]
            amax = np.abs(y).reshape(self.M, -1, 32)
            t = tol.reshape(amax.shape)
            lo, hi = (amax - t).max(-1), (amax + t).max(-1)
            p = 2.0 ** (s - 127.0)
            # the least power of two that keeps the largest value below 7 steps, for some value within tol
            assert (lo < 7 * p).all() and ((hi >= 3.5 * p) | (s == 0)).all()
            v, u = values(codes, s), y.reshape(amax.shape) / p[..., None]
            near = np.abs(np.abs(u)[..., None] - GRID).min(-1)
            close(v, y, ((near + 1e-12) * p[..., None] + 2 * t).reshape(y.shape), "fp4")


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp4"])
@pytest.mark.parametrize("M,K,N", [(1, 32, 32), (1, 1152, 128), (4, 288, 96), (16, 256, 64), (17, 96, 160), (33, 4608, 288),
                                   (64, 384, 320), (65, 160, 352), (77, 1152, 1152), (130, 2080, 256), (300, 608, 544)])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_linear(dtype, M, K, N, act):
    c = Linear(M, K, N, act=act, dtype=dtype, seed=M + N)
    c.check(c.run())


# shapes for each tile, for the kernels of few rows, and (the last two) for k divided into ranges
@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp4"])
@pytest.mark.parametrize("M,K,N", [(8000, 96, 3456), (2100, 96, 4416), (1997, 160, 4608), (4000, 2080, 1056), (2100, 352, 3456),
                                   (700, 96, 3456), (1000, 160, 2048), (600, 608, 1152), (16, 6432, 160), (40, 8224, 96),
                                   (70, 1056, 1152), (130, 4640, 352), (33, 12320, 352), (90, 1152, 4608), (300, 18432, 1152), (1000, 18400, 320)])
def test_every_tile(dtype, M, K, N):
    c = Linear(M, K, N, act="gelu" if dtype == "fp4" else "none", dtype=dtype, seed=K)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(40, 8224, 99), (130, 12320, 1), (1000, 18432, 333), (2101, 96, 4411), (1999, 288, 3453), (1, 4096, 4100), (16, 2080, 4611)])
def test_odd_widths_of_every_kind(dtype, M, K, N):
    c = Linear(M, K, N, act="gelu", dtype=dtype, seed=K)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(1, 64, 1), (3, 64, 7), (20, 320, 33), (70, 96, 131), (257, 1120, 259), (700, 64, 401)])
def test_linear_of_odd_widths(dtype, M, K, N):
    c = Linear(M, K, N, dtype=dtype, bias=M % 2 == 1, seed=7)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp4"])
@pytest.mark.parametrize("M,K,N", [(8, 96, 64), (300, 608, 544), (70, 8224, 96)])
def test_scales_behind_the_last_column_are_not_used(dtype, M, K, N):
    c = Linear(M, K, N, dtype=dtype, seed=9)
    first = c.run()
    for s in (c.a_scale, c.w_scale):
        s[-1, :, K % 256 // 32:] = 255
    again = c.run()
    for x, y in zip(*((t if isinstance(t, tuple) else (t,)) for t in (first, again))):
        assert torch.equal(x, y)
    c.check(again)


@pytest.mark.parametrize("M", [5, 300])
def test_blocks_that_are_not_numbers_reach_their_row_alone(M):
    c = Linear(M, 288, 96, seed=11)
    want = np64(c.run())
    c.a_scale[1, 2, 0] = 255  # the last block of row 2
    got = np64(c.run())
    assert np.isnan(got[2]).all()
    assert np.array_equal(np.delete(got, 2, 0), np.delete(want, 2, 0))
    c = Linear(M, 288, 96, dtype="fp4", seed=11)
    c.a_scale[1, 2, 0] = 255
    codes, scale = c.run()
    s, _ = rows_of(scale, 96)
    assert (s[2] == 255).all() and (np.delete(s, 2, 0) != 255).all() and not nibbles(codes)[2].any()


@pytest.mark.parametrize("M", [3, 400])
def test_scales_far_apart(M):
    """Powers of two from 2^-100 to 2^20 in one row: the sums hold what fp32 sums hold."""
    c = Linear(M, 512, 64, dtype="f32", bias=False, seed=13)
    e = torch.randint(27, 148, c.a_scale.shape, generator=torch.Generator().manual_seed(1), dtype=torch.uint8).cuda()
    c.a_scale.copy_(e)
    c.av = values(nibbles(c.a), rows_of(c.a_scale, 512)[0])
    y, tol = c.want()
    close(np64(c.run()), y, tol, "far")


def test_linear_of_no_rows():
    s = dm.linear_shape(0, 64, 32)
    assert dm.linear_fp4_workspace(s) is None
    a, a_s = buffers(0, 64)
    w, w_s = quantized(rand(0, 32, 64))
    dm.linear_fp4(s, a, a_s, w, w_s, torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"))


@pytest.mark.parametrize("M,K,N,dtype", [(4, 1152, 256, "fp4"), (300, 1152, 512, "bf16"), (700, 640, 576, "fp4"), (77, 12288, 352, "fp4"), (300, 18432, 1152, "fp4")])
def test_repeats_streams_and_graphs(M, K, N, dtype):
    c = Linear(M, K, N, act="gelu", dtype=dtype, seed=17)
    tup = lambda t: t if isinstance(t, tuple) else (t,)  # noqa: E731
    first = tup(c.run())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = tup(c.run())
    given = tup(c.run(stream=torch.cuda.current_stream()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = tup(c.run())
    for _ in range(3):
        for t in held:
            t.fill_(0)
        graph.replay()
        eager = tup(c.run())  # the workspace is used in between
        torch.cuda.synchronize()
        for x, *others in zip(first, on_side, given, held, eager):
            assert all(torch.equal(x, o) for o in others)
