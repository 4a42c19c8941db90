"""The kernel instantiations of the stand-alone operators that ordinary sizes
of test_operators_gpu.py do not reach: each case says which rule it is made for,
and checks on the host that it meets it."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from operator_refs import U, e4m3_tol, linear as ref_linear, norm_residual as ref_norm, spread
from test_operators_gpu import DT, Attn, close, i32, np64, quantized, rand, test_linear as check_linear, \
    test_norm_residual as check_norm

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- fp32 attention, workgroups of 32 rows
def many_rows(H, Hk, ql, kl, **kw):
    """An fp32 call of at least 512 workgroups of 32 rows (query, head)."""
    assert min(len(ql) * max(ql), sum(ql)) * (H // Hk) // 32 * Hk >= 512
    return dict(H=H, Hk=Hk, ql=ql, kl=kl, **kw)


F32 = [
    many_rows(24, 24, [401, 1, 329], [401, 1, 329]),
    many_rows(24, 8, [401, 0, 298, 5], [401, 0, 298, 5], mask="causal"),                           # odd lengths, 3 heads share keys
    many_rows(32, 4, [333, 250], [333, 250], mask="prefix", prefix=[65, 250]),                     # 8 heads
    many_rows(24, 8, [350, 333, 17], [33, 290, 0], room=300, mask="causal", cap=5.0, bias=True),   # rows without a key
    many_rows(32, 2, [257, 300], [257, 300], mask="causal", cap=30.0, bias=True, std=2.0),
    many_rows(24, 8, [690, 30], [690, 30], mask="causal", std=4.0),                                # maxima that move far
]


@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("case", range(len(F32)))
def test_attention_f32_many_rows(case, dh):
    a = Attn("f32", dh=dh, **F32[case], seed=11 * case + dh, spare=0 if F32[case].get("room") else 3)
    a.run()
    a.check()
    assert (a.o[a.q0[-1]:] == 7.0).all()


@pytest.mark.parametrize("dh", [64, 72, 128])
def test_attention_f32_many_rows_what_is_not_visible_does_not_count(dh):
    kw = many_rows(24, 24, [400, 333], [390, 333], room=400, mask="causal")
    a, b = (Attn("f32", dh=dh, **kw, seed=3, fused=False) for _ in range(2))
    for t in (a.k, a.v):
        for lo, hi in ((390, 400), (733, 800)):
            t[lo:hi:3], t[lo + 1:hi:3], t[lo + 2:hi:3] = float("nan"), float("inf"), float("-inf")
    a.run()
    b.run()
    assert torch.equal(a.o, b.o)
    b.check()
    # a visible NaN value and infinity: exactly the rows that see their key, in their column
    a.v[500, 5, 9], a.v[601, 6, dh - 1] = float("nan"), float("inf")
    a.run()
    got, want = a.o[400:].clone(), b.o[400:]
    assert got[100:, 5, 9].isnan().all() and (got[201:, 6, dh - 1] == float("inf")).all()
    got[100:, 5, 9], got[201:, 6, dh - 1] = want[100:, 5, 9], want[201:, 6, dh - 1]
    assert torch.equal(got, want) and torch.equal(a.o[:400], b.o[:400])


# ---------------------------------------------------------------- linear layers of few rows
# Rows up to 16, 32, 64 (1, 2 or 4 fragments of 16) and blocks of k below 16, below 32, from 32 on (4, 8, 16 waves; 8
# where there are 4 fragments), so that every instantiation meets a partial last block, fragment or group of columns.
FEW = [(9, 2064, 136), (16, 3968, 41), (5, 4112, 128), (31, 1936, 130), (31, 2064, 130), (29, 4112, 129), (64, 1040, 24),
       (64, 2064, 257), (50, 8192, 40)]


@pytest.mark.parametrize("act,dtype", [("none", "bf16"), ("gelu", "f32"), ("gelu", "e4m3")])
@pytest.mark.parametrize("M,K,N", FEW)
def test_linear_few_rows(M, K, N, act, dtype):
    assert M <= 64
    check_linear(M, K, N, act, dtype)


# ---------------------------------------------------------------- sums of the 8-bit matrix pipe
def pipe_bound(a, a_scale, w, w_scale):
    """What the 8-bit pipe's alignment may take from a row's sums: every 8 consecutive products are aligned to the
    largest with a last place of 2^-13 of its binade, so that each of the 7 others loses less than 2^-13 of it."""
    A, W = np.abs(a) * spread(a_scale, 1, *a.shape), np.abs(w) * spread(w_scale, 128, *w.shape)
    A, W = (torch.from_numpy(x).cuda() for x in (A, W))
    lost = torch.zeros(len(A), len(W), dtype=torch.float64, device="cuda")
    for k in range(0, A.shape[1], 8):
        top = A[:, k, None] * W[None, :, k]
        for e in range(1, 8):
            top = torch.maximum(top, A[:, k + e, None] * W[None, :, k + e])
        lost += 7 * 2.0 ** -13 * top
    return lost.cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("M,K,N", [(9, 528, 130), (60, 4112, 257), (200, 1040, 264), (1900, 272, 4400), (3990, 912, 1024)])
def test_linear_outliers_that_cancel(M, K, N, dtype):
    """Products of 448 * 448 of both signs in other groups of 8 than each other, among small ones: what is left of
    a sum is what the alignment left of the small products, and no more may be lost than it says (none of it in fp32)."""
    x, y = rand(M + K, M, K), rand(N, N, K)
    for d in (3, 90, 140):  # both of one block of 128, and of two
        sign = torch.where(rand(d, M) > 0, 1.0, -1.0)
        at, to = d, min(d + 45, K - 1)
        x[:, at], x[:, to] = 300 * sign, -300 * sign
        y[:, at], y[:, to] = 50.0, 50.0
    a, sa = quantized(x, 1)
    w, sw = quantized(y, 128)
    shape = dm.linear_shape(M, K, N, dtype=dtype)
    ws = dm.linear_fp8_workspace(shape)
    out = torch.empty(M, N, dtype=DT[dtype], device="cuda")
    osc = torch.empty(M, -(-N // 128), device="cuda") if dtype == "e4m3" else None
    dm.linear_fp8(shape, a, sa, w, sw, out, ws, out_scale=osc)
    host = [np64(t) for t in (a, sa, w, sw)]
    want, tol = ref_linear(*host, None, "none")
    if dtype != "f32":
        tol = tol + pipe_bound(*host)
    got = np64(out)
    if dtype != "e4m3":
        return close(got, want, tol + U[dtype] * (np.abs(want) + tol), "y")
    amax = np.stack([np.abs(want[:, c:c + 128]).max(1) for c in range(0, N, 128)], 1)
    atol = np.stack([tol[:, c:c + 128].max(1) for c in range(0, N, 128)], 1)
    close(np64(osc), amax / 448, atol / 448 + amax / 448 * 2.0 ** -22, "scale")
    s = spread(np64(osc), 1, M, N)
    close(got * s, want, tol + e4m3_tol(np.abs(want) + tol, s), "codes")


# ---------------------------------------------------------------- norms
# From 2048 rows on a wave owns a row: of up to 1536 and 2048 columns (6 and 8 chunks of 256)
@pytest.mark.parametrize("post,pre,ydt,hdt", [("none", "rms", "f32", "f32"), ("layer", "layer", "bf16", "bf16"), ("rms", "rms", "bf16", "e4m3")])
@pytest.mark.parametrize("R,D", [(2053, 1536), (2048, 1544), (2051, 2040), (2049, 2048)])
def test_norm_wave_per_row(R, D, post, pre, ydt, hdt):
    check_norm(R, D, post, pre, ydt, hdt)


@pytest.mark.parametrize("hdt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("R,D", [(5, 1160), (2050, 328), (3, 8192)])
def test_norm_without_a_sub_layer(R, D, hdt):
    """No y: the first norm of a block, modulated or not, x handed on or not."""
    x, mod, w = rand(R, R, D), rand(1, 3, 2 * D, std=0.5), 1 + rand(2, D, std=0.2)
    rb = [r % 3 for r in range(R)]
    shift, scale = mod[:, :D], mod[:, D:]
    xo, h = torch.empty_like(x), torch.empty(R, D, dtype=DT[hdt], device="cuda")
    hs = torch.empty(R, -(-D // 128), device="cuda") if hdt == "e4m3" else None
    s = dm.norm_shape(R, D, batch=3, pre="layer", h_dtype=hdt, res_scale=0.5, mod_stride=2 * D)
    dm.norm_residual(s, x, xo, h, w_pre=w, shift=shift, scale=scale, row_batch=i32(rb), h_scale=hs)
    assert torch.equal(xo, 0.5 * x)
    _, _, want, tol = ref_norm(np64(x), None, None, None, np64(w), np64(shift)[rb], np64(scale)[rb], "none", "layer", 0.5,
                               np.float64(np.float32(1e-6)))
    if hdt != "e4m3":
        return close(np64(h), want, tol + U[hdt] * (np.abs(want) + tol), "h")
    sc = spread(np64(hs), 1, R, D)
    close(np64(h) * sc, want, tol + e4m3_tol(np.abs(want) + tol, sc), "h")
