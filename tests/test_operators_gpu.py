"""The stand-alone operators against their plain 64-bit definitions
(operator_refs.py), element by element within bounds derived there."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from operator_refs import U, attention as ref_attention, e4m3_tol, linear as ref_linear, norm_residual as ref_norm, \
    row_limits

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rand(seed, *shape, std=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def close(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])


# ---------------------------------------------------------------- attention
class Attn:
    """Inputs of one call; documents packed (room 0) or in rooms of `room` keys."""

    def __init__(self, dtype, H, Hk, dh, ql, kl, room=0, mask="full", prefix=None, cap=0.0, bias=False, seed=0, fused=True,
                 spare=0, max_q=None, max_k=None, std=1.0):
        dt = DT[dtype]
        self.dtype, self.ql, self.kl, self.mask, self.cap = dtype, ql, kl, mask, cap
        self.H, self.Hk, self.dh = H, Hk, dh
        tq, tk = sum(ql) + spare, len(kl) * room if room else sum(kl) + spare
        self.q0 = np.concatenate([[0], np.cumsum(ql)]).astype(int)
        self.k0 = np.arange(len(kl) + 1) * room if room else np.concatenate([[0], np.cumsum(kl)]).astype(int)
        if fused and tq == tk:
            qkv = rand(seed, tq, H + 2 * Hk, dh, std=std, dtype=dt)
            self.q, self.k, self.v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        else:
            self.q = rand(seed, tq, H, dh, std=std, dtype=dt)
            self.k, self.v = rand(seed + 1, tk, Hk, dh, std=std, dtype=dt), rand(seed + 2, tk, Hk, dh, std=std, dtype=dt)
        self.o = torch.full((tq, H, dh), 7.0, dtype=dt, device="cuda")
        self.prefix = prefix
        self.slopes = 2.0 ** (-8.0 * np.arange(1, H + 1) / H) if bias else None
        self.shape = dm.attn_shape(self.q, self.k, self.v, self.o, docs=len(ql), max_q=max_q or max(ql), max_k=max_k or max(kl),
                                   mask=mask, cap=cap)
        self.kw = dict(q_start=i32(self.q0), k_start=i32(self.k0), k_len=i32(kl) if room else None,
                       prefix=i32(prefix) if prefix is not None else None,
                       slopes=torch.tensor(self.slopes, dtype=torch.float32, device="cuda") if bias else None)
        self.ws = dm.attention_workspace(self.shape)
        if self.ws is not None:
            self.ws.fill_(0xFF)  # NaN everywhere: nothing may be read before it is written

    def run(self, **kw):
        dm.attention(self.shape, self.q, self.k, self.v, self.o, self.ws, **{**self.kw, **kw})
        return self.o

    def doc(self, t, d, n, starts):
        return np64(t[starts[d]:starts[d] + n])

    def check(self, rows=None):
        got = np64(self.o)
        for d, (nq, nk) in enumerate(zip(self.ql, self.kl)):
            q, k, v = self.doc(self.q, d, nq, self.q0), self.doc(self.k, d, nk, self.k0), self.doc(self.v, d, nk, self.k0)
            slopes = None if self.slopes is None else self.slopes.astype(np.float32).astype(np.float64)
            want, tol = ref_attention(q, k, v, np.float64(np.float32(self.dh ** -0.5)), self.mask,
                                      self.prefix[d] if self.prefix else 0, self.cap, slopes, self.dtype)
            close(got[self.q0[d]:self.q0[d] + nq], want, tol, f"document {d}")


CASES = [
    # one token, one key; around a tile; a tile and a workgroup's rows exactly
    dict(ql=[1], kl=[1]), dict(ql=[31, 32, 33], kl=[31, 32, 33]), dict(ql=[63, 64, 65], kl=[63, 64, 65]),
    dict(ql=[128], kl=[128]), dict(ql=[257, 1, 130], kl=[257, 1, 130]),
    # documents without queries or keys, first, last and between
    dict(ql=[0, 40, 0, 9, 0], kl=[0, 40, 0, 9, 0]), dict(ql=[5, 70, 3], kl=[0, 0, 200], room=210),
    # masks; fewer keys than queries leaves rows without any
    dict(ql=[200, 77], kl=[200, 77], mask="causal"), dict(ql=[150, 10], kl=[40, 300], room=300, mask="causal"),
    dict(ql=[200, 77, 20], kl=[200, 77, 20], mask="prefix", prefix=[65, 0, 20]),
    dict(ql=[100, 100], kl=[30, 90], room=100, mask="prefix", prefix=[7, 1000]),
    # caps and biases, together with masks
    dict(ql=[130, 50], kl=[130, 50], cap=5.0), dict(ql=[130, 50], kl=[130, 50], bias=True),
    dict(ql=[140], kl=[140], cap=30.0, bias=True, mask="causal", std=2.0),
    # single tokens and a few over caches (keys divided among workgroups), some of them empty
    dict(ql=[1, 1, 1, 1], kl=[1, 0, 1025, 3000], room=3100, mask="causal", bias=True), dict(ql=[4, 1, 3], kl=[2000, 1, 513], room=2048),
    dict(ql=[3, 2], kl=[1500, 2000], room=2000, mask="prefix", prefix=[100, 2000], cap=20.0),
]


@pytest.mark.parametrize("heads", [(2, 2), (6, 2), (8, 1)], ids=lambda h: f"h{h[0]}k{h[1]}")
@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, dtype, dh, heads):
    if heads != (6, 2) and case % 3 != 0:
        pytest.skip("every third case for the other head layouts")
    a = Attn(dtype, heads[0], heads[1], dh, **CASES[case], seed=100 * case + dh, spare=3 if case % 2 and not CASES[case].get("room") else 0)
    a.run()
    a.check()
    spare = a.o[a.q0[-1]:]
    assert (spare == 7.0).all(), "rows behind the last document were written"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 72, 128])
def test_attention_long_rows(dtype, dh):
    """Hundreds of key tiles, a workgroup count above the card's, scores large
    enough that the running maximum moves by more than 2^64."""
    a = Attn(dtype, 2, 1, dh, [700, 1300], [700, 1300], mask="causal", std=3.0, seed=dh)
    a.run()
    a.check()


# Grids that the kernel of few rows does not take: 256-row workgroups, several key tiles seen whole by all of their
# rows (one to five: the ring's slots in every turn), tiles on the diagonal and past the end.
WIDE = [
    dict(ql=[300, 1, 513, 64, 130, 0, 70], kl=[300, 1, 513, 64, 130, 0, 70]),
    dict(ql=[300, 1, 513, 64, 130], kl=[300, 1, 513, 64, 130], mask="causal"),
    dict(ql=[320, 257, 448], kl=[320, 257, 448], mask="prefix", prefix=[64, 257, 200]),
    dict(ql=[400, 400, 400], kl=[65, 128, 390], room=400, cap=5.0),
    dict(ql=[700, 380], kl=[700, 380], mask="causal", cap=30.0, bias=True, std=2.0),
    dict(ql=[1100], kl=[1100], bias=True),
    dict(ql=[900, 200], kl=[900, 200], mask="causal", std=4.0),
]


@pytest.mark.parametrize("heads", [(24, 24), (24, 8)], ids=lambda h: f"h{h[0]}k{h[1]}")
@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("case", range(len(WIDE)))
def test_attention_many_rows(case, dh, heads):
    a = Attn("bf16", heads[0], heads[1], dh, **WIDE[case], seed=7 * case + dh)
    a.run()
    a.check()


@pytest.mark.parametrize("mask", ["full", "causal"])
@pytest.mark.parametrize("dh", [64, 72, 128])
def test_attention_many_rows_divides_long_keys(dh, mask):
    """Many rows and so many keys that ranges of them run apart, some of them without a visible key."""
    a = Attn("bf16", 24, 3, dh, [700, 5, 0], [6000, 900, 40], room=6000, mask=mask, seed=dh)
    assert a.ws is not None
    a.run()
    a.check()


@pytest.mark.parametrize("dh", [64, 72, 128])
def test_attention_many_rows_what_is_not_visible_does_not_count(dh):
    """As test_attention_what_is_not_visible_does_not_count, for the kernel of many rows: a document's padding, the
    next document's keys and the keys above the diagonal."""
    a = Attn("bf16", 24, 24, dh, [600, 333], [590, 333], room=600, mask="causal", seed=3, fused=False)
    b = Attn("bf16", 24, 24, dh, [600, 333], [590, 333], room=600, mask="causal", seed=3, fused=False)
    for t in (a.k, a.v):
        for lo, hi in ((590, 600), (933, 1200)):
            t[lo:hi:3], t[lo + 1:hi:3], t[lo + 2:hi:3] = float("nan"), float("inf"), float("-inf")
    a.run()
    b.run()
    assert torch.equal(a.o, b.o)
    a.check()
    # a visible NaN value and infinity: exactly the rows that see their key, in their column
    a.v[700, 5, 9], a.v[801, 6, 10] = float("nan"), float("inf")
    a.run()
    got, want = a.o[600:933].clone(), b.o[600:933]
    assert got[100:, 5, 9].isnan().all() and (got[201:, 6, 10] == float("inf")).all()
    got[100:, 5, 9], got[201:, 6, 10] = want[100:, 5, 9], want[201:, 6, 10]
    assert torch.equal(got, want) and torch.equal(a.o[:600], b.o[:600])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_uniform_rooms_need_no_starts(dtype):
    a = Attn(dtype, 4, 2, 64, [50, 50, 50], [33, 50, 0], room=50, mask="full")
    a.run()
    want = a.o.clone()
    a.o.fill_(7.0)
    a.run(q_start=None, k_start=None)
    assert torch.equal(a.o, want)
    a.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 72, 128])
def test_attention_head_major_and_padded_strides(dtype, dh):
    """k and v stored head by head, q rows with a gap, o as columns of a wider matrix."""
    a = Attn(dtype, 4, 2, dh, [70, 20], [70, 20], fused=False, seed=5)
    dt = DT[dtype]
    a.k, a.v = [t.permute(1, 0, 2).contiguous().permute(1, 0, 2) for t in (a.k, a.v)]
    q = torch.full((90, 4, dh + 8), float("nan"), dtype=dt, device="cuda")
    q[..., :dh] = a.q
    a.q = q[..., :dh]
    wide = torch.full((90, 6, dh), 7.0, dtype=dt, device="cuda")
    a.o = wide[:, 1:5]
    a.shape = dm.attn_shape(a.q, a.k, a.v, a.o, docs=2, max_q=70, max_k=70)
    a.ws = dm.attention_workspace(a.shape)
    a.run()
    a.check()
    assert (wide[:, 0] == 7).all() and (wide[:, 5] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("few", [False, True])
def test_attention_what_is_not_visible_does_not_count(dtype, dh, few):
    """NaN and infinities in keys and values behind a document's filled length,
    between documents and above the diagonal reach no row that cannot see
    them; those that can see them get them, in their column."""
    ql = [3, 2] if few else [150, 90]
    a = Attn(dtype, 4, 2, dh, ql, [150, 90], room=200, mask="causal", seed=9, fused=False)
    bad = [float("nan"), float("inf"), float("-inf")]
    b = Attn(dtype, 4, 2, dh, ql, [150, 90], room=200, mask="causal", seed=9, fused=False)  # the same, left as it is
    for t in (a.k, a.v):
        for d, n in enumerate(a.kl):
            for x in range(3):
                t[d * 200 + n + x:(d + 1) * 200:3] = bad[x]
    a.run()
    a.check()
    # ... and inside the first document, at its last keys: keys 148 (V column 5 = inf, head 0), 149 (NaN)
    a.v[148, 0, 5] = float("inf")
    a.v[149, 0, 6] = float("nan")
    a.v[149, 1, 7] = float("-inf")
    a.k[149, 1, 3] = float("nan")
    a.run()
    got = np64(a.o)
    lim = row_limits(ql[0], 150, "causal", 0)
    want, tol = ref_attention(np64(a.q[:ql[0]]), np64(b.k[:150]), np64(b.v[:150]), np.float64(np.float32(dh ** -0.5)), "causal",
                              dtype=dtype)
    for i in range(ql[0]):
        for h in range(4):
            w, t, g = want[i, h].copy(), tol[i, h], got[i, h]
            if h < 2:
                if lim[i] > 148:
                    assert g[5] == np.inf
                    w[5] = g[5] = 0
                if lim[i] > 149:
                    assert np.isnan(g[6])
                    w[6] = g[6] = 0
            elif lim[i] > 149:
                assert np.isnan(g).all()
                continue
            close(g, w, t, (i, h))


def test_attention_offsets_beyond_32_bits():
    """A cache whose last rows lie more than 2^32 bytes behind its first."""
    H, dh, n, row = 2, 64, 700, 1 << 22
    k, v = (torch.empty(n * row, dtype=torch.bfloat16, device="cuda").as_strided((n, H, dh), (row, dh, 1)) for _ in range(2))
    a = Attn("bf16", H, H, dh, [3], [n], fused=False, seed=3)
    k.copy_(a.k)
    v.copy_(a.v)
    a.k, a.v = k, v
    a.shape = dm.attn_shape(a.q, a.k, a.v, a.o, docs=1, max_q=3, max_k=n)
    a.ws = dm.attention_workspace(a.shape)
    a.run()
    a.check()
    f = Attn("f32", H, H, dh, [40], [n], fused=False, seed=3)
    del a, k, v
    k, v = (torch.empty(n * (row // 2), dtype=torch.float32, device="cuda").as_strided((n, H, dh), (row // 2, dh, 1)) for _ in range(2))
    k.copy_(f.k)
    v.copy_(f.v)
    f.k, f.v = k, v
    f.shape = dm.attn_shape(f.q, f.k, f.v, f.o, docs=1, max_q=40, max_k=n)
    f.ws = dm.attention_workspace(f.shape)
    f.run()
    f.check()


@pytest.mark.parametrize("dtype,H,nq", [("bf16", 16, 1100), ("bf16", 2, 3), ("f32", 2, 3)])
def test_attention_bias_at_places_beyond_24_bits(dtype, H, nq):
    """The distance of a near key is exact, however far down the cache the query stands (slopes that leave
    keys more than 200 places away nothing)."""
    dh, n, near = 64, 2 ** 24 + 1001, nq + 300
    k, v = (torch.zeros(n, 1, dh, dtype=DT[dtype], device="cuda") for _ in range(2))
    k[-near:], v[-near:] = rand(1, near, 1, dh, dtype=DT[dtype]), rand(2, near, 1, dh, dtype=DT[dtype])
    q = rand(3, nq, H, dh, dtype=DT[dtype])
    o = torch.empty_like(q)
    slopes = np.linspace(1.0, 2.0, H)
    s = dm.attn_shape(q, k, v, o, docs=1, max_q=nq, max_k=n, mask="causal")
    dm.attention(s, q, k, v, o, dm.attention_workspace(s), slopes=torch.tensor(slopes, dtype=torch.float32, device="cuda"))
    want, tol = ref_attention(np64(q), np64(k[-near:]), np64(v[-near:]), np.float64(np.float32(dh ** -0.5)), "causal",
                              slopes=slopes.astype(np.float32).astype(np.float64), dtype=dtype)
    close(np64(o), want, tol, "near keys")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_cuts_what_is_out_of_range(dtype):
    """Index arrays that leave the tensors are cut to them (the library cannot
    see them before the kernel does); documents longer than max_q and max_k to those."""
    a = Attn(dtype, 2, 2, 64, [40, 30], [40, 30], seed=4)
    a.run(q_start=i32([0, 40, 4000]), k_start=i32([0, 40, 1 << 30]))
    a.check()
    a.o.fill_(7.0)
    a.run(q_start=i32([-5, 40, 70]), k_start=i32([-9, 40, 70]))
    a.check()
    a.o.fill_(7.0)
    a.run(q_start=i32([50, 40, 30]))  # no document has a row
    assert (a.o == 7.0).all()
    a.run(q_start=i32([50, -2 ** 31, 2 ** 31 - 1]), k_start=i32([50, -2 ** 31, 2 ** 31 - 1]))
    # the first has no row; the second is all rows, cut to max_q and max_k
    want, tol = ref_attention(np64(a.q[:40]), np64(a.k[:40]), np64(a.v[:40]), np.float64(np.float32(64 ** -0.5)), dtype=dtype)
    close(np64(a.o)[:40], want, tol, "all rows")
    assert (a.o[40:] == 7.0).all()
    b = Attn(dtype, 2, 2, 64, [40], [40], seed=4)
    b.shape = dm.attn_shape(b.q, b.k, b.v, b.o, docs=1, max_q=16, max_k=20)
    b.ws = dm.attention_workspace(b.shape)
    b.run()
    want, tol = ref_attention(np64(b.q[:16]), np64(b.k[:20]), np64(b.v[:20]), np.float64(np.float32(64 ** -0.5)), dtype=dtype)
    close(np64(b.o)[:16], want, tol, "cut")
    assert (b.o[16:] == 7.0).all()


# ---------------------------------------------------------------- products in 8 bits
def quantized(x, rows):
    codes = torch.empty(x.shape, dtype=DT["e4m3"], device="cuda")
    scale = torch.empty(-(-x.shape[0] // rows), -(-x.shape[1] // 128), device="cuda")
    dm.quantize_fp8(x, codes, scale, block_rows=rows)
    return codes, scale


def plain_quantize(x, rows):
    """fp32 on the CPU, the operator's own arithmetic."""
    x = x.float().cpu()
    R, C = x.shape
    nr, nc = -(-R // rows), -(-C // 128)
    full = torch.zeros(nr * rows, nc * 128)
    full[:R, :C] = x
    amax = full.abs().view(nr, rows, nc, 128).nan_to_num(nan=0.0, posinf=float("inf")).amax(dim=(1, 3))
    scale = (amax * torch.tensor(1.0 / 448, dtype=torch.float32)).clamp_min(2.0 ** -126)
    inv = (1.0 / scale).repeat_interleave(rows, 0)[:R].repeat_interleave(128, 1)[:, :C]
    return (x * inv).clamp(-448, 448).to(torch.float8_e4m3fn), scale


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(1, 8), (1, 128), (3, 136), (17, 1152), (128, 128), (129, 264), (300, 4608), (1000, 64)])
def test_quantize(R, C, dtype, rows):
    x = rand(R * C, R, C + 8, std=3.0, dtype=DT[dtype])[:, :C]  # rows with a gap
    if R > 1:
        x[R // 2] = 0.0       # a block of zeros among others (rows = 1)
        x[0, 0], x[0, C - 1] = 1e-38, -2.0 ** -126
        x[1] *= 1e-30
    codes, scale = quantized(x, rows)
    want, wscale = plain_quantize(x, rows)
    assert torch.equal(scale.cpu(), wscale)
    assert torch.equal(codes.cpu().view(torch.uint8), want.view(torch.uint8))


def test_quantize_what_is_not_finite():
    x = rand(1, 4, 256)
    x[0, 3], x[1, 130], x[2, 255] = float("nan"), float("inf"), float("-inf")
    x[3, :128] = float("nan")
    codes, scale = quantized(x, 1)
    c, s, w = codes.float().cpu(), scale.cpu(), plain_quantize(x, 1)
    assert torch.equal(s, w[1])
    assert torch.equal(c.isnan(), w[0].float().isnan()) and c[0, 3].isnan() and c[1, 130].isnan() and s[1, 1] == float("inf")
    assert torch.equal(c.nan_to_num(), w[0].float().nan_to_num())


LINEAR = [(1, 16, 1), (1, 1152, 6912), (3, 144, 40), (8, 1152, 136), (16, 4608, 1152), (17, 400, 24), (33, 128, 129), (65, 2048, 256),
          (130, 1152, 384), (257, 272, 1000), (300, 64, 520), (128, 128, 128), (640, 1536, 768)]


# ... and what the large tiles take: whole, and with the last round's tiles divided over k; a last block of 16
LARGE = [(3990, 784, 4090, "gelu", "bf16"), (3990, 912, 4088, "none", "e4m3"), (4990, 2704, 4088, "gelu", "e4m3"),
         (4990, 2704, 4090, "none", "bf16"), (1900, 272, 4400, "gelu", "e4m3"), (1900, 272, 4400, "none", "bf16"), (1901, 128, 4501, "gelu", "bf16"),
         (4500, 1040, 4400, "none", "e4m3"), (4500, 1040, 4400, "gelu", "bf16"), (1900, 272, 4400, "none", "f32"),
         (1030, 4608, 1160, "gelu", "f32"), (1030, 4608, 1160, "gelu", "e4m3"),
         (1343, 2320, 2970, "gelu", "bf16"), (1343, 2320, 2968, "none", "e4m3"),
         (1547, 3184, 2473, "gelu", "bf16"), (1547, 3184, 2472, "gelu", "e4m3"),
         (1343, 2320, 2969, "gelu", "e4m3"), (1547, 3184, 2474, "none", "e4m3"), (1900, 272, 4399, "gelu", "e4m3"), (1030, 4608, 1157, "gelu", "e4m3")]


@pytest.mark.parametrize("M,K,N,act,dtype", [(*s, a, d) for s in LINEAR for a in ("none", "gelu") for d in ("bf16", "f32", "e4m3")] + LARGE)
def test_linear(M, K, N, act, dtype):
    a, sa = quantized(rand(M + K, M, K) * torch.exp(rand(7, M, 1)), 1)
    w, sw = quantized(rand(N, N, K, std=0.05), 128)
    bias = rand(3, N, dtype=torch.float32 if dtype == "f32" else torch.bfloat16) if (M + N) % 2 or act == "gelu" else None
    shape = dm.linear_shape(M, K, N, act=act, dtype=dtype)
    ws = dm.linear_fp8_workspace(shape)
    if ws is not None:
        ws.fill_(0xFF)
    guard = torch.full((M + 2, N), 9.0, device="cuda").to(DT[dtype])
    out = guard[1:M + 1] if (N * guard.element_size()) % 16 == 0 else torch.empty(M, N, dtype=DT[dtype], device="cuda")
    osc = torch.empty(M, -(-N // 128), device="cuda") if dtype == "e4m3" else None
    dm.linear_fp8(shape, a, sa, w, sw, out, ws, bias=bias, out_scale=osc)
    y, tol = ref_linear(np64(a), np64(sa), np64(w), np64(sw), None if bias is None else np64(bias), act)
    got = np64(out)
    if dtype == "e4m3":
        from operator_refs import spread
        amax = np.stack([np.abs(y[:, c:c + 128]).max(1) for c in range(0, N, 128)], 1)
        atol = np.stack([tol[:, c:c + 128].max(1) for c in range(0, N, 128)], 1)
        s = np64(osc)
        close(s, np.maximum(amax / 448, 2.0 ** -126), atol / 448 + amax / 448 * 2.0 ** -22 + 1e-38, "scale")
        s = spread(s, 1, M, N)
        close(got * s, y, tol + e4m3_tol(np.abs(y) + tol, s), "codes")
    else:
        close(got, y, tol + U[dtype] * (np.abs(y) + tol), "y")
    assert (guard[0].float() == 9).all() and (guard[-1].float() == 9).all()


def test_linear_nan_stays_in_its_row_and_column():
    M, K, N = 40, 256, 200
    a, sa = quantized(rand(1, M, K), 1)
    w, sw = quantized(rand(2, N, K), 128)
    a[5, 17], w[150, 200] = float("nan"), float("nan")
    out = torch.empty(M, N, device="cuda")
    shape = dm.linear_shape(M, K, N, dtype="f32")
    dm.linear_fp8(shape, a, sa, w, sw, out, dm.linear_fp8_workspace(shape))
    want = torch.zeros(M, N, dtype=torch.bool)
    want[5], want[:, 150] = True, True
    assert torch.equal(out.isnan().cpu(), want)


# ---------------------------------------------------------------- norms
@pytest.mark.parametrize("R,D", [(1, 8), (5, 64), (77, 1152), (3, 1160), (130, 2048), (9, 2056), (33, 4096), (4, 4104), (2, 8192), (7, 8), (2050, 8), (2051, 1160), (2048, 2056),
                                 (2049, 4096)])
@pytest.mark.parametrize("post,pre,ydt,hdt", [("none", "layer", "f32", "bf16"), ("layer", "layer", "bf16", "f32"), ("rms", "rms", "bf16", "e4m3"),
                                              ("rms", "layer", "f32", "e4m3")])
def test_norm_residual(R, D, post, pre, ydt, hdt):
    B = min(R, 3)
    x, y = rand(R, R, D), rand(R + 1, R, D, std=3.0, dtype=DT[ydt])
    x += 2.0  # a mean that the variance must not lose digits to
    wp = 1 + rand(2, D, std=0.2) if post != "none" and D % 16 else None
    w = 1 + rand(3, D, std=0.2) if R % 2 else None
    mod = rand(4, B, 3 * D + 4, std=0.7)
    gate, shift, scale = mod[:, :D], mod[:, D:2 * D], mod[:, 2 * D:3 * D]
    rb = [r * 7 % B for r in range(R)]
    rs = 0.5 if R % 3 else 1.0
    s = dm.norm_shape(R, D, batch=B, post=post, pre=pre, y_dtype=ydt, h_dtype=hdt, eps=1e-5, res_scale=rs, mod_stride=mod.stride(0))
    xo, h = torch.empty_like(x), torch.empty(R, D, dtype=DT[hdt], device="cuda")
    hs = torch.empty(R, -(-D // 128), device="cuda") if hdt == "e4m3" else None
    dm.norm_residual(s, x, xo, h, y=y, w_post=wp, gate=gate, w_pre=w, shift=shift, scale=scale, row_batch=i32(rb), h_scale=hs)
    wx, tx, wh, th = ref_norm(np64(x), np64(y), None if wp is None else np64(wp), np64(gate)[rb], None if w is None else np64(w),
                              np64(shift)[rb], np64(scale)[rb], post, pre, rs, np.float64(np.float32(1e-5)))
    close(np64(xo), wx, tx, "x_out")
    if hdt == "e4m3":
        from operator_refs import spread
        sc = np64(hs)
        amax = np.stack([np.abs(wh[:, c:c + 128]).max(1) for c in range(0, D, 128)], 1)
        at = np.stack([th[:, c:c + 128].max(1) for c in range(0, D, 128)], 1)
        close(sc, amax / 448, at / 448 + amax / 448 * 2.0 ** -22, "h_scale")
        sc = spread(sc, 1, R, D)
        close(np64(h) * sc, wh, th + e4m3_tol(np.abs(wh) + th, sc), "h")
    else:
        close(np64(h), wh, th + U[hdt] * (np.abs(wh) + th), "h")
    # in place, and without what is optional
    x2 = x.clone()
    dm.norm_residual(s, x2, x2, h, y=y, w_post=wp, gate=gate, w_pre=w, shift=shift, scale=scale, row_batch=i32(rb), h_scale=hs)
    assert torch.equal(x2, xo)


def test_norm_residual_parts():
    R, D = 10, 384
    x, y = rand(1, R, D), rand(2, R, D)
    h, xo = torch.empty(R, D, device="cuda"), torch.empty(R, D, device="cuda")
    s = dm.norm_shape(R, D, pre="rms", h_dtype="f32")
    dm.norm_residual(s, x, None, h)  # a first norm alone
    _, _, wh, th = ref_norm(np64(x), None, None, None, None, None, None, "none", "rms", 1.0, 1e-6)
    close(np64(h), wh, th, "h alone")
    s = dm.norm_shape(R, D, batch=4, post="layer", res_scale=2.0)
    gate = rand(3, 4, D)
    dm.norm_residual(s, x, xo, None, y=y, gate=gate)  # the last residual: no norm follows; samples of 3, 3, 3 and 1 rows
    wx, tx, _, _ = ref_norm(np64(x), np64(y), None, np64(gate)[np.arange(R) // 3], None, None, None, "layer", "layer", 2.0, 1e-6)
    close(np64(xo), wx, tx, "x alone")
    s = dm.norm_shape(R, D, res_scale=0.25)
    dm.norm_residual(s, x, xo, None)
    assert torch.equal(xo, 0.25 * x)


# ---------------------------------------------------------------- how they are called
def some_calls():
    """(name, call, outputs) of every operator at a size that uses its workspace or not."""
    a = Attn("bf16", 4, 2, 64, [1, 2], [900, 1300], room=1400, mask="causal", seed=1)
    b = Attn("bf16", 4, 4, 128, [300, 40], [300, 40], cap=10.0, seed=2)
    c = Attn("f32", 4, 2, 72, [5, 60], [700, 60], room=800, seed=3)
    xa, sa = quantized(rand(1, 24, 2048), 1)
    w, sw = quantized(rand(2, 512, 2048), 128)
    ls = dm.linear_shape(24, 2048, 512, act="gelu", dtype="e4m3")
    lo, los, lws = torch.empty(24, 512, dtype=DT["e4m3"], device="cuda"), torch.empty(24, 4, device="cuda"), dm.linear_fp8_workspace(ls)
    x, y = rand(3, 50, 768), rand(4, 50, 768)
    xo, h, hs = torch.empty_like(x), torch.empty(50, 768, dtype=DT["e4m3"], device="cuda"), torch.empty(50, 6, device="cuda")
    ns = dm.norm_shape(50, 768, post="rms", pre="rms", h_dtype="e4m3")
    q, qs = torch.empty(50, 768, dtype=DT["e4m3"], device="cuda"), torch.empty(50, 6, device="cuda")
    return [("tokens", lambda st: a.run(stream=st), [a.o]), ("documents", lambda st: b.run(stream=st), [b.o]),
            ("fp32", lambda st: c.run(stream=st), [c.o]),
            ("linear", lambda st: dm.linear_fp8(ls, xa, sa, w, sw, lo, lws, out_scale=los, stream=st), [lo, los]),
            ("norm", lambda st: dm.norm_residual(ns, x, xo, h, y=y, h_scale=hs, stream=st), [xo, h, hs]),
            ("quantize", lambda st: dm.quantize_fp8(x, q, qs, stream=st), [q, qs])]


def snapshot(calls):
    torch.cuda.synchronize()
    return [[o.clone().view(torch.uint8) for o in outs] for _, _, outs in calls]


def blank(calls):
    for _, _, outs in calls:
        for o in outs:
            o.view(torch.uint8).fill_(0x55)


def test_streams_repeats_and_graphs():
    """The same bits from the current stream, another stream, repeated calls and
    every replay of a captured graph, with eager calls in between."""
    calls = some_calls()
    for _, f, _ in calls:
        f(None)
    want = snapshot(calls)

    def same(what):
        for (name, _, _), w, g in zip(calls, want, snapshot(calls)):
            assert all(torch.equal(x, y) for x, y in zip(w, g)), (what, name)

    blank(calls)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _, f, _ in calls:
        f(side)
    same("side stream")
    blank(calls)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _, f, _ in calls:
            f(None)
    for replay in range(4):
        blank(calls)
        torch.cuda.synchronize()
        graph.replay()
        same(f"replay {replay}")
        blank(calls)
        for _, f, _ in calls:
            f(None)
        same(f"eager after replay {replay}")


def test_two_calls_at_once():
    """Two streams, each with workspaces of its own."""
    one, two = some_calls(), some_calls()
    for _, f, _ in one:
        f(None)
    want = snapshot(one)
    blank(one)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        for (_, f, _), (_, g, _) in zip(one, two):
            f(s1)
            g(s2)
    for calls in (one, two):
        for (name, _, _), w, g in zip(calls, want, snapshot(calls)):
            assert all(torch.equal(x, y) for x, y in zip(w, g)), name
