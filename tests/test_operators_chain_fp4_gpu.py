"""The 4-bit operators and the norms and rotation of queries and keys as a block uses
them, each step against its definition in 64 bits on what the steps before it left."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from operator_refs import attention as ref_attention
from test_operators_fp4_gpu import Linear, buffers, nibbles, quantized, ref_codes, ref_scales, rows_of
from test_operators_gpu import close, i32, np64, rand
from test_operators_qk_gpu import U24, reference

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def quantize(x):
    codes, scale = quantized(x)
    s, _ = rows_of(scale, x.shape[1])
    assert np.array_equal(s, ref_scales(np64(x))) and np.array_equal(nibbles(codes), ref_codes(np64(x), s))
    return codes, scale


def linear(a, w, bias, act="none", dtype="bf16"):
    c = Linear.of(*a, *w, bias, act=act, dtype=dtype)
    out = c.run()
    c.check(out)
    return out


def test_joint_block_in_4_bits():
    """Image and text rows with weights of their own, normed, turned (image rows by row and column) and put into one
    joint sequence of documents [image; text]; attention; projections and the image rows' MLP."""
    H, dh, F = 4, 72, 576
    D, img, txt = H * dh, [(7, 10), (11, 12)], [9, 20]
    ni, nt = [a * b for a, b in img], txt
    T = {"img": sum(ni), "txt": sum(nt)}
    joint = np.concatenate([[0], np.cumsum([a + b for a, b in zip(ni, nt)])])
    dst = {"img": np.concatenate([joint[d] + np.arange(n) for d, n in enumerate(ni)]),
           "txt": np.concatenate([joint[d] + ni[d] + np.arange(n) for d, n in enumerate(nt)])}
    pos = {"img": np.concatenate([np.stack(np.divmod(np.arange(a * b), b), 1) for a, b in img]), "txt": np.zeros((T["txt"], 2))}
    freqs, pairs = dm.rope_freqs((18, 18)), (18, 18)
    all_q, all_k, all_v, o = (torch.full((joint[-1], H, dh), float("nan"), dtype=BF, device="cuda") for _ in range(4))
    x, seed = {}, iter(range(1, 100))
    for part in ("img", "txt"):
        n = T[part]
        x[part] = rand(next(seed), n, D)
        h = torch.empty(n, D, dtype=BF, device="cuda")
        dm.norm_residual(dm.norm_shape(n, D), x[part], None, h)
        w, bias = quantize(rand(next(seed), 3 * D, D, std=0.06)), rand(next(seed), 3 * D, std=0.1, dtype=BF)
        qkv = linear(quantize(h), w, bias).view(n, 3 * H, dh)
        q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
        wq, wk = 1 + rand(next(seed), dh, std=0.1), 1 + rand(next(seed), dh, std=0.1)
        s = dm.qk_shape(q, k, all_q, all_k, v=v, v_out=all_v, norm="rms", pairs=pairs)
        dm.qk_norm_rope(s, q, k, all_q, all_k, v=v, v_out=all_v, w_q=wq, w_k=wk, pos=i32(pos[part].astype(int).tolist()),
                        freqs=freqs, q_dst=i32(dst[part].tolist()), k_dst=i32(dst[part].tolist()))
        for got, src, weight in ((all_q, q, wq), (all_k, k, wk)):
            y, tol = reference(np64(src), np64(weight), "rms", pairs, "interleaved", pos[part], freqs.cpu().numpy(), "bf16")
            close(np64(got)[dst[part]], y, tol, part)
        assert torch.equal(all_v[torch.from_numpy(dst[part]).cuda()], v)
    for t in (all_q, all_k, all_v):
        assert torch.isfinite(t).all()  # every row of the joint sequence was written
    longest = int(np.diff(joint).max())
    s = dm.attn_shape(all_q, all_k, all_v, o, docs=2, max_q=longest, max_k=longest)
    dm.attention(s, all_q, all_k, all_v, o, dm.attention_workspace(s), q_start=i32(joint.tolist()), k_start=i32(joint.tolist()))
    for d in range(2):
        at = slice(joint[d], joint[d + 1])
        y, tol = ref_attention(np64(all_q)[at], np64(all_k)[at], np64(all_v)[at], np.float64(np.float32(dh ** -0.5)))
        close(np64(o)[at], y, tol, "attention")
    n = T["img"]
    rows = o.view(-1, D)[torch.from_numpy(dst["img"]).cuda()]
    y = linear(quantize(rows), quantize(rand(next(seed), D, D, std=0.06)), rand(next(seed), D, std=0.1, dtype=BF))
    xo, h = torch.empty_like(x["img"]), torch.empty(n, D, dtype=BF, device="cuda")
    dm.norm_residual(dm.norm_shape(n, D, y_dtype="bf16"), x["img"], xo, h, y=y)
    g = linear(quantize(h), quantize(rand(next(seed), F, D, std=0.06)), rand(next(seed), F, std=0.1, dtype=BF), act="gelu", dtype="fp4")
    y = linear(g, quantize(rand(next(seed), D, F, std=0.06)), None)
    out = torch.empty_like(xo)
    dm.norm_residual(dm.norm_shape(n, D, y_dtype="bf16"), xo, out, None, y=y)
    close(np64(out), np64(xo) + np64(y), 2 * U24 * (np.abs(np64(xo)) + np.abs(np64(y))), "residual")


def test_tokens_into_caches_from_a_replayed_graph():
    """One token for each of three requests a step: its keys and values go into the caches' rooms at the places that
    the device's arrays name, and attention reads the filled part; the step is captured once and replayed."""
    B, H, Hk, dh, room = 3, 6, 2, 128, 40
    fill = np.array([0, 7, 38])
    kc, vc = (torch.full((B * room, Hk, dh), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    past = rand(1, B * room, 2 * Hk, dh, dtype=BF)
    for b in range(B):
        at = slice(b * room, b * room + fill[b])
        kc[at], vc[at] = past[at, :Hk], past[at, Hk:]
    qkv, q, o = (torch.empty(B, n, dh, dtype=BF, device="cuda") for n in (H + 2 * Hk, H, H))
    pos, k_dst, k_len = (torch.zeros(*s, dtype=torch.int32, device="cuda") for s in ((B, 1), (B,), (B,)))
    wq, wk, freqs = 1 + rand(2, dh, std=0.1), 1 + rand(3, dh, std=0.1), dm.rope_freqs((64,))
    qs, ks, vs = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    s = dm.qk_shape(qs, ks, q, kc, v=vs, v_out=vc, pairs=(64,), pairing="halves")
    a = dm.attn_shape(q, kc, vc, o, docs=B, max_q=1, max_k=room, mask="causal")
    ws = dm.attention_workspace(a)

    def step():
        dm.qk_norm_rope(s, qs, ks, q, kc, v=vs, v_out=vc, w_q=wq, w_k=wk, pos=pos, freqs=freqs, k_dst=k_dst)
        dm.attention(a, q, kc, vc, o, ws, k_len=k_len)

    def feed(n, rows):
        qkv.copy_(rand(10 + n, B, H + 2 * Hk, dh, dtype=BF))
        pos.copy_(i32([[int(f) + n] for f in fill]))
        k_dst.copy_(i32([b * room + f + n if f + n < room else -1 for b, f in enumerate(fill.tolist())]))
        k_len.copy_(i32([min(f + n + 1, room) for f in fill.tolist()]))

    feed(0, None)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(4):  # the third request's room is full after two
        feed(n, None)
        before = kc.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(o).all()
        y, tol = reference(np64(ks), np64(wk), "rms", (64,), "halves", pos.cpu().numpy(), freqs.cpu().numpy(), "bf16")
        q64, _ = reference(np64(qs), np64(wq), "rms", (64,), "halves", pos.cpu().numpy(), freqs.cpu().numpy(), "bf16")
        for b in range(B):
            place, length = int(k_dst[b]), int(k_len[b])
            if place >= 0:
                close(np64(kc)[place], y[b], tol[b], "key")
                assert torch.equal(vc[place], vs[b])
                before[place] = kc[place]
            at = slice(b * room, b * room + length)
            want, tl = ref_attention(np64(q)[b:b + 1], np64(kc)[at], np64(vc)[at], np.float64(np.float32(dh ** -0.5)), "causal")
            close(np64(o)[b:b + 1], want, tl, "token")
        assert torch.equal(before.view(torch.int16), kc.view(torch.int16))  # nothing else was written


def test_two_calls_at_once():
    """Two streams, each with operands and workspaces of its own."""
    sets = []
    for n in range(2):
        c = Linear(300, 18432, 1152, dtype="fp4", seed=n)  # k divided: uses a workspace
        x = rand(50 + n, 300, 512, dtype=BF)
        q, k = rand(60 + n, 300, 6, 64, dtype=BF), rand(70 + n, 300, 2, 64, dtype=BF)
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        s = dm.qk_shape(q, k, qo, ko, pairs=(32,))
        pos, fr = i32([[i] for i in range(300)]), dm.rope_freqs((32,))
        assert c.ws is not None
        sets.append((c, x, buffers(300, 512), (s, q, k, qo, ko, pos, fr)))

    def go(z, stream):
        c, x, (codes, scale), (s, q, k, qo, ko, pos, fr) = z
        out = c.run(stream=stream)
        dm.quantize_fp4(x, codes, scale, stream=stream)
        dm.qk_norm_rope(s, q, k, qo, ko, pos=pos, freqs=fr, stream=stream)
        return [*out, codes, scale, qo, ko]

    want = [[t.clone() for t in go(z, None)] for z in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for z, st in zip(sets, streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got.append(go(z, st))
        torch.cuda.synchronize()
        for w, g in zip(want, got):
            assert all(torch.equal(a, b) for a, b in zip(w, g))


def test_refusals_on_the_device():
    q, k = rand(1, 4, 2, 64, dtype=BF), rand(2, 4, 1, 64, dtype=BF)
    s = dm.qk_shape(q, k, q, k, pairs=(32,))
    pos, fr = i32([[0]] * 4), dm.rope_freqs((32,))
    bad = [dict(pos=pos[:3]), dict(pos=pos.long()), dict(freqs=fr.float()), dict(freqs=fr[:31]), dict(w_q=torch.ones(63, device="cuda")),
           dict(w_q=torch.ones(64, dtype=BF, device="cuda")), dict(k_dst=i32([0, 1, 2])), dict(pos=pos.cpu()), dict(v=k)]
    for kw in bad:
        with pytest.raises((ValueError, dm.DitError)):
            dm.qk_norm_rope(s, q, k, q, k, **{**dict(pos=pos, freqs=fr), **kw})
    for args in ((q[:3], k, q, k), (q.float(), k, q, k), (q, k, q[:, :1], k), (q.cpu(), k, q, k), (q, None, q, None), (q, k, None, k)):
        with pytest.raises(ValueError):
            dm.qk_norm_rope(s, *args, pos=pos, freqs=fr)
    with pytest.raises(dm.DitError):  # moved in place
        dm.qk_norm_rope(s, q, k, q, k, pos=pos, freqs=fr, k_dst=i32([0, 1, 2, 3]))
    x = rand(3, 4, 64)
    codes, scale = buffers(4, 64)
    for args in ((x[:, ::2], codes, scale), (x, codes[:3], scale), (x, codes, scale[:, :3]), (x, codes.view(torch.int8), scale), (x.half(), codes, scale),
                 (x[0], codes, scale), (x.cpu(), codes, scale)):
        with pytest.raises(ValueError):
            dm.quantize_fp4(*args)
        with pytest.raises(ValueError):
            dm.dequantize_fp4(args[1], args[2], args[0])
    with pytest.raises(dm.DitError):
        dm.quantize_fp4(x[:, :40].contiguous(), torch.empty(4, 20, dtype=torch.uint8, device="cuda"), scale)
    c = Linear(300, 18432, 1152)
    out = torch.empty(300, 1152, dtype=BF, device="cuda")
    assert c.ws is not None
    with pytest.raises(dm.DitError):
        dm.linear_fp4(c.shape, c.a, c.a_scale, c.w, c.w_scale, out, None)
    with pytest.raises(dm.DitError):
        dm.linear_fp4(c.shape, c.a, c.a_scale, c.w, c.w_scale, out, c.ws[:-256])
    for kw in (dict(bias=torch.ones(1152, device="cuda")), dict(bias=torch.ones(1151, dtype=BF, device="cuda"))):
        with pytest.raises(ValueError):
            dm.linear_fp4(c.shape, c.a, c.a_scale, c.w, c.w_scale, out, c.ws, **kw)
    for args in ((c.a[:299], c.a_scale), (c.a, c.a_scale[1:]), (c.a.view(torch.int8), c.a_scale)):
        with pytest.raises(ValueError):
            dm.linear_fp4(c.shape, *args, c.w, c.w_scale, out, c.ws)


def test_offsets_past_32_bits():
    """Rows of a cache, of a strided input and of a product's output that lie more than 2^31 elements on."""
    n = (1 << 31) // 64 + 100
    cache = torch.empty(n, 1, 64, dtype=BF, device="cuda")
    k = rand(1, 5, 1, 64, dtype=BF)
    at = [n - 1, 0, n - 40, n // 2, n - 2]
    s = dm.qk_shape(None, k, None, cache, v=None, pairs=(32,))
    pos, fr = i32([[i] for i in range(5)]), dm.rope_freqs((32,))
    dm.qk_norm_rope(s, None, k, None, cache, pos=pos, freqs=fr, k_dst=i32(at))
    y, tol = reference(np64(k), 1.0, "rms", (32,), "interleaved", pos.cpu().numpy(), fr.cpu().numpy(), "bf16")
    close(np64(cache[at]), y, tol, "cache")
    del cache
    wide = torch.empty((1 << 31) + 4096, dtype=BF, device="cuda")
    x = wide.as_strided((3, 4096), (1 << 30, 1))
    for i in range(3):
        x[i] = rand(2 + i, 4096, dtype=BF)
    codes, scale = quantize(x)
    back = torch.empty_like(wide).as_strided((3, 4096), (1 << 30, 1))
    dm.dequantize_fp4(codes, scale, back)
    want = torch.empty(3, 4096, dtype=BF, device="cuda")
    dm.dequantize_fp4(codes, scale, want)
    assert torch.equal(back, want)
    del wide, back, x
    M, N = 70000, 32768  # 32 products of 4-bit codes: exact in fp32, and rounded once
    c = Linear.of(*quantized(rand(5, M, 32)), *quantized(rand(6, N, 32)), None)
    out = c.run()
    for r in (slice(0, 50), slice(65530, 65580), slice(M - 50, M)):
        y = c.av[r] @ c.wv.T
        close(np64(out[r]), y, 2.0 ** -8 * np.abs(y), "product")
