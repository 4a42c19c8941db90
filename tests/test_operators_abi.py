"""CPU tests of the stand-alone operators' refusals: every call below is refused
before any HIP call, so its pointers are never dereferenced."""
import ctypes

import pytest
import torch

BAD, UNSUP, WS = -1, -2, -3
P = 4096  # an aligned address


@pytest.fixture(scope="module")
def dm():
    import os

    import paper_2605_25550_amd as dm
    if not os.path.exists(dm.LIB_PATH):
        from paper_2605_25550_amd.build import build
        build()
    dm.lib()
    return dm


def attn(dm, **kw):
    d = dict(docs=2, heads=8, kv_heads=2, head_dim=64, q_rows=100, k_rows=200, max_q=50, max_k=100, dtype=1, mask=0,
             scale=0.125, cap=0.0, q_row=512, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, o_row=512, o_head=64)
    d.update(kw)
    return dm.AttnShape(*[d[n] for n, _ in dm.AttnShape._fields_])


def call_attn(dm, s, q=P, k=P, v=P, o=P, q_start=P, k_start=P, k_len=None, prefix=None, slopes=None, ws=P, n=1 << 40):
    return dm.lib().dit_attention(ctypes.byref(s) if s is not None else None, q, k, v, o, q_start, k_start, k_len, prefix, slopes,
                                  ws, n, None)


@pytest.mark.parametrize("kw,want", [
    (dict(docs=0), BAD), (dict(docs=70000), UNSUP), (dict(heads=7), BAD), (dict(kv_heads=0), BAD), (dict(head_dim=80), UNSUP),
    (dict(q_rows=-1), BAD), (dict(k_rows=-1), BAD), (dict(max_q=-1), BAD), (dict(max_k=-1), BAD), (dict(dtype=2), BAD),
    (dict(dtype=7), BAD), (dict(mask=3), BAD), (dict(mask=-1), BAD), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(cap=-1.0), BAD), (dict(cap=float("nan")), BAD),
    (dict(q_row=516), BAD), (dict(k_head=60), BAD), (dict(v_row=-128), BAD), (dict(o_row=32), BAD), (dict(k_head=56), BAD),
    (dict(k_row=1 << 23), UNSUP), (dict(max_q=1 << 28, q_rows=1 << 29), UNSUP), (dict(k_rows=1 << 30), UNSUP),
    (dict(scale=2e38), UNSUP), (dict(cap=1e-30), UNSUP), (dict(cap=1e4), UNSUP),
    (dict(dtype=0, max_q=1 << 24, q_rows=1 << 24), UNSUP),
])
def test_attention_shapes(dm, kw, want):
    s = attn(dm, **kw)
    assert call_attn(dm, s) == want and dm.last_error()
    assert dm.lib().dit_attention_workspace_bytes(s) == ctypes.c_size_t(-1).value
    with pytest.raises(dm.DitError):
        dm.attention_workspace(s, device="cpu")


def test_attention_pointers_and_workspace(dm):
    s = attn(dm)
    assert call_attn(dm, None) == BAD
    for n in ("q", "k", "v", "o"):
        assert call_attn(dm, s, **{n: None}) == BAD and n in dm.last_error()
        assert call_attn(dm, s, **{n: P + 8}) == BAD
    for n in ("q_start", "k_start", "k_len", "slopes"):
        assert call_attn(dm, s, **{n: P + 2}) == BAD and n in dm.last_error()
    assert call_attn(dm, s, prefix=P) == BAD and "prefix" in dm.last_error()
    assert call_attn(dm, attn(dm, mask=2)) == BAD and "prefix" in dm.last_error()
    # rooms that do not fit the tensors
    assert call_attn(dm, attn(dm, max_q=51), q_start=None) == BAD and "q_rows" in dm.last_error()
    assert call_attn(dm, attn(dm, max_k=101), k_start=None) == BAD and "k_rows" in dm.last_error()
    big = attn(dm, docs=1, max_k=200000, k_rows=200000, max_q=1, q_rows=1)
    need = dm.lib().dit_attention_workspace_bytes(big)
    assert 0 < need < 1 << 30
    assert call_attn(dm, big, n=need - 1) == WS
    assert call_attn(dm, big, ws=None) == BAD and call_attn(dm, big, ws=P + 16) == BAD


@pytest.mark.parametrize("row,head,rows,ok", [
    (512, 64, 100, True), (64, 6400, 100, True), (1024, 128, 100, True),      # by row, by head, with gaps
    (128, 64 + 128 * 100, 100, True), (448, 64, 1, True), (64, 128, 2, True),  # ... one row, rows between the heads
    (1088, 256, 100, True),                                                    # 4 head strides are a row less a piece
    (64, 64, 100, False), (128, 64, 100, False), (504, 64, 100, False), (448, 64, 2, False), (64, 6336, 100, False),
    (64, 192, 4, False), (1024, 256, 100, False), (1032, 256, 100, False), (1016, 256, 100, False)])
def test_attention_pieces_of_o_do_not_overlap(dm, row, head, rows, ok):
    s = attn(dm, o_row=row, o_head=head, q_rows=rows)
    at = {(r, h): r * row + h * head for r in range(rows) for h in range(8)}
    starts = sorted(at.values())
    assert ok == all(b - a >= 64 for a, b in zip(starts, starts[1:]))
    bad = dm.lib().dit_attention_workspace_bytes(s) == ctypes.c_size_t(-1).value
    assert bad != ok
    if not ok:
        assert call_attn(dm, s) == BAD and "o strides" in dm.last_error()


@pytest.mark.parametrize("max_q", [(1 << 27) // 33, (1 << 27) // 31])
def test_attention_merge_grid(dm, max_q):
    """Rows divide their keys only where the merge pass, a thread for four columns, has fewer than 2^32 threads."""
    s = attn(dm, docs=1, heads=32, kv_heads=16, head_dim=128, q_rows=max_q, max_q=max_q, k_rows=1 << 29, max_k=1 << 29, mask=1,
             q_row=4096, q_head=128, k_row=2048, k_head=128, v_row=2048, v_head=128, o_row=4096, o_head=128)
    need = dm.lib().dit_attention_workspace_bytes(s)
    assert need != ctypes.c_size_t(-1).value
    assert (need > 0) == (max_q * 32 * 32 < 1 << 32)


def test_attention_of_no_rows(dm):
    """Nothing to do is no error, and needs no tensors."""
    s = attn(dm, q_rows=0, max_q=0)
    assert call_attn(dm, s, q=None, o=None, ws=None, n=0) == 0


def test_quantize(dm):
    f = dm.lib().dit_quantize_fp8

    def call(rows=4, cols=128, block=1, dtype=1, x=P, row=128, codes=P, scale=P):
        return f(rows, cols, block, dtype, x, row, codes, scale, None)
    for kw in (dict(rows=-1), dict(cols=0), dict(cols=12), dict(row=120), dict(row=132), dict(block=2), dict(block=0), dict(dtype=2),
               dict(x=None), dict(x=P + 4), dict(codes=None), dict(codes=P + 1), dict(scale=None), dict(scale=P + 2)):
        assert call(**kw) == BAD, kw
    assert call(rows=70000 * 128, block=128) == UNSUP
    assert call(rows=1 << 28) == UNSUP and call(rows=1 << 20, cols=1 << 16, row=1 << 16) == UNSUP
    assert call(rows=1, cols=(1 << 30) + 8, row=1 << 31, block=128) == UNSUP
    assert call(rows=0, x=None, codes=None, scale=None) == 0


def test_linear(dm):
    f = dm.lib().dit_linear_fp8

    def call(M=4, K=256, N=128, act=0, dtype=1, a=P, sa=P, w=P, sw=P, bias=P, out=P, osc=None, ws=P, n=1 << 40):
        s = dm.LinearShape(M, K, N, act, dtype)
        return f(ctypes.byref(s), a, sa, w, sw, bias, out, osc, ws, n, None)
    for kw in (dict(M=-1), dict(K=0), dict(K=24), dict(N=0), dict(act=2), dict(dtype=3), dict(dtype=2),
               dict(osc=P), dict(a=None), dict(a=P + 8), dict(sa=None), dict(w=None), dict(sw=None), dict(sw=P + 1), dict(bias=P + 2),
               dict(out=None), dict(dtype=2, osc=P + 1)):
        assert call(**kw) == BAD, kw
    assert f(None, P, P, P, P, P, P, None, P, 1 << 40, None) == BAD
    assert call(K=1 << 23) == UNSUP
    assert call(M=0, a=None, sa=None, w=None, sw=None, bias=None, out=None, ws=None, n=0) == 0
    # where a product is divided over k, its workspace is checked
    for M, K, N in ((1, 8192, 256), (64, 12288, 1024)):
        s = dm.linear_shape(M, K, N)
        need = dm.lib().dit_linear_fp8_workspace_bytes(s)
        if need:
            assert call(M=M, K=K, N=N, n=need - 1) == WS
            assert call(M=M, K=K, N=N, ws=None) == BAD


def test_norm(dm):
    f = dm.lib().dit_norm_residual
    names = ("x", "x_out", "y", "w_post", "gate", "w_pre", "shift", "scale", "row_batch", "h", "h_scale")

    def call(shape=None, **kw):
        d = dict(rows=4, hidden=256, batch=2, post=2, pre=1, y_dtype=1, h_dtype=1, eps=1e-6, res_scale=1.0, mod_stride=256)
        d.update(shape or {})
        s = dm.NormShape(*[d[n] for n, _ in dm.NormShape._fields_])
        p = dict.fromkeys(names, P)
        p["h_scale"] = None
        p.update(kw)
        return f(ctypes.byref(s), *[p[n] for n in names], None)
    for sh in (dict(rows=-1), dict(hidden=0), dict(hidden=12), dict(batch=0), dict(post=3), dict(post=-1), dict(pre=0), dict(pre=3),
               dict(y_dtype=2), dict(h_dtype=3), dict(eps=0.0), dict(eps=float("inf")), dict(res_scale=float("nan")),
               dict(mod_stride=128), dict(mod_stride=258), dict(mod_stride=-256), dict(h_dtype=2), dict(post=0)):
        assert call(sh) == BAD, sh
    assert call(dict(hidden=8200, mod_stride=8200)) == UNSUP and call(dict(rows=(1 << 25) + 1)) == UNSUP
    for kw in (dict(x=None), dict(y=None), dict(x_out=None), dict(shift=None), dict(scale=None), dict(h=None), dict(h_scale=P),
               dict(x=P + 8), dict(y=P + 8), dict(gate=P + 4), dict(w_pre=P + 4), dict(row_batch=P + 2), dict(h=P + 2)):
        assert call(**kw) == BAD, kw
    assert call(dict(post=0), y=None, w_post=None, gate=None, x_out=None, h=None, w_pre=None, shift=None, scale=None) == BAD
    assert call(dict(rows=0), x=None, row_batch=None) == 0


@pytest.mark.parametrize("hidden,rows,ok", [(4096, 1 << 25, True), (4096, (1 << 25) + 1, False), (4104, (1 << 24) - 1, True),
                                            (4104, 1 << 24, False), (8192, 1 << 24, False), (8192, 1 << 25, False)])
def test_norm_grid(dm, hidden, rows, ok):
    """Rows of more than 4096 columns take 256 threads each, and a grid has fewer than 2^32.  (What passes is refused
    by the next check, for its pointer.)"""
    s = dm.NormShape(rows, hidden, 1, 0, 1, 0, 1, 1e-6, 1.0, hidden)
    got = dm.lib().dit_norm_residual(ctypes.byref(s), None, None, None, None, None, None, None, None, None, P, None, None)
    assert got == (BAD if ok else UNSUP), dm.last_error()
    assert not ok or "x NULL" in dm.last_error()


@pytest.mark.parametrize("M,K,N,dtype,ok", [
    (1, 4096, (1 << 26) - 16, 1, True), (1, 4096, (1 << 26) - 15, 1, False), (32, 4096, 1 << 26, 0, False),
    (33, 4096, 1 << 26, 1, True), (1, 128, 1 << 26, 2, True),                       # 1024, 512 and 256 threads for 16 columns
    (1 << 20, 128, (1 << 17) - 128, 0, True), (1 << 20, 128, 1 << 17, 0, False),    # fp32 has tiles of 128 x 128 alone
    (1 << 20, 128, 1 << 17, 2, True), (1 << 20, 128, 1 << 19, 2, False)])           # the others larger ones
def test_linear_grids(dm, M, K, N, dtype, ok):
    """No call that passes the checks asks for a grid of 2^32 threads."""
    s = dm.LinearShape(M, K, N, 0, dtype)
    got = dm.lib().dit_linear_fp8(ctypes.byref(s), None, P, P, P, None, P, P if dtype == 2 else None, None, 0, None)
    assert got == (BAD if ok else UNSUP), dm.last_error()
    assert not ok or "a NULL" in dm.last_error()
    assert ok != (dm.lib().dit_linear_fp8_workspace_bytes(s) == ctypes.c_size_t(-1).value)


@pytest.mark.parametrize("M,K,N,dtype", [(1, 8192, 256, 2), (64, 12288, 1021, 2), (1030, 4608, 1160, 1), (1030, 4608, 1160, 0)])
def test_linear_workspace(dm, M, K, N, dtype):
    """Few rows of 8-bit outputs, and products divided over k, need a workspace."""
    s = dm.LinearShape(M, K, N, 0, dtype)
    need = dm.lib().dit_linear_fp8_workspace_bytes(s)
    assert 0 < need < 1 << 30

    def call(ws, n):
        return dm.lib().dit_linear_fp8(ctypes.byref(s), P, P, P, P, None, P, P if dtype == 2 else None, ws, n, None)
    assert call(P, need - 1) == WS and str(need) in dm.last_error()
    assert call(None, need) == BAD and call(P + 16, need) == BAD and "workspace" in dm.last_error()


def test_binding_refuses_host_tensors_wrong_types_and_sizes(dm):
    t = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):  # mixed types
        dm.attn_shape(t, t, t, t.bfloat16(), docs=1, max_q=4, max_k=4)
    with pytest.raises(ValueError):
        dm.attn_shape(t[0], t, t, t, docs=1, max_q=4, max_k=4)
    with pytest.raises(ValueError):
        dm.attn_shape(t, t, t, t, docs=1, max_q=4, max_k=4, mask="window")
    s = dm.attn_shape(t, t, t, t, docs=1, max_q=4, max_k=4)
    with pytest.raises(ValueError, match="device tensor"):
        dm.attention(s, t, t, t, t)
    with pytest.raises(ValueError, match="strides"):
        dm.attention(s, torch.zeros(4, 4, 64)[:, ::2], t, t, t)
    with pytest.raises(ValueError):
        dm.quantize_fp8(torch.zeros(4, 128), torch.zeros(4, 128, dtype=torch.float8_e4m3fn), torch.zeros(4, 1))
    with pytest.raises(ValueError):
        dm.linear_shape(4, 128, 128, act="relu")
    with pytest.raises(ValueError):
        dm.norm_shape(4, 128, post="batch")
    f8 = torch.zeros(4, 128, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="device tensor"):
        dm.linear_fp8(dm.linear_shape(4, 128, 4), f8, torch.zeros(4, 1), f8, torch.zeros(1, 1), torch.zeros(4, 4, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="device tensor"):
        dm.norm_residual(dm.norm_shape(4, 128), torch.zeros(4, 128), None, torch.zeros(4, 128, dtype=torch.bfloat16))


def test_host_code_under_asan_and_ubsan(dm, tmp_path):
    """These tests again with the host code under the sanitizers (as test_abi_sanitized.py does for the block and step)."""
    import os
    import subprocess
    import sys

    from paper_2605_25550_amd import build as B
    if os.environ.get("DITMI_LIB"):
        pytest.skip("the sanitized run itself")
    try:
        rt = B.sanitizer_runtime()
    except RuntimeError as e:
        pytest.skip(str(e))
    lib = B.build_sanitized(str(tmp_path))
    env = dict(os.environ, LD_PRELOAD=rt, DITMI_LIB=lib, ASAN_OPTIONS="detect_leaks=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", __file__, "-q", "-x", "-p", "no:cacheprovider"], cwd=B.ROOT, env=env,
                       capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "AddressSanitizer" not in out and "runtime error:" not in out, out[-4000:]
