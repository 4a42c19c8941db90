"""CPU tests of the refusals of the 4-bit operators and of queries' and keys' norms
and rotation: every call below is refused before any HIP call, so its pointers are
never dereferenced."""
import ctypes

import pytest
import torch

from test_operators_abi import BAD, P, UNSUP, WS, dm  # noqa: F401  (dm: a fixture)


def qk(dm, **kw):
    d = dict(rows=10, heads=8, kv_heads=2, head_dim=64, q_out_rows=10, k_out_rows=10, dtype=1, norm=2, pairing=0, axes=2,
             pairs=(16, 16), eps=1e-6, q_row=512, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, q_out_row=512,
             q_out_head=64, k_out_row=128, k_out_head=64, v_out_row=128, v_out_head=64)
    d.update(kw)
    d["pairs"] = (ctypes.c_int32 * 4)(*d["pairs"])
    return dm.QkShape(*[d[n] for n, _ in dm.QkShape._fields_])


# distinct aligned addresses
Q, K, V, QO, KO, VO = (P * i for i in range(1, 7))


def call_qk(dm, s, q=Q, k=K, v=V, q_out=QO, k_out=KO, v_out=VO, w_q=P, w_k=P, pos=P, freqs=P, q_dst=None, k_dst=None):
    return dm.lib().dit_qk_norm_rope(ctypes.byref(s) if s is not None else None, q, k, v, q_out, k_out, v_out, w_q, w_k, pos,
                                     freqs, q_dst, k_dst, None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), BAD), (dict(heads=-1), BAD), (dict(kv_heads=-1), BAD), (dict(q_out_rows=-1), BAD), (dict(k_out_rows=-1), BAD),
    (dict(heads=0, kv_heads=0), BAD), (dict(heads=65536), UNSUP), (dict(rows=(1 << 24) + 1, q_out_rows=1 << 25), UNSUP),
    (dict(head_dim=60), UNSUP), (dict(head_dim=0), UNSUP), (dict(head_dim=264), UNSUP), (dict(dtype=2), BAD), (dict(dtype=-1), BAD),
    (dict(norm=3), BAD), (dict(norm=-1), BAD), (dict(pairing=2), BAD), (dict(pairing=-1), BAD), (dict(eps=0.0), BAD), (dict(eps=1e-39), BAD),
    (dict(eps=float("nan")), BAD), (dict(eps=float("inf")), BAD), (dict(axes=-1), BAD), (dict(axes=5), BAD),
    (dict(pairs=(16, -1)), BAD), (dict(pairs=(16, 17)), BAD), (dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1)), BAD),
    (dict(pairing=1, pairs=(16, 14)), UNSUP), (dict(q_row=500), BAD), (dict(q_row=256), True), (dict(k_head=60), BAD), (dict(v_row=32), BAD),
    (dict(q_out_row=32), BAD), (dict(k_out_head=-64), BAD), (dict(v_out_row=1 << 23), UNSUP), (dict(q_out_row=448), BAD),
    (dict(q_out_row=64, q_out_head=64), BAD), (dict(k_out_row=64), BAD), (dict(v_out_row=64), BAD),
    (dict(q_out_rows=9), BAD), (dict(k_out_rows=9), BAD), (dict(norm=0), BAD),
])
def test_qk_shapes(dm, kw, want):
    if want is True:  # inputs may overlap one another: refused for another reason
        assert call_qk(dm, qk(dm, **kw), q=None) == BAD and "q NULL" in dm.last_error()
        return
    assert call_qk(dm, qk(dm, **kw)) == want and dm.last_error()


def test_qk_pointers(dm):
    s = qk(dm)
    assert call_qk(dm, None) == BAD
    for n in ("q", "k", "q_out", "k_out"):
        assert call_qk(dm, s, **{n: None}) == BAD and n in dm.last_error()
    for n in ("q", "k", "v", "q_out", "k_out", "v_out", "w_q", "w_k"):
        assert call_qk(dm, s, **{n: 100 * P + 8}) == BAD and n in dm.last_error()
    assert call_qk(dm, s, v=None) == BAD and call_qk(dm, s, v_out=None) == BAD
    none = qk(dm, rows=0)  # tensors without rows have no memory
    assert call_qk(dm, none, q=None, k=None, v=None) == 0 and call_qk(dm, none, v_out=None) == 0
    assert call_qk(dm, s, pos=None) == BAD and "pos" in dm.last_error()
    assert call_qk(dm, s, freqs=None) == BAD and call_qk(dm, s, freqs=P + 4) == BAD and "freqs" in dm.last_error()
    assert call_qk(dm, s, pos=P + 2) == BAD and call_qk(dm, s, q_dst=P + 1) == BAD and call_qk(dm, s, k_dst=P + 2) == BAD
    assert call_qk(dm, qk(dm, kv_heads=0)) == BAD and "v " in dm.last_error()


def test_qk_in_place(dm):
    for kw in (dict(q_out=Q), dict(k_out=K), dict(v_out=V)):
        moved = {"q_out": dict(q_out_row=1024), "k_out": dict(k_out_row=256), "v_out": dict(v_out_row=256)}[next(iter(kw))]
        assert call_qk(dm, qk(dm, **moved), **kw) == BAD and "in place" in dm.last_error()
        assert call_qk(dm, qk(dm), q_dst=P, k_dst=P, **kw) == BAD and "in place" in dm.last_error()


def test_qk_of_no_rows(dm):
    assert call_qk(dm, qk(dm, rows=0, q_out_rows=0, k_out_rows=0), q=None, k=None, v=None, q_out=None, k_out=None, v_out=None) == 0


def test_blocks_of_32(dm):
    f, g = dm.lib().dit_quantize_fp4, dm.lib().dit_dequantize_fp4

    def both(rows=4, cols=128, dtype=1, x=P, row=128, codes=P, scale=P):
        return {f(rows, cols, dtype, x, row, codes, scale, None), g(rows, cols, dtype, codes, scale, x, row, None)}
    for kw in (dict(rows=-1), dict(cols=0), dict(cols=48), dict(cols=-32), dict(row=120), dict(row=132), dict(dtype=2), dict(dtype=3),
               dict(x=None), dict(x=P + 4), dict(codes=None), dict(codes=P + 8), dict(scale=None), dict(scale=P + 4)):
        assert both(**kw) == {BAD}, kw
    assert both(rows=1 << 27) == {UNSUP} and both(rows=1 << 20, cols=1 << 16, row=1 << 16) == {UNSUP}
    assert both(rows=1, cols=(1 << 30) + 32, row=1 << 31) == {UNSUP} and both(row=1 << 41) == {UNSUP}
    assert both(rows=0, x=None, codes=None, scale=None) == {0}


def call_linear(dm, s, a=P, a_scale=P, w=P, w_scale=P, bias=None, out=P, out_scale=None, ws=P, n=1 << 40):
    return dm.lib().dit_linear_fp4(ctypes.byref(s) if s is not None else None, a, a_scale, w, w_scale, bias, out, out_scale, ws, n,
                                   None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), BAD), (dict(inn=0), BAD), (dict(inn=48), BAD), (dict(inn=-32), BAD), (dict(out=0), BAD), (dict(act=2), BAD),
    (dict(act=-1), BAD), (dict(dtype=2), BAD), (dict(dtype=4), BAD), (dict(dtype=-1), BAD), (dict(dtype=3, out=48), BAD),
    (dict(inn=1 << 23), UNSUP), (dict(out=1 << 27), UNSUP), (dict(rows=1 << 27), UNSUP), (dict(rows=1 << 26, out=1 << 26), UNSUP)])
def test_linear_shapes(dm, kw, want):
    d = dict(rows=8, inn=128, out=64, act=0, dtype=1)
    d.update(kw)
    s = dm.LinearShape(d["rows"], d["inn"], d["out"], d["act"], d["dtype"])
    assert call_linear(dm, s, out_scale=P if d["dtype"] == 3 else None) == want and dm.last_error()
    assert dm.lib().dit_linear_fp4_workspace_bytes(s) == ctypes.c_size_t(-1).value
    with pytest.raises(dm.DitError):
        dm.linear_fp4_workspace(s, device="cpu")


def test_linear_pointers_and_workspace(dm):
    s = dm.linear_shape(8, 128, 64)
    assert call_linear(dm, None) == BAD
    for n in ("a", "a_scale", "w", "w_scale", "out"):
        assert call_linear(dm, s, **{n: None}) == BAD and n in dm.last_error()
        assert call_linear(dm, s, **{n: P + 8}) == BAD and n in dm.last_error()
    assert call_linear(dm, s, bias=P + 8) == BAD and call_linear(dm, s, out_scale=P) == BAD
    s4 = dm.linear_shape(8, 128, 64, dtype="fp4")
    assert call_linear(dm, s4) == BAD and "out_scale" in dm.last_error()
    need = dm.lib().dit_linear_fp4_workspace_bytes(s4)
    if need:
        assert call_linear(dm, s4, out_scale=P, n=need - 1) == WS and call_linear(dm, s4, out_scale=P, ws=None) == BAD
        assert call_linear(dm, s4, out_scale=P, ws=P + 16) == BAD
    assert call_linear(dm, dm.linear_shape(0, 128, 64), a=None, w=None, out=None) == 0


def test_other_operators_refuse_4_bit_types(dm):
    s = dm.linear_shape(8, 128, 64, dtype="fp4")
    assert dm.lib().dit_linear_fp8_workspace_bytes(s) == ctypes.c_size_t(-1).value
    with pytest.raises(dm.DitError):
        dm.linear_fp8_workspace(s, device="cpu")


def test_binding_refuses_before_the_library(dm):
    q, k = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q or k"):
        dm.qk_shape(None, None, None, None)
    with pytest.raises(ValueError, match="come together"):
        dm.qk_shape(q, k, q, None)
    with pytest.raises(ValueError, match="axes"):
        dm.qk_shape(q, k, q, k, pairs=(1, 1, 1, 1, 1))
    with pytest.raises(ValueError, match="float32 or all bfloat16"):
        dm.qk_shape(q, k.float(), q, k.float())
    with pytest.raises(ValueError, match="rows"):
        dm.qk_shape(q, k[:3], q, k)
    with pytest.raises(ValueError, match="heads"):
        dm.qk_shape(q, k, q[:, :1], k)
    with pytest.raises(ValueError, match="need k"):
        dm.qk_shape(q, None, q, None, v=k, v_out=k)
    with pytest.raises(ValueError, match="norm"):
        dm.qk_shape(q, k, q, k, norm="batch")
    with pytest.raises(ValueError, match="pairing"):
        dm.qk_shape(q, k, q, k, pairing="thirds")
    s = dm.qk_shape(q, k, q, k, pairs=(32,))
    with pytest.raises(ValueError, match="device tensor"):
        dm.qk_norm_rope(s, q, k, q, k)
    with pytest.raises(ValueError, match="states"):
        dm.qk_norm_rope(s, q, None, q, None)
    for f in (lambda: dm.quantize_fp4(q[0], q[0], q[0]), lambda: dm.dequantize_fp4(q[0], q[0], q[0])):
        with pytest.raises(ValueError, match="device tensor"):
            f()
    with pytest.raises(ValueError):
        dm.linear_fp4(dm.linear_shape(4, 64, 32), q, q, q, q, q)


def test_rope_freqs(dm):
    f = dm.rope_freqs((2, 0, 4), theta=16.0, device="cpu")
    assert f.dtype == torch.float64 and torch.equal(f, torch.tensor([1.0, 0.25, 1.0, 0.5, 0.25, 0.125], dtype=torch.float64))
    assert dm.rope_freqs((), device="cpu").shape == (0,)
