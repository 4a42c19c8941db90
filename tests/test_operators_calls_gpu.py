"""The compiled calls of queries and keys and of the 4-bit operators: they are loaded and
take the ordinary calls, and what they take or leave gives what the checks in Python
give: results, errors, on every stream and captured."""
import threading

import pytest
import torch

import paper_2605_25550_amd as dm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(params=["compiled", "python"])
def path(request, monkeypatch):
    dm.lib()
    assert dm._CALLS is not None, "the compiled calls are not built"
    if request.param == "python":
        monkeypatch.setattr(dm, "_CALLS", None)
    return request.param


class Seen:
    """The compiled calls, with what each returned."""

    def __init__(self, calls):
        self.calls, self.returned = calls, []

    def __getattr__(self, name):
        def call(*args):
            st = getattr(self.calls, name)(*args)
            self.returned.append((name, st))
            return st
        return call


def tensors(rows=5, heads=4, kv_heads=2, dh=64, cols=128, out=96, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(7)

    def new(*size, kind=torch.float32):
        return torch.randn(*size, generator=g, dtype=torch.float64).to(kind).to(DEV)
    packed = new(rows, heads + 2 * kv_heads, dh, kind=dtype)
    t = dict(q=packed[:, :heads], k=packed[:, heads:heads + kv_heads], v=packed[:, heads + kv_heads:],
             q_out=torch.zeros(rows, heads, dh, dtype=dtype, device=DEV),
             k_out=torch.zeros(rows + 3, kv_heads, dh, dtype=dtype, device=DEV), w_q=new(dh), w_k=new(dh),
             pos=torch.arange(2 * rows, dtype=torch.int32, device=DEV).view(rows, 2), freqs=dm.rope_freqs((16, 16), device=DEV),
             k_dst=torch.arange(rows, 0, -1, dtype=torch.int32, device=DEV) + 1, x=new(rows, cols, kind=dtype), w=new(out, cols),
             bias=new(out, kind=torch.bfloat16), y=torch.zeros(rows, out, dtype=torch.bfloat16, device=DEV),
             back=torch.zeros(rows, cols, device=DEV))
    t["v_out"] = torch.zeros_like(t["k_out"])
    for n, r in (("x", rows), ("w", out)):
        t[n + "_codes"] = torch.zeros(r, cols // 2, dtype=torch.uint8, device=DEV)
        t[n + "_scale"] = torch.zeros(-(-cols // 256), r, 8, dtype=torch.uint8, device=DEV)
    t["y4"] = torch.zeros(rows, out // 2, dtype=torch.uint8, device=DEV)
    t["y4_scale"] = torch.zeros(-(-out // 256), rows, 8, dtype=torch.uint8, device=DEV)
    return t


def run(t, **kw):
    qs = dm.qk_shape(t["q"], t["k"], t["q_out"], t["k_out"], t["v"], t["v_out"], pairs=(16, 16))
    dm.qk_norm_rope(qs, t["q"], t["k"], t["q_out"], t["k_out"], t["v"], t["v_out"], t["w_q"], t["w_k"], t["pos"], t["freqs"],
                    k_dst=t["k_dst"], **kw)
    for n in ("x", "w"):
        dm.quantize_fp4(t[n], t[n + "_codes"], t[n + "_scale"], **kw)
    dm.dequantize_fp4(t["x_codes"], t["x_scale"], t["back"], **kw)
    a = (t["x_codes"], t["x_scale"], t["w_codes"], t["w_scale"])
    M, K, N = len(t["x"]), t["x"].shape[1], len(t["w"])
    dm.linear_fp4(dm.linear_shape(M, K, N), *a, t["y"], dm.linear_fp4_workspace(dm.linear_shape(M, K, N)), t["bias"], **kw)
    dm.linear_fp4(dm.linear_shape(M, K, N, dtype="fp4"), *a, t["y4"], bias=t["bias"], out_scale=t["y4_scale"], **kw)


OUTS = ("q_out", "k_out", "v_out", "x_codes", "x_scale", "w_codes", "w_scale", "back", "y", "y4", "y4_scale")


def test_they_take_the_ordinary_calls(monkeypatch):
    dm.lib()
    assert dm._CALLS is not None, "the compiled calls are not built"
    t, p = tensors(), tensors()
    seen = Seen(dm._CALLS)
    monkeypatch.setattr(dm, "_CALLS", seen)
    run(t)
    assert seen.returned == [("qk_norm_rope", 0), ("quantize_fp4", 0), ("quantize_fp4", 0), ("dequantize_fp4", 0),
                             ("linear_fp4", 0), ("linear_fp4", 0)]
    monkeypatch.setattr(dm, "_CALLS", None)
    run(p)
    for n in OUTS:
        assert torch.equal(t[n], p[n]) and (n == "x_scale" or t[n].any()), n


def test_streams(path):
    """On the current stream, on one that is given, and captured: the same results."""
    ref, cur, given, graphed = (tensors() for _ in range(4))
    run(ref)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)  # what runs on another stream than this one is done before it
        for n in ("q", "k", "v", "x"):
            cur[n] = cur[n] * 1
        run(cur)
    torch.cuda._sleep(2_000_000)
    run(given, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(graphed)
    for _ in range(3):
        for n in OUTS:
            graphed[n].zero_()
        g.replay()
        torch.cuda.synchronize()
        for n in OUTS:
            assert torch.equal(graphed[n], ref[n]), n
    for n in OUTS:
        assert torch.equal(cur[n], ref[n]) and torch.equal(given[n], ref[n]), n


def test_threads(path):
    """Calls of several threads at once, each on a stream of its own."""
    ref = tensors()
    run(ref)
    sets = [tensors() for _ in range(4)]
    torch.cuda.synchronize()
    failed = []

    def work(t):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    run(t)
                with pytest.raises(ValueError, match="elements"):
                    dm.quantize_fp4(t["x"], t["x_codes"][1:], t["x_scale"])
        except BaseException as e:  # noqa: BLE001  (reported by the test's own thread)
            failed.append(e)
    threads = [threading.Thread(target=work, args=(t,)) for t in sets]
    for th in threads:
        th.start()
    for th in threads:
        th.join(60)
    torch.cuda.synchronize()
    assert not failed, failed
    for t in sets:
        for n in OUTS:
            assert torch.equal(t[n], ref[n]), n


def test_strides_that_no_element_uses(path):
    """One row, one head, no rows: whatever strides torch states."""
    t = tensors(rows=1)
    ref = tensors(rows=1)
    run(ref)
    for n in ("q", "k", "v", "q_out"):
        t[n] = t[n].as_strided(t[n].shape, (12344, t[n].stride(1), 1))
    t["x"] = t["x"].as_strided(t["x"].shape, (9999, 1))
    run(t)
    for n in OUTS:
        assert torch.equal(t[n], ref[n]), n
    none = tensors(rows=0)
    none["k_dst"] = none["k_dst"][:0]
    run(none)
    torch.cuda.synchronize()
    assert not none["k_out"].any() and not none["v_out"].any() and none["w_codes"].any()
    away = tensors()  # no row of the outputs: every row of k and v is dropped
    away["k_out"], away["v_out"] = away["k_out"][:0], away["v_out"][:0]
    run(away)
    full = tensors()
    run(full)
    assert torch.equal(away["q_out"], full["q_out"])


def refused(fn):
    with pytest.raises(Exception) as e:
        fn()
    dm._CALLS, kept = None, dm._CALLS
    try:
        with pytest.raises(type(e.value)) as again:
            fn()
    finally:
        dm._CALLS = kept
    assert str(e.value) == str(again.value) and str(e.value)


LINEAR = dict(a="x_codes", a_scale="x_scale", w="w_codes", w_scale="w_scale", out="y", bias="bias")


@pytest.mark.parametrize("name", list(LINEAR))
@pytest.mark.parametrize("how", ["cpu", "type", "size", "strided", "list"])
def test_linear_refusals(name, how):
    t = tensors()
    s = dm.linear_shape(5, 128, 96)
    x = t[LINEAR[name]]
    x = {"cpu": x.cpu, "type": x.to(torch.int64).clone, "size": x.flatten()[1:].clone, "list": lambda: [1],
         "strided": lambda: torch.stack([x, x], -1)[..., 0]}[how]()
    args = {n: t[k] for n, k in LINEAR.items()}
    args[name] = x
    dm.lib()
    refused(lambda: dm.linear_fp4(s, args["a"], args["a_scale"], args["w"], args["w_scale"], args["out"], None, args["bias"]))


@pytest.mark.parametrize("name", ["q", "k", "v", "q_out", "k_out", "v_out", "w_q", "w_k", "pos", "freqs", "k_dst"])
@pytest.mark.parametrize("how", ["cpu", "type", "size", "strided"])
def test_qk_refusals(name, how):
    t = tensors()
    s = dm.qk_shape(t["q"], t["k"], t["q_out"], t["k_out"], t["v"], t["v_out"], pairs=(16, 16))
    x = t[name]
    t[name] = {"cpu": x.cpu, "type": x.to(torch.int64).clone, "size": x[1:].clone, "strided": lambda: torch.stack([x, x], -1)[..., 0]}[how]()
    dm.lib()
    refused(lambda: dm.qk_norm_rope(s, t["q"], t["k"], t["q_out"], t["k_out"], t["v"], t["v_out"], t["w_q"], t["w_k"],
                                          t["pos"], t["freqs"], k_dst=t["k_dst"]))


def test_other_refusals():
    t = tensors()
    dm.lib()
    s, f = dm.linear_shape(5, 128, 96), dm.linear_shape(5, 128, 96, dtype="e4m3")
    a = (t["x_codes"], t["x_scale"], t["w_codes"], t["w_scale"])
    qs = dm.qk_shape(t["q"], None, t["q_out"], None, pairs=(16, 16))
    for fn in (lambda: dm.linear_fp4(f, *a, t["y"].to(torch.float8_e4m3fn)),
               lambda: dm.linear_fp4(dm.linear_shape(-1, 128, 96), *a, t["y"]),
               lambda: dm.linear_fp4(s, *a, t["y"], torch.zeros(8)),
               lambda: dm.linear_fp4(s, *a, None),
               lambda: dm.linear_fp4(None, *a, t["y"]),
               lambda: dm.linear_fp4(bytes(s), *a, t["y"]),
               lambda: dm.linear_fp4(s, *a, t["y"], out_scale=t["y4_scale"]),
               lambda: dm.linear_fp4(s, t["x_codes"].flatten()[:0], *a[1:], t["y"]),
               lambda: dm.quantize_fp4(t["x"].half(), t["x_codes"], t["x_scale"]),
               lambda: dm.quantize_fp4(t["x"][0], t["x_codes"], t["x_scale"]),
               lambda: dm.quantize_fp4(t["x"].t(), t["x_codes"], t["x_scale"]),
               lambda: dm.quantize_fp4(t["x"], None, t["x_scale"]),
               lambda: dm.quantize_fp4(t["x"], t["x_codes"], t["x_scale"][:, 1:]),
               lambda: dm.quantize_fp4(t["x"][:, :100], t["x_codes"], t["x_scale"]),
               lambda: dm.dequantize_fp4(t["x_codes"], None, t["back"]),
               lambda: dm.dequantize_fp4(t["x_codes"], t["x_scale"], t["back"].cpu()),
               lambda: dm.dequantize_fp4(t["x_codes"].to(torch.int8), t["x_scale"], t["back"]),
               lambda: dm.qk_norm_rope(qs, t["q"], t["k"], t["q_out"], None, pos=t["pos"], freqs=t["freqs"]),
               lambda: dm.qk_norm_rope(qs, None, None, None, None, pos=t["pos"], freqs=t["freqs"]),
               lambda: dm.qk_norm_rope(qs, t["q"], None, None, None, pos=t["pos"], freqs=t["freqs"]),
               lambda: dm.qk_norm_rope(qs, t["q"], None, t["q_out"], None, pos=t["pos"]),
               lambda: dm.qk_norm_rope(qs, t["q"], None, t["q_out"], None, freqs=t["freqs"]),
               lambda: dm.qk_norm_rope(qs, t["q"], None, t["q"], None, pos=t["pos"], freqs=t["freqs"])):
        refused(fn)
