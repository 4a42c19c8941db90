"""Performance cases of the library's stand-alone operators around attention and
below 8 bits: queries and keys normed for each head and rotated by positions of
several axes, and linear layers in microscaled 4-bit floating point.

  qk        dit_qk_norm_rope: every head of q and k normed (RMS, layer or not) and
            its pairs turned by the row's positions (row and column; frame, row and
            column), v carried along, rows put into the rooms of a cache
  quantize  dit_quantize_fp4, and dit_dequantize_fp4 behind it: e2m1 codes with a
            power of two for each 32 columns, and the values that they stand for
  linear    dit_linear_fp4: products of two such operands, bias, tanh-GELU, stored
            as bf16, fp32 or quantised anew (then read back)

The sizes are this repository's own workloads (DiT-XL/2, the joint text-image
DiT, the video DiT) and ordinary ones around them.  The plain form of each is
elementary torch arithmetic in 32 bits (angles in 64), rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


# ---------------------------------------------------------------- the cases
def _qk(name, rows, heads, kv_heads, head_dim, dtype, norm, pairs, pairing, far=1.0, v=False, room=0):
    """pairs: of each axis.  far: what the grid's positions are multiplied by.
    room: rows of a cache's room for each row (0: no cache)."""
    c = dict(op="qk", rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, norm=norm, pairs=pairs,
             pairing=pairing, far=far, v=v, room=room)
    return dict(c, name=name) if name else c


def _quantize(name, rows, cols, dtype):
    c = dict(op="quantize", rows=rows, cols=cols, dtype=dtype)
    return dict(c, name=name) if name else c


def _linear(name, rows, inn, out, act, dtype, bias=True):
    c = dict(op="linear", rows=rows, inn=inn, out=out, act=act, dtype=dtype, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token for each of four requests, its keys and values put into
        # the rooms of their caches: latency.
        _qk("qk_token_b4", 4, 24, 8, 128, "bf16", "rms", "64", "halves", far=1000.0, v=True, room=600),
        # DiT-XL/2 requests of several resolutions packed in one sequence, places
        # in a grid of rows and columns.
        _qk("qk_packed_xl2", 3431, 16, 16, 72, "bf16", "layer", "18,18", "interleaved"),
        # A caller who wants no 16-bit rounding, shared keys, positions far out.
        _qk("qk_far_f32", 1997, 12, 4, 64, "f32", "rms", "8,12,12", "halves", far=65536.0),
        # The video DiT's tokens: frame, row and column.
        _qk("qk_video", 17550, 24, 24, 128, "bf16", "rms", "22,21,21", "interleaved"),
        # Attention output of one 256 px sample on its way to the projection.
        _quantize("quantize_xl2_t256", 256, 1152, "bf16"),
        # The video DiT's MLP activations, not yet in 16 bits.
        _quantize("quantize_video_f32", 17550, 12288, "f32"),
        # The modulation vectors of eight samples: a product bound by the
        # weights' bytes.
        _linear("linear_cond_b8", 8, 1152, 6912, "none", "f32"),
        # The text rows of a joint block on their own.
        _linear("linear_text_77", 77, 4608, 1152, "none", "bf16"),
        # DiT-XL/2's first MLP product over ragged rows, its result handed on
        # in 4 bits.
        _linear("linear_fc1_xl2_1997", 1997, 1152, 4608, "gelu", "fp4"),
        # DiT-XL/2's second MLP product, one 512 px batch of four.
        _linear("linear_fc2_xl2_4096", 4096, 4608, 1152, "none", "bf16"),
        # A wide model's second MLP product over the video DiT's tokens.
        _linear("linear_fc2_wide", 17550, 18432, 4608, "none", "bf16"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the listed ranges: 1..17550 rows, heads of 64, 72 and 128 with
    one to three axes, widths of 64..18432."""
    op = rng.choice(["qk", "qk", "quantize", "linear", "linear"])
    rows = _logint(rng, 1, 17550)
    if op == "qk":
        heads, kv = rng.choice([(6, 6), (12, 4), (16, 16), (16, 2), (24, 24), (24, 8), (16, 1)])
        dh = rng.choice([64, 72, 128])
        pairing = rng.choice(["interleaved", "halves"])
        total = dh // 2 if rng.random() < 0.7 else dh // 4 // 4 * 4
        axes = rng.choice([1, 2, 3, 3])
        pairs = [total // axes] * axes
        pairs[0] += total - sum(pairs)
        if axes > 1:
            move = rng.randrange(0, pairs[1])
            pairs[1] -= move
            pairs[0] += move
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        room = rng.choice([0, 0, 0, 3])
        return _qk("", rows, heads, kv, dh, dtype, rng.choice(["rms", "rms", "layer", "none"]), ",".join(map(str, pairs)),
                   pairing, rng.choice([1.0, 1.0, 1000.0, 65536.0]), rng.random() < 0.4, room)
    if op == "quantize":
        return _quantize("", rows, 32 * _logint(rng, 2, 384), rng.choice(["bf16", "bf16", "f32"]))
    while True:
        inn, out = 32 * _logint(rng, 2, 576), _logint(rng, 16, 12288)
        if rng.random() < 0.6:
            inn, out = rng.choice([384, 1152, 1536, 4608, 2048, 8192]), rng.choice([384, 1152, 3456, 4608, 2048, 6144])
        dtype = rng.choice(["bf16", "bf16", "f32", "fp4"])
        if dtype == "fp4":
            out = -(-out // 32) * 32
        if rows * inn * out <= 17550 * 18432 * 4608:
            return _linear("", rows, inn, out, rng.choice(["none", "gelu"]), dtype, rng.random() < 0.8)


# ---------------------------------------------------------------- 4-bit blocks
def _exponents(x):
    """fp32 [R, C] to the exponent of each block of 32: the least e >= -127 with
    amax / 2^e < 7, which is what rounds to at most 6."""
    amax = x.reshape(x.shape[0], -1, 32).abs().amax(-1)
    m, e = torch.frexp(amax)
    return torch.where(amax == 0, -127, (e - 3 + (m >= 0.875)).clamp_min(-127))


def _to_grid(x, e):
    """x / 2^e to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to even codes)."""
    y = torch.ldexp(x.reshape(*e.shape, 32), -e[..., None])
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return torch.round(y / step) * step


def _panels(e):
    """[R, C / 32] exponents as the stored bytes: [ceil(C / 256), R, 8]."""
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 8))
    return s.view(s.shape[0], -1, 8).permute(1, 0, 2).contiguous()


def _pack(x):
    """fp32 [R, C] to codes [R, C / 2] (the even column in the low half) and scales."""
    e = _exponents(x)
    y = _to_grid(x, e)
    # the code of a magnitude, by its double
    table = torch.tensor([0, 1, 2, 3, 4, 0, 5, 0, 6, 0, 0, 0, 7], dtype=torch.uint8, device=x.device)
    c = (table[(y.abs() * 2).long()] + torch.where(torch.signbit(y), 8, 0).to(torch.uint8)).view(x.shape[0], -1, 2)
    return c[..., 0] + 16 * c[..., 1], _panels(e)


def _unpack(codes, scale):
    """The values of codes and scales in fp32."""
    R, half = codes.shape
    table = torch.tensor(E2M1 + [-v for v in E2M1], device=codes.device)
    y = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).view(R, -1, 32)
    s = scale.permute(1, 0, 2).reshape(R, -1)[:, :half // 16]
    return (y * torch.exp2(s.float() - 127)[..., None]).view(R, 2 * half)


# ---------------------------------------------------------------- inputs
def _ints(text):
    return [int(v) for v in text.split(",")]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    def pick(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)

    s = {"case": case}
    op = case["op"]
    if op == "qk":
        R, H, Hk, dh, dt = case["rows"], case["heads"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
        # views of a fused projection's rows
        qkv = normal(R, H + 2 * Hk, dh, std=1.5, dtype=dt)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:] if case["v"] else None
        s["w_q"], s["w_k"] = [None, None] if case["norm"] == "none" else [1 + normal(dh, std=0.1), 1 + normal(dh, std=0.1)]
        # places in a grid, row after row, from a random origin on
        pairs = _ints(case["pairs"])
        grid = torch.arange(R, device="cuda")[:, None] // torch.tensor([1560, 52, 1][-len(pairs):], device="cuda")
        grid = grid % torch.tensor([100000, 30, 52][-len(pairs):], device="cuda") if len(pairs) > 1 else grid
        s["pos"] = (grid * case["far"]).int() + pick(0, 1000, 1, len(pairs))
        s["freqs"] = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n) for n in pairs])
        cache = R * case["room"] if case["room"] else R
        s["q_out"] = torch.zeros(R, H, dh, dtype=dt, device="cuda")
        s["k_out"] = torch.zeros(cache, Hk, dh, dtype=dt, device="cuda")
        s["v_out"] = torch.zeros(cache, Hk, dh, dtype=dt, device="cuda") if case["v"] else None
        # one slot in each row's room
        s["k_dst"] = None
        if case["room"]:
            s["k_dst"] = torch.arange(R, dtype=torch.int32, device="cuda") * case["room"] + pick(0, case["room"], R)
    elif op == "quantize":
        R, C = case["rows"], case["cols"]
        s["x"] = (normal(R, C) * torch.exp(normal(R, 1))).to(DTYPES[case["dtype"]])
        s["codes"] = torch.empty(R, C // 2, dtype=torch.uint8, device="cuda")
        s["scale"] = torch.empty(-(-C // 256), R, 8, dtype=torch.uint8, device="cuda")
        s["back"] = torch.empty(R, C, dtype=s["x"].dtype, device="cuda")
    else:
        M, K, N = case["rows"], case["inn"], case["out"]
        s["a"], s["a_scale"] = _pack(normal(M, K) * torch.exp(0.5 * normal(M, 1)))
        s["w"], s["w_scale"] = _pack(normal(N, K, std=0.02))
        wide = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s["bias"] = normal(N, std=0.02, dtype=wide) if case["bias"] else None
        s["out_scale"] = None
        if case["dtype"] == "fp4":
            s["out"] = torch.empty(M, N // 2, dtype=torch.uint8, device="cuda")
            s["out_scale"] = torch.empty(-(-N // 256), M, 8, dtype=torch.uint8, device="cuda")
            s["back"] = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        else:
            s["out"] = torch.empty(M, N, dtype=DTYPES[case["dtype"]], device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the operator's shape and workspace, kept by a program between calls
        import paper_2605_25550_amd as dm

        if case["op"] == "qk":
            s["shape"] = dm.qk_shape(s["q"], s["k"], s["q_out"], s["k_out"], v=s["v"], v_out=s["v_out"], norm=case["norm"],
                                     pairs=_ints(case["pairs"]), pairing=case["pairing"], eps=1e-6)
        elif case["op"] == "linear":
            s["shape"] = dm.linear_shape(case["rows"], case["inn"], case["out"], act=case["act"], dtype=case["dtype"])
            s["ws"] = dm.linear_fp4_workspace(s["shape"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2605_25550_amd as dm

        if op == "qk":
            dm.qk_norm_rope(s["shape"], s["q"], s["k"], s["q_out"], s["k_out"], v=s["v"], v_out=s["v_out"], w_q=s["w_q"],
                            w_k=s["w_k"], pos=s["pos"], freqs=s["freqs"], k_dst=s["k_dst"])
            return [s["q_out"], s["k_out"]] + ([s["v_out"]] if case["v"] else [])
        if op == "quantize":
            dm.quantize_fp4(s["x"], s["codes"], s["scale"])
            dm.dequantize_fp4(s["codes"], s["scale"], s["back"])
            return [s["back"]]
        dm.linear_fp4(s["shape"], s["a"], s["a_scale"], s["w"], s["w_scale"], s["out"], s["ws"], bias=s["bias"],
                      out_scale=s["out_scale"])
        if case["dtype"] != "fp4":
            return [s["out"]]
        dm.dequantize_fp4(s["out"], s["out_scale"], s["back"])
        return [s["back"]]

    if op == "qk":
        return _plain_qk(s)
    if op == "quantize":
        x = s["x"].float()
        e = _exponents(x)
        return [torch.ldexp(_to_grid(x, e), e[..., None]).view_as(x).to(s["x"].dtype)]
    y = _unpack(s["a"], s["a_scale"]) @ _unpack(s["w"], s["w_scale"]).t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if case["act"] == "gelu":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    if case["dtype"] == "fp4":
        e = _exponents(y)
        return [torch.ldexp(_to_grid(y, e), e[..., None]).view_as(y).to(torch.bfloat16)]
    return [y.to(s["out"].dtype)]


def _plain_qk(s):
    case = s["case"]
    pairs = _ints(case["pairs"])
    P = sum(pairs)
    axis = torch.repeat_interleave(torch.arange(len(pairs), device="cuda"), torch.tensor(pairs, device="cuda"))
    t = s["pos"].double()[:, axis] * s["freqs"]
    cos, sin = torch.cos(t).float()[:, None], torch.sin(t).float()[:, None]
    first, second = ((slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if case["pairing"] == "interleaved"
                     else (slice(0, P), slice(P, 2 * P)))

    def one(x, w, out, dst):
        x = x.float()
        if case["norm"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        if case["norm"] != "none":
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        y = x.clone()
        a, b = x[..., first], x[..., second]
        y[..., first] = a * cos - b * sin
        y[..., second] = a * sin + b * cos
        y = y.to(out.dtype)
        if dst is None:
            return y
        out[dst.long()] = y
        return out

    got = [one(s["q"], s["w_q"], s["q_out"], None), one(s["k"], s["w_k"], s["k_out"], s["k_dst"])]
    if case["v"]:
        if s["k_dst"] is None:
            return got + [s["v"].clone()]
        s["v_out"][s["k_dst"].long()] = s["v"]
        got.append(s["v_out"])
    return got


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "qk":
        R, H, Hk, dh, e = case["rows"], case["heads"], case["kv_heads"], case["head_dim"], BYTES[case["dtype"]]
        P, axes = sum(_ints(case["pairs"])), len(_ints(case["pairs"]))
        return {"bytes": 2 * e * R * dh * (H + (2 if case["v"] else 1) * Hk) + 4 * R * axes + 8 * P,
                "flops": 8 * R * dh * (H + Hk)}
    if op == "quantize":  # the values in, the codes and scales out and in again, the values out
        R, C = case["rows"], case["cols"]
        return {"bytes": 2 * R * C * BYTES[case["dtype"]] + 2 * (R * C // 2 + R * C // 32), "flops": 4 * R * C}
    M, K, N = case["rows"], case["inn"], case["out"]
    out = 2 * M * N + 2 * (M * N // 2 + M * N // 32) if case["dtype"] == "fp4" else M * N * BYTES[case["dtype"]]
    return {"bytes": (M + N) * (K // 2 + K // 32) + out, "flops": 2 * M * N * K}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    """run()'s outputs in 64 bits: a rotation as a product of complex numbers, 4-bit
    values by the distances to all of them, products of unpacked operands.  A product
    stored in 4 bits has no such value: a sum next to a border may take either code."""
    s = _inputs(case, seed)
    op = case["op"]
    dev = "cuda"
    grid = torch.tensor(E2M1, dtype=torch.float64, device=dev)

    def values(z):
        """The 4-bit values that stand for z."""
        got = torch.empty_like(z)
        for r in range(0, z.shape[0], 512):
            b = z[r:r + 512].reshape(-1, 32)
            top = b.abs().amax(1, keepdim=True)
            e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2
            e = torch.where(top / torch.exp2(e) >= 7, e + 1, e)
            e = torch.where(top / torch.exp2(e - 1) < 7, e - 1, e)
            u = (b / torch.exp2(e)).abs()
            best = torch.zeros_like(u)
            for i in range(1, 8):  # past the middle, or on it when the next code is even
                mid = (grid[i - 1] + grid[i]) / 2
                best = torch.where((u > mid) | ((u == mid) & (i % 2 == 0)), grid[i], best)
            got[r:r + 512] = (torch.sign(b) * best * torch.exp2(e)).view(-1, z.shape[1])
        return got

    if op == "quantize":
        return [values(s["x"].double())]
    if op == "linear":
        if case["dtype"] == "fp4":
            return None

        def wide(codes, scale):
            c = torch.zeros(codes.shape[0], codes.shape[1], 2, dtype=torch.int64, device=dev)
            c[..., 0], c[..., 1] = codes % 16, codes // 16
            v = grid[c % 8] * (1 - 2 * (c // 8))
            r = torch.arange(codes.shape[0], device=dev)[:, None]
            col = torch.arange(2 * codes.shape[1], device=dev)[None]
            return v.view(codes.shape[0], -1) * torch.exp2(scale[col // 256, r, col % 256 // 32].double() - 127)

        w = wide(s["w"], s["w_scale"])
        y = torch.empty(case["rows"], case["out"], dtype=torch.float64, device=dev)
        for r in range(0, case["rows"], 2048):
            y[r:r + 2048] = wide(s["a"][r:r + 2048], s["a_scale"][:, r:r + 2048]) @ w.t()
        if s["bias"] is not None:
            y += s["bias"].double()
        if case["act"] == "gelu":
            y = y * torch.sigmoid(math.sqrt(8 / math.pi) * (y + 0.044715 * y ** 3))
        return [y]

    pairs = _ints(case["pairs"])
    P = sum(pairs)
    turn = torch.cat([s["pos"][:, a:a + 1].double() * f for a, f in enumerate(s["freqs"].split(pairs))], 1)
    turn = torch.polar(torch.ones_like(turn), turn)[:, None]

    def one(x, w):
        z = x.double()
        if case["norm"] != "none":
            mean = z.mean(-1, keepdim=True) if case["norm"] == "layer" else 0.0
            z = (z - mean) / torch.sqrt((z - mean).pow(2).mean(-1, keepdim=True) + 1e-6) * w.double()
        head, tail = z[..., :2 * P], z[..., 2 * P:]
        if case["pairing"] == "interleaved":
            c = torch.view_as_complex(head.reshape(*head.shape[:-1], P, 2).contiguous()) * turn
            head = torch.view_as_real(c).reshape(head.shape)
        else:
            c = torch.complex(head[..., :P].contiguous(), head[..., P:].contiguous()) * turn
            head = torch.cat([c.real, c.imag], -1)
        return torch.cat([head, tail], -1)

    def put(z, out):
        if s["k_dst"] is None:
            return z
        full = out.double()
        full[s["k_dst"].long()] = z
        return full

    got = [one(s["q"], s["w_q"]), put(one(s["k"], s["w_k"]), s["k_out"])]
    return got + [put(s["v"].double(), s["v_out"])] if case["v"] else got
