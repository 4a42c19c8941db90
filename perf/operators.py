"""Performance cases of the library's stand-alone operators: masked attention
over packed or padded documents, products in 8-bit floating point with a scale
for each block of 128, and the norms around a sub-layer fused with its gate and
residual.

  attention  dit_attention: documents packed in one sequence or padded in
             equal rooms; full, causal or prefix mask; scores capped by a tanh
             or biased by distance; heads that share keys
  quantize   dit_quantize_fp8: rows (1 x 128) or weights (128 x 128) to e4m3
  linear     dit_linear_fp8: e4m3 x e4m3 with block scales, bias, tanh-GELU,
             stored as bf16, fp32 or e4m3 with new scales
  norm       dit_norm_residual: x' = r x + gate * norm(y), h = norm(x') modulated

The sizes are this repository's own workloads (DiT-XL/2, the joint text-image
DiT, the video DiT) and ordinary ones around them.  The plain form of each is
elementary torch arithmetic in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

F8 = torch.float8_e4m3fn
F8_MAX = 448.0
TINY = 2.0 ** -126
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": F8}
BYTES = {"bf16": 2, "f32": 4, "e4m3": 1}


# ---------------------------------------------------------------- the cases
def _attention(name, dtype, heads, kv_heads, head_dim, q, k=None, room=0, mask="full", prefix="", cap=0.0, bias=False):
    c = dict(op="attention", dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, q=q, k=k or q, room=room,
             mask=mask, prefix=prefix, cap=cap, bias=bias)
    return dict(c, name=name) if name else c


def _linear(name, rows, inn, out, act, dtype, bias=True):
    c = dict(op="linear", rows=rows, inn=inn, out=out, act=act, dtype=dtype, bias=bias)
    return dict(c, name=name) if name else c


def _quantize(name, rows, cols, dtype, block):
    c = dict(op="quantize", rows=rows, cols=cols, dtype=dtype, block=block)
    return dict(c, name=name) if name else c


def _norm(name, rows, hidden, post, pre, y, h, res_scale=1.0):
    c = dict(op="norm", rows=rows, hidden=hidden, post=post, pre=pre, y=y, h=h, res_scale=res_scale)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token for each of four requests over caches of very unequal
        # fill, heads sharing keys: latency and the caches' bandwidth.
        _attention("attn_token_b4", "bf16", 24, 8, 128, "1,1,1,1", "4096,1531,77,2900", room=4400, mask="causal",
                   bias=True),
        # DiT-XL/2 requests of different resolutions packed in one sequence.
        _attention("attn_packed_xl2", "bf16", 16, 16, 72, "256,1024,333,64,576,1,400,777"),
        # A caller who wants no 16-bit rounding: prefix mask, distance bias.
        _attention("attn_prefix_f32", "f32", 12, 4, 64, "1024,77,515", mask="prefix", prefix="77,200,0", bias=True),
        # Joint text-image batch of two, text padded to 256, capped scores.
        _attention("attn_joint_pad_cap", "bf16", 24, 24, 128, "4352,4352", "4120,4313", room=4352, cap=30.0),
        # Two clips of the video DiT's token budget in one sequence.
        _attention("attn_video_2clips", "bf16", 24, 24, 128, "12870,4680"),
        # The modulation vectors of eight samples: a product bound by the
        # weights' bytes.
        _linear("linear_cond_b8", 8, 1152, 6912, "none", "f32"),
        # DiT-XL/2's first MLP product over ragged rows, its result handed on
        # in 8 bits.
        _linear("linear_fc1_xl2_1997", 1997, 1152, 4608, "gelu", "e4m3"),
        # The video DiT's second MLP product.
        _linear("linear_fc2_video", 17550, 12288, 3072, "none", "bf16"),
        # Attention output of one 256 px sample on its way to the projection.
        _quantize("quantize_xl2_t256", 256, 1152, "bf16", 1),
        # The video DiT's MLP weights, laid out when a model is loaded.
        _quantize("quantize_weight_video", 12288, 3072, "bf16", 128),
        # Text rows of one joint block: a small call.
        _norm("norm_text_77", 77, 1152, "layer", "layer", "f32", "bf16"),
        # Between attention and MLP of the video DiT, on to an 8-bit product.
        _norm("norm_video_e4m3", 17550, 3072, "rms", "rms", "bf16", "e4m3"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the listed ranges: attention over 1..16 documents of
    1..12870 tokens, products of 1..17550 rows, norms and quantisations of
    1..17550 rows at widths 64..12288."""
    op = rng.choice(["attention", "attention", "attention", "linear", "linear", "quantize", "norm"])
    if op == "attention":
        while True:
            dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
            heads, kv = rng.choice([(6, 6), (12, 4), (16, 16), (16, 2), (24, 24), (24, 8), (16, 1)])
            dh = rng.choice([64, 72, 128])
            docs = rng.choice([1, 1, 2, 3, 5, 8, 16])
            decode = rng.random() < 0.3
            k = [_logint(rng, 1, 12870) for _ in range(docs)]
            q = [rng.choice([1, 1, 1, 4]) for _ in range(docs)] if decode else list(k)
            room = max(max(k), max(q)) + rng.randrange(0, 200) if decode or rng.random() < 0.3 else 0
            if room and not decode:
                q = [room] * docs
            mask = rng.choice(["full", "full", "causal", "prefix"])
            prefix = ",".join(str(rng.randrange(0, n + 1)) for n in k) if mask == "prefix" else ""
            cap = rng.choice([0.0, 0.0, 0.0, 30.0, 50.0])
            c = _attention("", dtype, heads, kv, dh, ",".join(map(str, q)), ",".join(map(str, k)), room, mask, prefix,
                           cap, rng.random() < 0.25)
            # the plain form's padded scores bound the drawn cost too
            if docs * max(q) * max(k) * heads <= (2 if dtype == "bf16" else 0.25) * 12870 ** 2 * 24:
                return c
    if op == "linear":
        while True:
            rows, inn, out = _logint(rng, 1, 17550), 16 * _logint(rng, 4, 768), _logint(rng, 16, 12288)
            if rng.random() < 0.6:
                inn, out = rng.choice([384, 1152, 1536, 4608, 2048, 8192]), rng.choice([384, 1152, 3456, 4608, 2048, 6144])
            if rows * inn * out <= 17550 * 12288 * 3072:
                return _linear("", rows, inn, out, rng.choice(["none", "gelu"]), rng.choice(["bf16", "bf16", "f32", "e4m3"]),
                               rng.random() < 0.8)
    if op == "quantize":
        while True:
            rows, cols = _logint(rng, 1, 17550), 8 * _logint(rng, 2, 1536)
            if rows * cols <= 12288 * 4608:
                return _quantize("", rows, cols, rng.choice(["bf16", "bf16", "f32"]), rng.choice([1, 1, 128]))
    rows, hidden = _logint(rng, 1, 17550), rng.choice([384, 768, 1152, 1536, 2048, 2560, 8 * _logint(rng, 8, 384)])
    return _norm("", rows, hidden, rng.choice(["none", "layer", "rms"]), rng.choice(["layer", "rms"]),
                 rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16", "e4m3"]), rng.choice([1.0, 0.5]))


# ---------------------------------------------------------------- inputs
def _ints(text):
    return [int(v) for v in text.split(",")] if text else []


def _starts(lens):
    return [0] + np.cumsum(lens).tolist()


def _blocks(x, rows):
    """amax of every (rows x 128) block of x, as a whole tensor's blocks."""
    R, C = x.shape
    pr, pc = -R % rows, -C % 128
    x = torch.nn.functional.pad(x.abs(), (0, pc, 0, pr))
    return x.view((R + pr) // rows, rows, (C + pc) // 128, 128).amax(dim=(1, 3))


def _spread(s, rows, R, C):
    """A block scale for every element."""
    return s.repeat_interleave(rows, 0)[:R].repeat_interleave(128, 1)[:, :C]


def _to_e4m3(x, rows):
    """fp32 x to e4m3 with a scale for every (rows x 128) block: the block's
    amax stands for 448, and a block of zeros has the smallest normal scale."""
    scale = (_blocks(x, rows) * (1.0 / F8_MAX)).clamp_min(TINY)
    q = x * _spread(1.0 / scale, rows, *x.shape)
    return q.clamp(-F8_MAX, F8_MAX).to(F8), scale


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    def i32(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    s = {"case": case}
    op = case["op"]
    if op == "attention":
        dt = DTYPES[case["dtype"]]
        H, Hk, dh, room = case["heads"], case["kv_heads"], case["head_dim"], case["room"]
        ql, kl = _ints(case["q"]), _ints(case["k"])
        docs, total_q = len(ql), sum(ql)
        total_k = docs * room if room else sum(kl)
        if total_q == total_k:  # self-attention: views of a fused projection's rows
            qkv = normal(total_q, H + 2 * Hk, dh, dtype=dt)
            s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        else:  # a cache, and new rows that look into it
            s["q"] = normal(total_q, H, dh, dtype=dt)
            s["k"], s["v"] = normal(total_k, Hk, dh, dtype=dt), normal(total_k, Hk, dh, dtype=dt)
        s["o"] = torch.zeros(total_q, H, dh, dtype=dt, device="cuda")
        s["q_start"] = i32(_starts(ql))
        s["k_start"] = i32([d * room for d in range(docs + 1)] if room else _starts(kl))
        s["k_len"] = i32(kl) if room else None
        s["prefix"] = i32(_ints(case["prefix"])) if case["mask"] == "prefix" else None
        s["slopes"] = (torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda", dtype=torch.float32) / H)
                       if case["bias"] else None)
        s["max_q"], s["max_k"] = max(ql), max(kl)
        # the row of each query in [documents * longest]
        s["rows_at"] = torch.tensor([d * max(ql) + i for d, n in enumerate(ql) for i in range(n)], device="cuda")
    elif op == "linear":
        M, K, N = case["rows"], case["inn"], case["out"]
        s["a"], s["a_scale"] = _to_e4m3(normal(M, K) * torch.exp(0.5 * normal(M, 1)), 1)
        s["w"], s["w_scale"] = _to_e4m3(normal(N, K, std=0.02), 128)
        wide = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s["bias"] = normal(N, std=0.02, dtype=wide) if case["bias"] else None
        s["out"] = torch.empty(M, N, dtype=DTYPES[case["dtype"]], device="cuda")
        s["out_scale"] = torch.empty(M, -(-N // 128), device="cuda") if case["dtype"] == "e4m3" else None
    elif op == "quantize":
        R, C, b = case["rows"], case["cols"], case["block"]
        std = 0.02 if b == 128 else 1.0
        s["x"] = normal(R, C, std=std, dtype=DTYPES[case["dtype"]])
        s["q"] = torch.empty(R, C, dtype=F8, device="cuda")
        s["scale"] = torch.empty(-(-R // b), -(-C // 128), device="cuda")
    else:
        R, D = case["rows"], case["hidden"]
        batch = min(R, 3)
        s["x"], s["y"] = normal(R, D), normal(R, D, std=3.0, dtype=DTYPES[case["y"]])
        s["w_post"] = 1 + normal(D, std=0.1) if case["post"] != "none" else None
        s["w_pre"] = 1 + normal(D, std=0.1)
        mod = normal(batch, 3 * D, std=0.5)
        s["gate"], s["shift"], s["scale"] = mod[:, :D], mod[:, D:2 * D], mod[:, 2 * D:]
        s["row_batch"] = i32(sorted(r % batch for r in range(R)))
        s["x_out"] = torch.empty_like(s["x"])
        s["h"] = torch.empty(R, D, dtype=DTYPES[case["h"]], device="cuda")
        s["h_scale"] = torch.empty(R, -(-D // 128), device="cuda") if case["h"] == "e4m3" else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the operator's shape and workspace, kept by a program between calls
        import paper_2605_25550_amd as dm

        op = case["op"]
        if op == "attention":
            s["shape"] = dm.attn_shape(s["q"], s["k"], s["v"], s["o"], docs=s["q_start"].numel() - 1, max_q=s["max_q"],
                                       max_k=s["max_k"], mask=case["mask"], cap=case["cap"])
            s["ws"] = dm.attention_workspace(s["shape"])
        elif op == "linear":
            s["shape"] = dm.linear_shape(case["rows"], case["inn"], case["out"], act=case["act"], dtype=case["dtype"])
            s["ws"] = dm.linear_fp8_workspace(s["shape"])
        elif op == "norm":
            s["shape"] = dm.norm_shape(case["rows"], case["hidden"], batch=s["gate"].shape[0], post=case["post"],
                                       pre=case["pre"], y_dtype=case["y"], h_dtype=case["h"],
                                       mod_stride=s["gate"].stride(0), res_scale=case["res_scale"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2605_25550_amd as dm

        if op == "attention":
            dm.attention(s["shape"], s["q"], s["k"], s["v"], s["o"], s["ws"], q_start=s["q_start"],
                         k_start=s["k_start"], k_len=s["k_len"], prefix=s["prefix"], slopes=s["slopes"])
            return s["o"]
        if op == "linear":
            dm.linear_fp8(s["shape"], s["a"], s["a_scale"], s["w"], s["w_scale"], s["out"], s["ws"], bias=s["bias"],
                          out_scale=s["out_scale"])
            return [s["out"]] if s["out_scale"] is None else [s["out"], s["out_scale"]]
        if op == "quantize":
            dm.quantize_fp8(s["x"], s["q"], s["scale"], block_rows=case["block"])
            return [s["q"], s["scale"]]
        dm.norm_residual(s["shape"], s["x"], s["x_out"], s["h"], y=s["y"], w_post=s["w_post"], gate=s["gate"],
                         w_pre=s["w_pre"], shift=s["shift"], scale=s["scale"], row_batch=s["row_batch"],
                         h_scale=s["h_scale"])
        return [s["x_out"], s["h"]] if s["h_scale"] is None else [s["x_out"], s["h"], s["h_scale"]]

    if op == "attention":
        return _plain_attention(s)
    if op == "linear":
        a = s["a"].float() * _spread(s["a_scale"], 1, *s["a"].shape)
        w = s["w"].float() * _spread(s["w_scale"], 128, *s["w"].shape)
        y = a @ w.t()
        if s["bias"] is not None:
            y = y + s["bias"].float()
        if case["act"] == "gelu":
            y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
        return list(_to_e4m3(y, 1)) if case["dtype"] == "e4m3" else [y.to(DTYPES[case["dtype"]])]
    if op == "quantize":
        return list(_to_e4m3(s["x"].float(), case["block"]))
    at = s["row_batch"].long()
    y = s["y"].float()
    if case["post"] != "none":
        y = _plain_norm(y, case["post"]) * s["w_post"]
    x = case["res_scale"] * s["x"] + s["gate"][at] * y
    h = _plain_norm(x, case["pre"]) * s["w_pre"] * (1 + s["scale"][at]) + s["shift"][at]
    return [x, *_to_e4m3(h, 1)] if case["h"] == "e4m3" else [x, h.to(DTYPES[case["h"]])]


def _plain_norm(x, kind, eps=1e-6):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)


def _plain_attention(s):
    case = s["case"]
    H, Hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    G, docs = H // Hk, s["q_start"].numel() - 1
    mq, mk = s["max_q"], s["max_k"]
    i = torch.arange(mq, device="cuda")[None, :]
    j = torch.arange(mk, device="cuda")[None, :]
    qn = (s["q_start"][1:] - s["q_start"][:-1])[:, None]
    kn = (s["k_len"] if s["k_len"] is not None else s["k_start"][1:] - s["k_start"][:-1])[:, None]
    # every document padded to the longest, its spare rows reading row 0
    q = s["q"].float()[torch.where(i < qn, s["q_start"][:-1, None] + i, 0)]
    at = torch.where(j < kn, s["k_start"][:-1, None] + j, 0)
    k, v = s["k"].float()[at], torch.where((j < kn)[..., None, None], s["v"].float()[at], 0)
    q = q.view(docs, mq, Hk, G, dh).permute(0, 2, 3, 1, 4).reshape(docs * Hk, G * mq, dh).contiguous()
    k = k.permute(0, 2, 3, 1).reshape(docs * Hk, dh, mk).contiguous()
    v = v.permute(0, 2, 1, 3).reshape(docs * Hk, mk, dh).contiguous()
    sc = torch.matmul(q * (1.0 / math.sqrt(dh)), k).view(docs, Hk, G, mq, mk)
    if case["cap"] > 0:
        sc = case["cap"] * torch.tanh(sc / case["cap"])
    here = (i + kn - qn)[:, :, None]  # the key at a query's own place
    key = torch.arange(mk, device="cuda")[None, None, :]
    if case["bias"]:
        sc = sc - s["slopes"].view(1, Hk, G, 1, 1) * (here - key).abs()[:, None, None]
    seen = (key < kn[:, :, None]).expand(docs, mq, mk)
    if case["mask"] == "causal":
        seen = seen & (key <= here)
    elif case["mask"] == "prefix":
        seen = seen & ((key <= here) | (key < s["prefix"][:, None, None]))
    sc = sc.masked_fill(~seen[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(torch.isinf(top), 0.0, top))
    del sc
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(docs * Hk, G * mq, mk), v).view(docs, Hk, G, mq, dh)
    o = o / torch.where(total == 0, 1.0, total)
    return o.permute(0, 3, 1, 2, 4).reshape(docs * mq, H, dh)[s["rows_at"]].to(s["o"].dtype)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "attention":
        H, Hk, dh, e = case["heads"], case["kv_heads"], case["head_dim"], BYTES[case["dtype"]]
        ql, kl = _ints(case["q"]), _ints(case["k"])
        pairs = 0
        for d, (nq, nk) in enumerate(zip(ql, kl)):
            seen = np.full(nq, nk, dtype=np.int64)
            if case["mask"] != "full":
                seen = np.clip(np.arange(nq, dtype=np.int64) + nk - nq + 1, 0, nk)
            if case["mask"] == "prefix":
                seen = np.maximum(seen, min(nk, _ints(case["prefix"])[d]))
            pairs += int(seen.sum())
        return {"bytes": 2 * e * dh * (H * sum(ql) + Hk * sum(kl)), "flops": 4 * dh * H * pairs}
    if op == "linear":
        M, K, N = case["rows"], case["inn"], case["out"]
        kb, nb = -(-K // 128), -(-N // 128)
        out = M * N * BYTES[case["dtype"]] + (4 * M * nb if case["dtype"] == "e4m3" else 0)
        return {"bytes": M * K + N * K + 4 * kb * (M + nb) + out, "flops": 2 * M * N * K}
    if op == "quantize":
        R, C, b = case["rows"], case["cols"], case["block"]
        return {"bytes": R * C * (BYTES[case["dtype"]] + 1) + 4 * -(-R // b) * -(-C // 128), "flops": 3 * R * C}
    R, D = case["rows"], case["hidden"]
    h = R * D * BYTES[case["h"]] + (4 * R * -(-D // 128) if case["h"] == "e4m3" else 0)
    return {"bytes": R * D * (8 + BYTES[case["y"]]) + h, "flops": 16 * R * D}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    """run()'s outputs in 64 bits and not rounded: a code of 8 bits stands for
    its block's value over the scale."""
    s = _inputs(case, seed)
    op = case["op"]

    def codes(h, rows):
        R, C = h.shape
        nr, nc = -(-R // rows), -(-C // 128)
        full = torch.zeros(nr * rows, nc * 128, dtype=torch.float64, device="cuda")
        full[:R, :C] = h
        tiles = full.reshape(nr, rows, nc, 128)
        scale = torch.maximum(tiles.abs().amax(3).amax(1) / F8_MAX, torch.tensor(TINY, dtype=torch.float64, device="cuda"))
        q = tiles / scale[:, None, :, None]
        return [q.reshape(nr * rows, nc * 128)[:R, :C].contiguous(), scale]

    if op == "attention":
        return _exact_attention(case, s)
    if op == "linear":
        M, K, N = case["rows"], case["inn"], case["out"]
        y = torch.zeros(M, N, dtype=torch.float64, device="cuda")
        for b in range(0, N, 128):  # one row of weight blocks at a time
            cols = torch.arange(K, device="cuda") // 128
            a = s["a"].double() * s["a_scale"].double()[:, cols] if b == 0 else a
            y[:, b:b + 128] = a @ (s["w"][b:b + 128].double() * s["w_scale"].double()[b // 128, cols]).t()
        if s["bias"] is not None:
            y += s["bias"].double()
        if case["act"] == "gelu":
            y = y * torch.sigmoid(math.sqrt(8 / math.pi) * (y + 0.044715 * y ** 3))
        return codes(y, 1) if case["dtype"] == "e4m3" else [y]
    if op == "quantize":
        return codes(s["x"].double(), case["block"])
    at = s["row_batch"].long()

    def unit(z, kind):
        var = z.var(-1, unbiased=False, keepdim=True) if kind == "layer" else z.pow(2).mean(-1, keepdim=True)
        return (z - (z.mean(-1, keepdim=True) if kind == "layer" else 0)) / torch.sqrt(var + 1e-6)

    y = s["y"].double()
    if case["post"] != "none":
        y = unit(y, case["post"]) * s["w_post"].double()
    x = case["res_scale"] * s["x"].double() + s["gate"].double()[at] * y
    h = unit(x, case["pre"]) * s["w_pre"].double() * (1 + s["scale"].double()[at]) + s["shift"].double()[at]
    return [x, *codes(h, 1)] if case["h"] == "e4m3" else [x, h]


def _exact_attention(case, s):
    H, Hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    q0, k0 = s["q_start"].tolist(), s["k_start"].tolist()
    pre = _ints(case["prefix"])
    for d, (nq, nk) in enumerate(zip(_ints(case["q"]), _ints(case["k"]))):
        key = torch.arange(nk, device="cuda")
        for h in range(H):
            k = s["k"][k0[d]:k0[d] + nk, h * Hk // H].double()
            v = s["v"][k0[d]:k0[d] + nk, h * Hk // H].double()
            for r in range(0, nq, 4096):
                n = min(4096, nq - r)
                z = s["q"][q0[d] + r:q0[d] + r + n, h].double() @ k.t() / math.sqrt(dh)
                if case["cap"] > 0:
                    z = torch.tanh(z / case["cap"]) * case["cap"]
                at = torch.arange(r, r + n, device="cuda")[:, None] + (nk - nq)
                if case["bias"]:
                    z = z - s["slopes"][h].double() * (at - key).abs()
                if case["mask"] != "full":
                    ok = key <= at
                    ok = ok | (key < pre[d]) if case["mask"] == "prefix" else ok
                    z = torch.where(ok, z, -math.inf)
                w = torch.exp(z - torch.logsumexp(z, -1, keepdim=True)) if nk else z
                o[q0[d] + r:q0[d] + r + n, h] = torch.nan_to_num(w, nan=0.0) @ v
    return o
