"""Queries and keys where a wave takes several chunks of heads, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from test_operators_gpu import close, i32, np64
from test_operators_qk_gpu import Qk, reference

pytestmark = pytest.mark.gpu


def test_most_rows_of_many_heads():
    """2^24 rows of 20 chunks of heads, from views that overlap (a stride of one head), into a few rows: four waves a
    row would be a grid of 2^32 threads."""
    R, H, dh, places = 1 << 24, 1280, 8, 5
    base = torch.randn(R + H, dh, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    q = base.as_strided((R, H, dh), (dh, dh, 1))
    out = torch.full((places, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    dst = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    rows = [R - 1, 0, 12345678, 2 ** 23, 4096]
    dst[torch.tensor(rows, device="cuda")] = i32(range(places))
    pos = torch.zeros(R, 1, dtype=torch.int32, device="cuda")
    pos[:, 0] = torch.arange(R, device="cuda") % 1000
    freqs, w = dm.rope_freqs((4,)), torch.ones(dh, device="cuda")
    dm.qk_norm_rope(dm.qk_shape(q, None, out, None, pairs=(4,)), q, None, out, None, w_q=w, pos=pos, freqs=freqs, q_dst=dst)
    x = np.stack([np64(base[r:r + H]) for r in rows])
    y, tol = reference(x, 1.0, "rms", (4,), "interleaved", np64(pos)[rows], freqs.cpu().numpy(), "bf16")
    close(np64(out), y, tol, "q")
