"""Queries and keys where a wave takes several chunks of heads, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_25550_amd as dm
from test_operators_gpu import close, i32, np64
from test_operators_plans import chunks
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


def one_wave_many(R, H, Hk, dh, Hv=0):
    """The call is one whose waves take more than one chunk each."""
    fn = dm.lib()._ZN5ditmi11qk_segmentsEiiiii
    assert fn(R, dh, H, Hk, Hv) < chunks(dh, H, Hk, Hv)


PAIRS = {8: (4,), 16: (4, 4), 24: (8,), 40: (8, 8), 64: (8, 12, 12), 72: (18, 18), 128: (20, 22, 22), 200: (60,), 256: (64, 32, 32)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
@pytest.mark.parametrize("R,H,Hk,dh,v,norm", [
    (2100, 24, 8, 128, True, "rms"),    # ten chunks in two segments: q, k and v in turn
    (4097, 16, 5, 72, True, "layer"),   # five in one, each tensor's last chunk in part
    (3431, 16, 16, 72, False, "rms"),   # six in two
    (4100, 13, 3, 64, True, "none"),
    (4099, 1, 1, 256, True, "rms"),     # a tensor a chunk
    (2049, 9, 3, 200, False, "layer"),  # seven in two: one wave has a chunk more
])
def test_waves_of_many_chunks(dtype, pairing, R, H, Hk, dh, v, norm):
    one_wave_many(R, H, Hk, dh, Hk if v else 0)
    pairs = tuple(n // 4 * 4 for n in PAIRS[dh]) if pairing == "halves" else PAIRS[dh]
    Qk(R, H, Hk, dh, dtype, norm, pairs, pairing, v=v, seed=R).run().check()


@pytest.mark.parametrize("dh,H,Hk", [(8, 70, 65), (16, 33, 40), (24, 20, 17), (40, 9, 12)])
def test_narrow_heads_in_waves_of_many_chunks(dh, H, Hk):
    one_wave_many(4097, H, Hk, dh, Hk)
    Qk(4097, H, Hk, dh, "bf16", "rms", PAIRS[dh], v=True, seed=dh).run().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,H,Hk,dh", [(2100, 24, 10, 128), (4097, 16, 5, 72)])
def test_in_place_with_the_next_chunk_on_its_way(dtype, R, H, Hk, dh):
    one_wave_many(R, H, Hk, dh, Hk)
    c = Qk(R, H, Hk, dh, dtype, "rms", PAIRS[dh], v=True, seed=6)
    q, k, v = c.q.clone(), c.k.clone(), c.v.clone()
    c.shape = dm.qk_shape(c.q, c.k, c.q, c.k, v=c.v, v_out=c.v, norm="rms", pairs=PAIRS[dh])
    c.out = [c.q, c.k, c.v]
    c.run().check(q=q, k=k, v=v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_go_elsewhere_in_waves_of_many_chunks(dtype):
    R, n = 2100, 5000
    one_wave_many(R, 24, 8, 128, 8)
    rng = np.random.default_rng(0)
    k_dst, q_dst = rng.permutation(n)[:R], rng.permutation(n)[:R]
    k_dst[7], k_dst[R - 1], q_dst[0], q_dst[9] = -1, n, 2 ** 31 - 1, -2 ** 31
    Qk(R, 24, 8, 128, dtype, "layer", (20, 22, 22), v=True, out_rows=n, k_dst=k_dst.tolist(), q_dst=q_dst.tolist()).run().check()
