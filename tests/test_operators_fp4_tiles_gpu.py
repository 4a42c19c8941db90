"""4-bit linear layers: every tile's loop over k at work (rings that are filled again, a last panel in part, ranges of
k), with sums that are exact."""
import pytest
import torch

import paper_2605_25550_amd as dm
from test_operators_fp4_gpu import U24, Linear, buffers, np64, quantized
from test_operators_plans import LOOPS

pytestmark = pytest.mark.gpu
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def wide(codes, scale):
    """The values of codes and scales in 64 bits, on the device."""
    table = torch.tensor(E2M1 + [-v for v in E2M1], dtype=torch.float64, device="cuda")
    v = table[torch.stack([codes & 15, codes >> 4], -1).int()].view(codes.shape[0], -1, 32)
    s = scale.permute(1, 0, 2).reshape(codes.shape[0], -1)[:, :v.shape[1]]
    return (v * torch.exp2(s.double() - 127)[..., None]).view(codes.shape[0], -1)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp4"])
@pytest.mark.parametrize("M,K,N,tile,split", LOOPS)
def test_loops(dtype, M, K, N, tile, split):
    """Random codes with scales of 1/2 and 1: every term is a multiple of 1/16, and their magnitudes' sum is below
    2^20, so that fp32 holds every partial sum exactly and the result does not depend on an order."""
    g = torch.Generator("cuda").manual_seed(K + N)

    def operand(R):
        return (torch.randint(0, 256, (R, K // 2), generator=g, device="cuda", dtype=torch.uint8),
                torch.randint(126, 128, (-(-K // 256), R, 8), generator=g, device="cuda", dtype=torch.uint8))
    (a, a_scale), (w, w_scale) = operand(M), operand(N)
    bias = torch.randint(-16, 17, (N,), generator=g, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    av, wv = wide(a, a_scale), wide(w, w_scale)
    assert (av.abs() @ wv.abs().t()).max() + 16 < 2 ** 20
    y = (av @ wv.t() + bias.double()).float()
    s = dm.linear_shape(M, K, N, dtype=dtype)
    ws = dm.linear_fp4_workspace(s)
    if ws is not None:
        ws.fill_(0xFF)  # what lies in a workspace is no input: NaN
    if dtype == "fp4":
        (out, out_scale), want = buffers(M, N), quantized(y)
    else:
        out, out_scale = torch.full((M, N), 7.0, dtype=y.dtype if dtype == "f32" else torch.bfloat16, device="cuda"), None
        want = (y.to(out.dtype), None)
    for _ in range(2):
        dm.linear_fp4(s, a, a_scale, w, w_scale, out, ws, bias=bias, out_scale=out_scale)
        assert torch.equal(out, want[0])
        assert out_scale is None or torch.equal(out_scale, want[1])
        out.fill_(1)


@pytest.mark.parametrize("M", [5, 40, 400])
@pytest.mark.parametrize("ea,ew", [(0, 254), (254, 0), (1, 253), (30, 224), (254, 127), (0, 127), (127, 0), (64, 63)])
def test_scales_at_the_ends_of_their_range(M, ea, ew):
    """Powers of two of both operands whose product is in range, or past an end of it: one of 2^-127 stands for that,
    also where it meets one of 2^127.  Sums below the normal numbers may be rounded to a multiple of 2^-149 or to 0."""
    K, N = 288, 64
    c = Linear(M, K, N, dtype="f32", bias=False, seed=21)
    c.a_scale.fill_(ea), c.w_scale.fill_(ew)
    codes = [wide(x, torch.full_like(s, 127)).cpu().numpy() for x, s in ((c.a, c.a_scale), (c.w, c.w_scale))]
    p = 2.0 ** (ea + ew - 254.0)
    y, mag = codes[0] @ codes[1].T * p, abs(codes[0]) @ abs(codes[1]).T * p
    got = np64(c.run())
    big = mag >= 2.0 ** 127
    tol = (K / 8 + 40) * 2 * U24 * mag + 2.0 ** -126
    assert (abs(got - y) <= tol)[~big].all()
