"""Scores and values at the ends of their types, for each kernel of the
masked attention, against the 64-bit definitions of operator_refs.py."""
import pytest
import torch

from test_operators_gpu import Attn

pytestmark = pytest.mark.gpu

# (type, query heads, key heads, queries, keys, room) of a call that the kernel takes
KERNELS = {"rows": ("bf16", 24, 24, [600, 333], [600, 333], 0),        # 256-row workgroups: whole and masked tiles
           "ranges": ("bf16", 24, 3, [700, 5], [6000, 900], 6000),     # ... that divide the keys
           "few": ("bf16", 4, 2, [150, 3], [150, 90], 200),            # 32-row workgroups
           "tokens": ("bf16", 4, 2, [1, 2], [2000, 700], 2000),        # ... that divide the keys
           "f32": ("f32", 6, 2, [150, 3], [150, 90], 200)}


def call(kernel, dh, **kw):
    dtype, H, Hk, ql, kl, room = KERNELS[kernel]
    return Attn(dtype, H, Hk, dh, ql, kl, room=room, fused=False, seed=dh, **kw)


@pytest.mark.parametrize("bias", [False, True], ids=["cap", "cap+bias"])
@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("kernel", KERNELS)
def test_capped_scores_of_infinite_products(kernel, dh, bias):
    """cap * tanh(-inf / cap) is -cap, a score like any other, wherever its key
    lies: in tiles that every row sees whole, on the diagonal, in the last."""
    a = call(kernel, dh, mask="causal", cap=1.0, bias=bias)
    a.q[:, :, 0] = 1.0
    a.k[:, :, 0] = 0.0
    # the definition's infinities: tanh(-40) is -1 within 2^-113
    far = float(torch.tensor(40 * dh ** 0.5, dtype=a.k.dtype))
    finite = a.k.clone()
    for d, n in enumerate(a.kl):
        rows, fin = a.k[a.k0[d]:a.k0[d] + n], finite[a.k0[d]:a.k0[d] + n]
        for at, sign in ((slice(0, 1), -1), (slice(3, None, 7), -1), (slice(5, None, 31), 1), (slice(n - 1, n), -1)):
            rows[at, :, 0], fin[at, :, 0] = sign * float("inf"), sign * far
    a.run()
    a.k = finite
    a.check()


@pytest.mark.parametrize("rise", [15, 40, 63])
@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("kernel", KERNELS)
def test_large_values_under_rising_scores(kernel, dh, rise):
    """Scores that rise by a factor of 2^rise from tile to tile, values of some
    2^100: their number times the largest is below 2^127, so that every result is
    finite, whichever maximum the probabilities are taken relative to."""
    a = call(kernel, dh, mask="causal")
    a.q[:, :, 0] = 1.0
    for d, n in enumerate(a.kl):
        a.k[a.k0[d]:a.k0[d] + n, :, 0] = (torch.arange(n, device="cuda") // 64 * (rise * dh ** 0.5 / 1.4427))[:, None]
    a.v.mul_(2.0 ** 100)
    a.run()
    assert a.o.isfinite().all()
    a.check()
