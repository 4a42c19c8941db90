"""CPU tests of the operators' launch plans, which are host code of the library."""
import ctypes

import pytest

import paper_2605_25550_amd as dm


@pytest.fixture(scope="module")
def segments():
    fn = dm.lib()._ZN5ditmi11qk_segmentsEiiiii
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.c_int] * 5
    return fn


def chunks(dh, H, Hk, Hv):
    lanes = dh // 8
    per = 7 if lanes == 9 else 64 // (1 << (lanes - 1).bit_length())
    return sum(-(-n // per) for n in (H, Hk, Hv))


@pytest.mark.parametrize("dh", [8, 64, 72, 128, 136, 256])
@pytest.mark.parametrize("H,Hk,Hv", [(1, 0, 0), (24, 24, 0), (24, 8, 8), (38, 0, 0), (1280, 0, 0), (0, 65535, 65535), (65535, 65535, 65535)])
def test_queries_and_keys_fit_a_grid(segments, dh, H, Hk, Hv):
    """Every accepted call's grid has fewer than 2^32 threads (four waves of 64 a workgroup), a segment for each row
    at least, and none without a chunk."""
    for rows in (1, 3, 4095, 17550, 2 ** 20 - 1, 2 ** 22 + 1, 2 ** 23 + 3, 2 ** 24 - 1, 2 ** 24):
        s = segments(rows, dh, H, Hk, Hv)
        assert 1 <= s <= chunks(dh, H, Hk, Hv), (rows, s)
        assert -(-rows * s // 4) * 256 < 2 ** 32, (rows, s)


# ---------------------------------------------------------------- 4-bit linear layers
class Plan4(ctypes.Structure):
    _fields_ = [("tile", ctypes.c_int), ("split", ctypes.c_int), ("bytes", ctypes.c_size_t)]


@pytest.fixture(scope="module")
def plan4():
    fn = dm.lib()._ZN5ditmi15linear_fp4_planEiiii
    fn.restype, fn.argtypes = Plan4, [ctypes.c_int] * 4
    return fn


# slots of each tile's ring (of the kernels of few rows: panels that four waves hold)
RING = {256: 2, 193: 2, 192: 3, 128: 2, 65: 3, 64: 4, 32: 4, 2: 8, 1: 8}
# (rows, in, out, tile, ranges of k): every tile's loop in its steady state, behind it its last stages and a panel in
# part, for odd and even numbers of panels; and ranges of k of unequal lengths
LOOPS = [(8000, 1120, 3456, 256, 1), (8000, 1440, 3456, 256, 1), (2100, 1120, 4416, 193, 1), (2100, 1440, 4416, 193, 1),
         (4000, 2080, 1056, 192, 1), (904, 1312, 5824, 192, 1), (2100, 1376, 3456, 128, 1), (2100, 1120, 3456, 128, 1),
         (700, 1120, 3456, 65, 1), (700, 1376, 3456, 65, 1), (1000, 2080, 2048, 64, 1), (1000, 1824, 2048, 64, 1),
         (6922, 1696, 32, 64, 1), (4112, 1696, 32, 32, 1), (4112, 1888, 32, 32, 1), (4112, 2144, 32, 32, 1),
         (300, 4640, 1152, 2, 1), (130, 8224, 1152, 1, 1), (1957, 58656, 1536, 256, 5), (1798, 56000, 1696, 193, 3),
         (1110, 32320, 1184, 192, 4), (1023, 56448, 1312, 128, 5), (1097, 27072, 608, 65, 4), (4130, 9888, 32, 64, 4),
         (66, 17504, 5824, 32, 3)]


@pytest.mark.parametrize("dtype", [0, 1, 3])
@pytest.mark.parametrize("M,K,N,tile,split", LOOPS)
def test_shapes_take_the_tiles_that_they_test(plan4, dtype, M, K, N, tile, split):
    p = plan4(M, N, K, dtype)
    assert (p.tile, p.split) == (tile, split)
    assert -(-K // 256) // split > RING[tile] + 1 and K % 256
    assert p.bytes == (split * M * N * 4 if split > 1 else 0)


def test_every_tile_is_tested():
    assert {c[3] for c in LOOPS} == set(RING)
    assert {c[3] for c in LOOPS if c[4] > 1} == {t for t in RING if t > 2}  # (the others divide no k)
    for t in RING:
        if t > 2:  # both parities
            assert {-(-c[1] // 256) % 2 for c in LOOPS if c[3] == t and c[4] == 1} == {0, 1}, t
