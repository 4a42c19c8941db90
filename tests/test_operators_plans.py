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


def plan4(M, K, N, dtype=1):
    fn = dm.lib()._ZN5ditmi15linear_fp4_planEiiii
    fn.restype, fn.argtypes = Plan4, [ctypes.c_int] * 4
    return fn(M, N, K, dtype)


def loops():
    """(rows, in, out, tile, ranges of k): for every kernel that the plan picks, whole k and divided, and for odd and even
    numbers of panels, the smallest and the largest product of these whose workgroups take seven panels of 256 k at least (the kernels of few
    rows, whose four waves share them, 33), the last one in part: their loops are in the steady state, rings are filled again
    and run empty."""
    found = {}
    for M in (66, 130, 300, 700, 904, 1023, 1110, 1957, 2100, 4000, 4130, 6922, 8000):
        for K in (1632, 1888, 2080, 3168, 8224, 8480, 9888, 17504, 18400, 27072, 32320, 56448, 58656):
            for N in (32, 320, 608, 1056, 1152, 1312, 1536, 2048, 3456, 4416, 5824):
                p, panels = plan4(M, K, N), -(-K // 256)
                if panels // p.split < (33 if p.tile <= 2 else 7) or (M + N) * K > 2.2e8 or M * K * N > 2e11:
                    continue
                found.setdefault((p.tile, p.split > 1, panels % 2), []).append((M * K * N, (M, K, N, p.tile, p.split)))
    return sorted({pick(found[k])[1] for k in found for pick in (min, max)}, key=lambda c: c[3:] + c[:3])


LOOPS = loops()


def test_every_kernel_is_among_them():
    """Whatever the plan picks for ordinary products is one that the loops' tests run, divided too where it divides."""
    picked = set()
    for M in (1, 8, 16, 33, 77, 200, 300, 600, 1000, 1997, 4096, 8192, 17550):
        for K in (96, 1152, 4608, 8192, 18432):
            for N in (1, 96, 384, 1152, 3456, 4608, 9216):
                for dtype in (0, 1, 3):
                    p = plan4(M, K, -(-N // 32) * 32 if dtype == 3 else N, dtype)
                    picked.add((p.tile, p.split > 1))
                    assert p.bytes == (p.split * M * ((-(-N // 32) * 32 if dtype == 3 else N) + 7 & ~7) * 4 if p.split > 1 else 0)
    tested = {(tile, split > 1) for _, _, _, tile, split in LOOPS}
    assert picked <= tested, picked - tested
    for tile, divided in tested:
        if not divided:
            assert {-(-K // 256) % 2 for _, K, _, t, s in LOOPS if t == tile and s == 1} == {0, 1}, tile
