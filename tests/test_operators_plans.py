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
