"""CPU tests of the compiled calls: what does not fit is left to the checks in Python (None), never called."""
import ctypes

import pytest
import torch

import paper_2605_25550_amd as dm


@pytest.fixture(scope="module")
def calls():
    dm.lib()
    if dm._CALLS is None:
        pytest.skip("the compiled calls are not built")
    return dm._CALLS


@pytest.mark.parametrize("name,n", [("linear_fp4", 9), ("quantize_fp4", 3), ("dequantize_fp4", 3), ("qk_norm_rope", 13)])
def test_what_does_not_fit(calls, name, n):
    x = torch.zeros(4, 64)
    s = dm.linear_shape(4, 64, 64) if name == "linear_fp4" else dm.QkShape(4, 2, 2, 32, 4, 4, 0, 2, 0, 0)
    fn = getattr(calls, name)
    for args in ([], [None] * n, [x] * n, [s] + [x] * (n - 1), [s] + [None] * (n - 1), [s] * n, [s] + [x] * n, [1] * n,
                 [bytes(s)] + [x] * (n - 1), [x.to("meta")] * n, [s] + [x.to("meta")] * (n - 1),
                 [torch.nn.Buffer(x) if hasattr(torch.nn, "Buffer") else x] * n, [x.to_sparse()] * n):
        assert fn(*args) is None


def test_structures(calls):
    """The sizes that the compiled calls read are the binding's."""
    assert ctypes.sizeof(dm.LinearShape) == 20 and ctypes.sizeof(dm.QkShape) == 160
    with pytest.raises(TypeError):
        calls.bind(1)
    with pytest.raises(TypeError):
        calls.bind(dm.LinearShape, dm.QkShape, "a", "b", "c", "d")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp4"])
def test_errors_are_the_bindings_own(calls, dtype):
    u = torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensor"):
        dm.linear_fp4(dm.linear_shape(2, 64, 64, dtype=dtype), u, u, u, u, u)
    with pytest.raises(ValueError, match="device tensor"):
        dm.quantize_fp4(torch.zeros(2, 64), u, u)
    with pytest.raises(ValueError, match="device tensor"):
        dm.dequantize_fp4(u, u, torch.zeros(2, 64))
