"""The row types that the binding passes on: a table handle takes f32 and bf16 alone."""
import numpy as np
import pytest
import torch

from paper_2204_05436_amd import hotline as hl


@pytest.mark.parametrize("dtype", ["fp32", "F32", "", None, 1.0, "int8", torch.int8, np.float32])
def test_no_row_type(dtype):
    with pytest.raises(ValueError):
        hl.hl_create([10], 8, dtype, 4)


@pytest.mark.parametrize("dtype", ["f16", "float16", torch.float16, hl.HL_F16, 3, -1])
def test_types_that_the_library_refuses(dtype):
    """The library's own check, before it looks for a GPU."""
    with pytest.raises(hl.HotlineError) as e:
        hl.hl_create([10], 8, dtype, 4)
    assert e.value.status == 1


@pytest.mark.parametrize("dtype,want", [("f32", 0), ("bf16", 1), (hl.HL_F32, 0), (hl.HL_BF16, 1), (np.int32(0), 0),
                                        (np.int64(1), 1), (torch.float32, 0), (torch.bfloat16, 1), ("bfloat16", 1)])
def test_row_types(dtype, want, monkeypatch):
    got = []

    class Lib:
        @staticmethod
        def hl_create(out, n, rows, dim, dt, cap):
            got.append(dt)
            return 3

    monkeypatch.setattr(hl, "lib", lambda: Lib)
    with pytest.raises(hl.HotlineError):
        hl.hl_create([10], 8, dtype, 4)
    assert got == [want]
