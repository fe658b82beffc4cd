"""fs_quantise_rows writes e4m3 codes: tensors whose bytes mean something else are refused (no GPU needed)."""

import pytest
import torch

from test_mm_refusals import Rows, binding, tensors  # noqa: F401 (a fixture)


@pytest.mark.parametrize("dtype", [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.int8, torch.bool])
def test_bytes_of_another_meaning(binding, dtype):  # noqa: F811
    x, scale = tensors().x, Rows((3,), torch.float32)
    with pytest.raises(ValueError, match="not float8_e4m3fn or uint8"):
        binding.fs_quantise_rows(x, Rows((3, 20), dtype), scale)


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.uint8])
def test_codes(binding, dtype):  # noqa: F811
    with pytest.raises(AssertionError, match="the library was called"):
        binding.fs_quantise_rows(tensors().x, Rows((3, 20), dtype), Rows((3,), torch.float32))
