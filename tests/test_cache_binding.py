"""l2a.cache: tensors that are not what they would be taken for are refused."""
import pytest
import torch

from paper_2603_17484_b200 import l2a


def pools(dtype):
    return torch.zeros((3, 2, 16, 64), dtype=dtype)


E = torch.zeros((3, 2, 16), dtype=torch.uint8)
TABLE, LENGTHS = torch.zeros((4, 3), dtype=torch.int32), torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float8_e5m2, torch.int8, torch.bool, torch.float16, torch.int16])
def test_other_types_are_no_codes(dtype):
    for scales in ((E, E), (None, None)):
        with pytest.raises(ValueError):
            l2a.cache(pools(dtype), pools(dtype), TABLE, LENGTHS, *scales)


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.uint8])
def test_types_of_codes(dtype):
    assert l2a.cache(pools(dtype), pools(dtype), TABLE, LENGTHS, E, E).kind == l2a.CACHE_E4M3


def test_bf16_values_have_no_exponents():
    x = pools(torch.bfloat16)
    for scales in ((E, None), (None, E), (E, E)):
        with pytest.raises(ValueError):
            l2a.cache(x, x, TABLE, LENGTHS, *scales)


def test_lengths_and_rows_of_the_table_are_dense():
    x = pools(torch.bfloat16)
    wide = torch.zeros((4, 6), dtype=torch.int32)
    assert l2a.cache(x, x, wide[:, :3], LENGTHS).table_stride == 6          # rows may be further apart
    assert l2a.cache(x, x, wide[:1, ::6], wide[:1, 0]).table_stride == 1    # one entry, one length
    for table, lengths in ((wide[:, ::2], LENGTHS), (TABLE, wide[:, 0]), (TABLE, torch.zeros(8, dtype=torch.int32)[::2]),
                           (TABLE[0], LENGTHS[:1]), (TABLE, LENGTHS[:, None])):
        with pytest.raises(ValueError):
            l2a.cache(x, x, table, lengths)
