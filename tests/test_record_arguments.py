"""Arguments of the record operators that need no device: strides of 0, numbers beyond 32 bits."""
import ctypes

import pytest

from test_record_oracle import problem


def test_one_table_row_for_all_requests():
    from paper_2608_07009_b200 import hisparse as hs
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    call = hs.lib().hisparse_record_attention_workspace_bytes
    assert call(problem(hs), n) == hs.OK
    assert call(problem(hs, table_stride=0), m) == hs.OK and m.value == n.value
    for stride in (1, 9, -1, -10):
        assert call(problem(hs, table_stride=stride), n) == hs.EINVAL


def test_formats_beyond_32_bits():
    from paper_2608_07009_b200 import hisparse as hs
    for dims, quant in (((1 << 32) + 576, 512), (576, (1 << 32) + 512), (576 - (1 << 32), 512), (1 << 31, 0)):
        with pytest.raises(hs.HiSparseError) as e:
            hs.RecordFormat(dims, quant)
        assert e.value.code == hs.EINVAL
