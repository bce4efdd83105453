"""Arguments of the record operators that need no device: strides of 0."""
import ctypes

from test_record_oracle import problem


def test_one_table_row_for_all_requests():
    from paper_2608_07009_b200 import hisparse as hs
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    call = hs.lib().hisparse_record_attention_workspace_bytes
    assert call(problem(hs), n) == hs.OK
    assert call(problem(hs, table_stride=0), m) == hs.OK and m.value == n.value
    for stride in (1, 9, -1, -10):
        assert call(problem(hs, table_stride=stride), n) == hs.EINVAL
