"""The record operators at the edges of what they are given: pools without records, tables that requests share, batches without
requests, tensors whose strides along an axis of one mean nothing, contexts near 2^31 keys, errors in the handle's status word."""
import numpy as np
import pytest
import torch

import paper_2608_07009_b200 as hs
from oracle import record_oracle as ro
from paper_2608_07009_b200 import hisparse
from test_gpu_records import DEV, bf16, check, chunk_case, numbers, pool_of, run_chunk

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------ pools without records

# the kernel of single tokens over codes, the one of few rows in both formats, pairs on pages, pairs on records laid out once
PATHS = [(1, 128, 1, 8), (1, 128, 64, 8), (1, 0, 1, 8), (1, 0, 64, 8), (3, 128, 16, 8), (3, 0, 16, 8), (20, 0, 64, 8), (30, 128, 16, 8), (30, 0, 7, 8)]


@pytest.mark.parametrize("m,Dq,page,H", PATHS)
@pytest.mark.parametrize("address", [False, True])
def test_attention_over_an_empty_pool(m, Dq, page, H, address):
    """Nothing is read, not even where the address has NaN records behind it."""
    fmt, D, Dv, K = hs.RecordFormat(144, Dq), 144, 128, 150
    pool = torch.full((400, fmt.entry_bytes), 0x7F, dtype=torch.uint8, device=DEV)
    ptr = pool.data_ptr() if address else pool[:0].clone().data_ptr()
    q, table = torch.randn((2 * m, H, D), device=DEV).to(torch.bfloat16), torch.full((2, -(-K // page)), -1, dtype=torch.int32, device=DEV)
    status = i32([0])
    args = lambda: (fmt, ptr, 0, 0, table, q, Dv, 0.1, page, i32([0, m, 2 * m]), i32([K, 9]), m, K, 1, None, None, None, status, None)  # noqa: E731
    for entries, want in ((None, 0), (torch.arange(table.shape[1], dtype=torch.int32, device=DEV), hs.STATUS_OUT_OF_RANGE)):
        if entries is not None:
            table[0] = entries
        out, lse = hisparse._attend(*args())
        assert torch.all(out == 0) and torch.all(torch.isneginf(lse)) and status.item() == want


def test_writing_and_reading_an_empty_pool():
    fmt = hs.RecordFormat(144, 128)
    pool = torch.empty((0, fmt.entry_bytes), dtype=torch.uint8, device=DEV)
    x, status = torch.randn((3, 144), device=DEV).to(torch.bfloat16), i32([0])
    slots = torch.tensor([-1, -1, -1], device=DEV)
    hs.write_records(fmt, x, pool, slots=slots, status=status)
    assert torch.all(hs.read_records(fmt, pool, i32([[-1, -1]]), status=status) == 0) and status.item() == 0
    assert torch.all(hs.read_records(fmt, pool, i32([[-1, 0]]), status=status) == 0) and status.item() == hs.STATUS_OUT_OF_RANGE
    status.zero_()
    slots[1] = 0
    hs.write_records(fmt, x, pool, slots=slots, status=status)
    assert status.item() == hs.STATUS_OUT_OF_RANGE
    out, lse = hs.record_attention(fmt, pool, torch.full((2, 5), -1, dtype=torch.int32, device=DEV), x[:2, None].expand(2, 4, 144), 128, 1.0)
    assert torch.all(out == 0) and torch.all(torch.isneginf(lse))


# ------------------------------------------------------------------------------------------ the handle's status word

def test_errors_over_a_handles_cache_reach_its_status():
    N, L, B, k, D = 2, 2, 16, 8, 144
    fmt = hs.RecordFormat(D, 128)
    hist = [hs.HostHistory(L, 40, fmt.entry_bytes) for _ in range(N)]
    gpu = hs.HiSparse(N, L, 1, B, k, fmt.entry_bytes, [40] * N, [30] * N, hist)
    try:
        q, rows = torch.randn((N, 4, D), device=DEV).to(torch.bfloat16), N * (B + 1)
        table = torch.arange(N * k, dtype=torch.int32, device=DEV).reshape(N, k)
        gpu.gather_values(1, fmt, table)
        gpu.record_attention(1, fmt, q, table, 128, 0.1)
        assert gpu.status() == 0
        for beyond in (rows, 2147483647):
            table[1, 3] = beyond
            assert torch.all(gpu.gather_values(1, fmt, table)[1, 3] == 0)
            assert gpu.status() == hs.STATUS_OUT_OF_RANGE
            gpu.clear_status()
            gpu.record_attention(1, fmt, q, table, 128, 0.1)
            assert gpu.status() == hs.STATUS_OUT_OF_RANGE
            gpu.clear_status()
    finally:
        gpu.close()
        for h in hist:
            h.free()


# ------------------------------------------------------------------------------------------ contexts near 2^31 keys

@pytest.mark.parametrize("m,H,Dq", [(1, 4, 0), (2, 3, 128), (20, 4, 0)])
def test_the_longest_context_that_is_taken(m, H, Dq):
    """2^31 - 1024 keys of which a few pages are there, the last one among them: the last split ends at its context's end."""
    rng = np.random.default_rng(m)
    D, page = 128, 1024
    width = 2 ** 21 - 1
    raw, num = pool_of(rng, 3 * page, D, Dq)
    table = torch.full((1, width), -1, dtype=torch.int32, device=DEV)
    for at, p in ((0, 2), (1234567, 0), (width - 1, 1)):
        table[0, at] = p
    K = width * page
    q = ro.bf16_values(ro.round_to_bf16(rng.standard_normal((m, H, D))))
    out, lse = hs.chunk_attention(hs.RecordFormat(D, Dq), torch.from_numpy(raw).to(DEV), table, i32([K]), bf16(q).to(DEV), i32([0, m]), 128, 0.1,
                                  page_size=page, max_q_len=m)
    keys = np.concatenate([num[2 * page:], num[:page], num[page:2 * page]])
    ref = [ro.attention(keys, np.arange(3 * page) < 3 * page - m + t + 1, q[t], 128, 0.1) for t in range(m)]
    check(out, lse, np.stack([r[0] for r in ref]), np.stack([r[1] for r in ref]), q, num, 0.1, D)


# ------------------------------------------------------------------------------------------ strides

@pytest.mark.parametrize("Dq", [0, 128])
@pytest.mark.parametrize("m", [1, 2, 30])
def test_requests_that_share_a_table_row(m, Dq):
    rng = np.random.default_rng(m + Dq)
    D, N, page, K = 144, 3, 16, 100
    raw, num, table, cs, q, q_start = chunk_case(rng, [m] * N, [K] * N, 8, D, Dq, page)
    row = torch.from_numpy(table[:1]).to(DEV)
    args = (hs.RecordFormat(D, Dq), torch.from_numpy(raw).to(DEV))
    rest = (i32([K] * N), bf16(q).to(DEV), torch.from_numpy(q_start).to(DEV), 128, 0.1)
    out, lse = hs.chunk_attention(*args, row.expand(N, -1), *rest, page_size=page, max_q_len=m)
    out_ref, lse_ref, _ = ro.chunk(num, np.repeat(table[:1], N, 0), cs, q, q_start, 128, 0.1, page)
    check(out[:-2], lse[:-2], out_ref[:-2], lse_ref[:-2], q, num, 0.1, D)


def test_axes_of_one_with_any_stride():
    rng = np.random.default_rng(1)
    D, K = 144, 40
    raw, num = pool_of(rng, K, D, 128)
    pool, table = torch.from_numpy(raw).to(DEV), torch.arange(K, dtype=torch.int32, device=DEV)[None]
    q = ro.bf16_values(ro.round_to_bf16(rng.standard_normal((1, 1, D))))
    ref = ro.attention(num, np.ones(K, bool), q[0], 128, 0.1)
    flat = bf16(q).to(DEV).reshape(-1)
    for strides in ((3, 5, 1), (D, 1, 1), (1001, 7, 1)):
        out, lse = hs.record_attention(hs.RecordFormat(D, 128), pool, table, flat.as_strided((1, 1, D), strides), 128, 0.1)
        check(out, lse, ref[0][None], ref[1][None], q, num, 0.1, D)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_row_written_to_many_slots(dtype):
    fmt = hs.RecordFormat(576, 512)
    row = torch.randn((1, 576), device=DEV).to(dtype)
    pool = torch.zeros((20, fmt.entry_bytes), dtype=torch.uint8, device=DEV)
    slots = torch.tensor([3, 0, -1, 19, 7], device=DEV)
    hs.write_records(fmt, row.expand(5, 576), pool, slots=slots)
    want = np.zeros((20, fmt.entry_bytes), dtype=np.uint8)
    want[[3, 0, 19, 7]] = ro.encode(row.double().cpu().numpy(), 512)
    assert np.array_equal(pool.cpu().numpy(), want)


# ------------------------------------------------------------------------------------------ batches without requests

def test_no_requests():
    fmt = hs.RecordFormat(144, 128)
    pool = torch.zeros((8, fmt.entry_bytes), dtype=torch.uint8, device=DEV)
    none = torch.zeros((0, 5), dtype=torch.int32, device=DEV)
    q = torch.zeros((3, 4, 144), dtype=torch.bfloat16, device=DEV)
    out, lse = hs.record_attention(fmt, pool, none, q[:0], 128, 1.0)
    assert out.shape == (0, 4, 128) and out.dtype == torch.bfloat16 and lse.shape == (0, 4) and lse.dtype == torch.float32
    mine = torch.full((3, 4, 128), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((3, 4), 7.0, device=DEV)
    got = hs.chunk_attention(fmt, pool, none, i32([]), q, i32([0]), 128, 1.0, page_size=1, max_q_len=1, out=mine[0], lse=mine[1])
    assert got[0] is mine[0] and got[1] is mine[1] and torch.all(mine[0] == 7) and torch.all(mine[1] == 7)
    assert hs.chunk_attention(fmt, pool, none, i32([]), q, i32([0]), 128, 1.0, page_size=1, max_q_len=1)[0].shape == (3, 4, 128)
    with pytest.raises(hs.HiSparseError):                           # a row a request, and no request for the rows
        hs.record_attention(fmt, pool, none, q, 128, 1.0)


# ------------------------------------------------------------------------------------------ numbers beyond 32 bits

def test_sizes_beyond_32_bits_are_refused():
    """They used to be cut to their low 32 bits: 2^32 + 1 tokens became 1."""
    fmt = hs.RecordFormat(144, 128)
    pool = torch.zeros((64, fmt.entry_bytes), dtype=torch.uint8, device=DEV)
    q = torch.zeros((2, 16, 144), dtype=torch.bfloat16, device=DEV)
    sizes = dict(value_dims=128, page_size=4, max_q_len=1, max_kv_len=8)
    for name in sizes:
        for more in (1 << 32, -(1 << 32)):
            args = dict(sizes, **{name: sizes[name] + more})
            with pytest.raises(hs.HiSparseError) as e:
                hs.chunk_attention(fmt, pool, i32([[0, 1], [2, 3]]), i32([8, 8]), q, i32([0, 1, 2]), args.pop("value_dims"), 1.0, **args)
            assert e.value.code == hisparse.EINVAL
