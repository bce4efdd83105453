"""Streams of the record operators given as numbers: 0 (and 1) is the legacy default stream, and a call that makes several
steps makes all of them on one stream."""
import types

import numpy as np
import pytest
import torch

import paper_2608_07009_b200 as hs
from oracle import record_oracle as ro
from paper_2608_07009_b200 import hisparse


class FakeStream:
    def __init__(self, ptr, device=0):
        self.cuda_stream, self.device = ptr, types.SimpleNamespace(index=device)


@pytest.fixture
def fake_streams(monkeypatch):
    """torch's streams as it makes them, without a device: an external stream of number 0 is a new one from its pool."""
    pool = iter(range(0x7000, 0x8000, 0x10))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr, device=0: FakeStream(ptr or next(pool), device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=0: FakeStream(0, device))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: s)


def test_a_number_names_its_stream(fake_streams):
    for number, want in ((0, 0), (1, 0), (2, 2), (0x5550, 0x5550)):
        assert hisparse._Launch(number, 0).ptr == want
    assert hisparse._Launch(FakeStream(0x40), 0).ptr == 0x40
    with pytest.raises(ValueError):
        hisparse._Launch(FakeStream(0x40, device=1), 0)


def test_append_values_writes_and_appends_on_one_stream(fake_streams, monkeypatch):
    at = []
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: None)
    monkeypatch.setattr(hisparse, "write_records", lambda *a, stream, **k: at.append(hisparse._Launch(stream, 0).ptr))
    monkeypatch.setattr(hisparse.HiSparse, "append", lambda self, records, stream: at.append(hisparse._stream_ptr(stream)))
    monkeypatch.setattr(hisparse.HiSparse, "__del__", lambda self: None, raising=False)
    h = object.__new__(hisparse.HiSparse)
    h.N, h.L, h.E, h.device = 2, 1, 656, 0
    fmt = types.SimpleNamespace(entry_bytes=656, dims=576)
    for stream in (None, 0, 0x5550):
        at.clear()
        monkeypatch.setattr(hisparse._Launch, "__enter__", lambda self: self)
        monkeypatch.setattr(hisparse._Launch, "__exit__", lambda self, *e: None)
        h.append_values(fmt, torch.zeros(2, 1, 576), stream=stream)
        assert at == [stream or 0] * 2, stream


@pytest.mark.gpu
def test_stream_zero_follows_the_default_stream():
    """Values that the default stream is still making when the calls are issued, with a stream of 0 and with none."""
    rng = np.random.default_rng(3)
    dev = torch.device("cuda", 0)
    D, Dq, H, K = 144, 128, 4, 90
    fmt = hs.RecordFormat(D, Dq)
    raw = torch.from_numpy(ro.round_to_bf16(rng.standard_normal((K, D))).view(np.int16)).view(torch.bfloat16).to(dev)
    want = ro.encode(raw.float().cpu().numpy().astype(np.float64), Dq)
    q = torch.randn((1, H, D), device=dev).to(torch.bfloat16)
    table = torch.arange(K, dtype=torch.int32, device=dev)[None]
    start, kv = torch.tensor([0, 1], dtype=torch.int32, device=dev), torch.tensor([K], dtype=torch.int32, device=dev)

    def calls(x, pool, stream):
        hs.write_records(fmt, x, pool, stream=stream)
        return (hs.read_records(fmt, pool, table, stream=stream), *hs.record_attention(fmt, pool, table, q, 128, 0.1, stream=stream),
                *hs.chunk_attention(fmt, pool, table, kv, q, start, 128, 0.1, page_size=1, max_q_len=1, stream=stream))

    ref = calls(raw, torch.zeros((K, fmt.entry_bytes), dtype=torch.uint8, device=dev), None)
    torch.cuda.synchronize()
    for stream in (0, torch.cuda.default_stream().cuda_stream, None):
        x, pool = torch.zeros_like(raw), torch.zeros((K, fmt.entry_bytes), dtype=torch.uint8, device=dev)
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)
        x.copy_(raw)
        got = calls(x, pool, stream)
        x.zero_()
        torch.cuda.synchronize()
        assert np.array_equal(pool.cpu().numpy(), want)
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.gpu
def test_append_values_behind_work_of_the_default_stream():
    rng = np.random.default_rng(4)
    dev = torch.device("cuda", 0)
    N, L, B, k, D, Dq, ctx, steps = 2, 2, 16, 8, 144, 128, 20, 6
    fmt = hs.RecordFormat(D, Dq)
    hist = [hs.HostHistory(L, ctx + steps, fmt.entry_bytes) for _ in range(N)]
    gpu = hs.HiSparse(N, L, 1, B, k, fmt.entry_bytes, [ctx + steps] * N, [ctx] * N, hist)
    try:
        values = torch.from_numpy(rng.standard_normal((steps, N, L, D))).to(torch.bfloat16)
        ready, x = values.to(dev), torch.zeros((N, L, D), dtype=torch.bfloat16, device=dev)
        sel = torch.full((N, k), -1, dtype=torch.int32, device=dev)
        torch.cuda.synchronize()
        for step in range(steps):
            torch.cuda._sleep(20_000_000)
            x.copy_(ready[step])
            gpu.append_values(fmt, x, stream=None if step % 2 else 0)
            x.zero_()
            for l in range(L):
                gpu.resolve(l, sel)
        torch.cuda.synchronize()
        want = ro.encode(values.float().numpy().astype(np.float64).reshape(-1, D), Dq).reshape(steps, N, L, -1)
        for n in range(N):
            assert np.array_equal(hist[n].numpy()[:, ctx:ctx + steps], want[:, n].transpose(1, 0, 2))
        assert gpu.status() == 0
    finally:
        gpu.close()
        for h in hist:
            h.free()
