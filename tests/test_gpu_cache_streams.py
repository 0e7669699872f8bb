"""Rotation, append and attention on a stream that is not the current one, with buffers that the calls allocate."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


@pytest.mark.parametrize("call", ["rope", "kv_append", "packed_append", "packed_attn"])
def test_buffers_are_of_the_streams_memory(C, call, monkeypatch):
    hq, hkv, d, ps, n = 8, 2, 64, 16, 3000
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, n, hq + 2 * hkv, d), generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
    table = torch.arange(-(-n // ps), dtype=torch.int32)[None]
    rope, pos = C.Rope(C.rope_table(100.0, d, n), [0] * (d // 2)), torch.arange(n, dtype=torch.int32, device="cuda")[None]
    seqs = C.Seqs([0, n], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    one = C.Seqs([0, 1], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    pool = torch.zeros((1, table.numel(), hkv, ps, d), dtype=torch.bfloat16, device="cuda")
    plain = C.KvCache(pool, pool.clone(), hq, ps, table)
    packed = C.PackedKv.empty(1, table.numel(), hq, hkv, d, ps, table)
    C.conduit_packed_append(packed, seqs, k, v)
    run = {
        "rope": lambda **kw: C.conduit_rope(rope, q, pos, **kw),
        "kv_append": lambda **kw: C.conduit_kv_append(plain, seqs, k, v, rope, pos, q, **kw),
        "packed_append": lambda **kw: C.conduit_packed_append(packed, seqs, k, v, rope, pos, q, **kw),
        "packed_attn": lambda **kw: C.conduit_packed_attn(packed, one, q[:, -1:], **kw),
    }[call]
    want = run()
    torch.cuda.synchronize()
    streams, empty = [], torch.empty

    def watched(*args, **kw):
        streams.append(torch.cuda.current_stream())
        return empty(*args, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    monkeypatch.setattr(torch, "empty", watched)
    got = run(stream=side)
    monkeypatch.undo()
    assert len(streams) == (2 if call == "packed_attn" else 1) and all(s == side for s in streams)
    side.synchronize()
    assert torch.equal(got, want)
