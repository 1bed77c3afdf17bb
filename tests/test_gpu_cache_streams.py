"""Calls of the key/value cache's operators on the default stream, from a program whose current stream is another."""

import pytest

pytestmark = pytest.mark.gpu


def test_memory_of_a_call_on_the_default_stream_is_the_default_streams(monkeypatch):
    import torch
    import paper_2511_23113_amd as dbsp
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()      # noqa: E731
    q, k, v, pk, pv = rand(3, 4, 2, 64), rand(3, 2, 300, 64), rand(3, 2, 300, 64), rand(2, 900, 64), rand(2, 900, 64)
    lens = torch.tensor([300, 7, 120], dtype=torch.int32, device="cuda")
    cache = dbsp.KVCache(k, v, lens, pk, pv)
    want = dbsp.cache_attn_fwd(cache, q)
    evicted = [dbsp.KVCache(k.clone(), v.clone(), lens.clone(), weights=torch.arange(1800, device="cuda").view(3, 2, 300).float(),
                            positions=torch.arange(300, device="cuda", dtype=torch.int32).repeat(3, 2, 1)) for _ in range(3)]
    dbsp.cache_evict(evicted[0], 100)
    torch.cuda.synchronize()
    entered, enter = [], torch.cuda.stream
    monkeypatch.setattr(torch.cuda, "stream", lambda s: (entered.append(s.cuda_stream), enter(s))[1])
    with enter(torch.cuda.Stream()):
        for i, stream in enumerate((torch.cuda.default_stream(), 0)):
            got = dbsp.cache_attn_fwd(cache, q, stream=stream)
            dbsp.cache_evict(evicted[1 + i], 100, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            for name in ("k", "v", "lens", "weights", "positions"):
                assert torch.equal(getattr(evicted[1 + i], name), getattr(evicted[0], name))
    assert entered == [0] * 8              # o, lse and a workspace, and the eviction's; twice
