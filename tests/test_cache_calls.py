"""Calls on a cache in the order and company that a program may bring them in: after a refused one, on several streams, with
other work pending, with counts outside their range, after a drop."""
import cache_reference as ref
import numpy as np
import pytest
import torch
from test_cache_pipeline import near, values

from paper_2503_00022_amd import binding as kv
from paper_2503_00022_amd.pipeline import DecodeCache, KVCache


def decode_cache(n=100, capacity=600, Hkv=2, D=64):
    k, v = (values((1, Hkv, n, D), i).cuda() for i in range(2))
    return DecodeCache(k, v, torch.rand(1, Hkv, n).cuda(), 8, 4, capacity)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [100, 600])
def test_a_refused_attention_does_not_change_the_next(n):
    """A query of another type or on the host is turned down; the next one gets its result, whichever came first."""
    cache, q = decode_cache(n), values((1, 4, 64), 5)
    with pytest.raises(kv.KVCrushError):
        cache.attend(q.half().cuda())
    with pytest.raises(ValueError):
        cache.attend(q)
    out, lse = cache.attend(q.cuda())
    rows = [x[:, :, :n].cpu().double().numpy() for x in (cache.k, cache.v)]
    want = ref.attend(q.double().numpy()[:, :, None], *rows, [n], [1])
    near(out, want[0][:, :, 0], lse, want[1][:, :, 0], want[2][:, :, 0], torch.bfloat16)


def kv_cache(fmt, B=2, Hkv=2, D=128, capacity=4096, n=3000, unit=16, seed=1):
    c = KVCache(B, Hkv, capacity, D, format=fmt, unit=unit)
    k, v = (values((B, Hkv, n, D), seed + i).cuda() for i in range(2))
    c.append(k, v)
    return c


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["all", "chosen", "decode"])
def test_attention_on_several_streams_at_a_time(what):
    """Calls on one object only read it: on two streams with queries of their own, unordered, each has its result.  Long
    caches, so that the calls have pieces and scores in scratch memory, and many calls, so that they overlap."""
    B, Hq, D = (1, 8, 64) if what == "decode" else (2, 8, 128)
    cache = decode_cache(3000, 4096) if what == "decode" else kv_cache("i8")
    call = cache.attend if what == "decode" else lambda q: cache.attend(q, n_select=40 if what == "chosen" else 0)
    qs = [values((B, Hq, D) if what == "decode" else (B, Hq, 1, D), 70 + i).cuda() for i in range(2)]
    want = [call(q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[], []]
    for _ in range(30):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(call(qs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])


@pytest.mark.gpu
def test_a_replayed_graph_beside_eager_attention():
    cache = kv_cache("e4m3")
    qs = [values((2, 8, 2, 128), 80 + i).cuda() for i in range(2)]
    want = [cache.attend(q, n_select=s) for q in qs for s in (0, 30)]
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            captured = [cache.attend(qs[0], n_select=s) for s in (0, 30)]
    for _ in range(5):
        with torch.cuda.stream(side):
            for _ in range(4):
                graph.replay()
        eager = [[cache.attend(qs[1], n_select=s) for s in (0, 30)] for _ in range(8)]
        torch.cuda.synchronize()
        for got, expected in [(captured, want[:2])] + [(e, want[2:]) for e in eager]:
            for x, y in zip(got, expected):
                assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


@pytest.mark.gpu
def test_scratch_memory_does_not_pile_up():
    """Drafts of many lengths: nothing stays allocated behind a call but its results."""
    cache = kv_cache("i8", B=1, Hkv=8, capacity=4096, n=3000)
    cache.attend(values((1, 32, 1, 128), 1).cuda(), n_select=8)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for T in range(1, 65):
        for n_select in (0, 8):
            cache.attend(torch.zeros(1, 32, T, 128, dtype=torch.bfloat16, device="cuda"), n_select=n_select)
    assert torch.cuda.memory_allocated() == before
