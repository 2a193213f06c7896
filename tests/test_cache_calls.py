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
