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


@pytest.mark.gpu
def test_what_a_call_on_another_stream_makes_is_not_in_use():
    """Work is pending on the current stream that still writes tensors which are free already; results and scratch memory of
    calls on another stream, whose sizes fit, must not be there."""
    B, Hq, Hkv, S, D = 2, 8, 2, 1024, 128
    q, k, v = (values((B, H, S, D), i).cuda() for i, H in enumerate((Hq, Hkv, Hkv)))
    new, scores0 = q[:, :, -1].contiguous(), torch.rand(B, Hkv, S, device="cuda")
    table = torch.arange(B * S // 16, dtype=torch.int32, device="cuda").view(B, -1)
    cache = kv.make_cache(k, v, S)
    bnd = kv.kvcrush_block_bounds(cache, 16)
    idx, *_ = kv.kvcrush_select(scores0, 512, 256, unit=16)

    def calls(stream, running):
        scores, _ = kv.kvcrush_scores(q, k, True, stream=stream)
        yield scores
        yield kv.kvcrush_row_lse(q, k, stream=stream)
        yield kv.kvcrush_pool_scores(scores0, 7, stream=stream)
        yield from kv.kvcrush_select(scores0, 512, 256, want_bits=True, stream=stream)
        yield from kv.kvcrush_compact(k, v, idx, validate=False, stream=stream)
        yield kv.kvcrush_compact_block_table(idx, table, 16, stream=stream)
        yield kv.kvcrush_scores_append(new, k, running, S, True, stream=stream)
        yield from kv.kvcrush_cache_read(cache, stream=stream)
        yield from kv.kvcrush_cache_read(cache, idx=idx, stream=stream)
        yield from kv.kvcrush_block_bounds(cache, 16, stream=stream)
        blocks = kv.kvcrush_block_select(cache, q[:, :, -4:], *bnd, 16, 20, stream=stream)
        yield blocks
        yield from kv.kvcrush_attend(cache, q[:, :, -4:], stream=stream)
        yield from kv.kvcrush_attend(cache, q[:, :, -4:], blocks=blocks, unit=16, stream=stream)

    want = [x.clone() for x in calls(None, scores0.clone())]
    torch.cuda.synchronize()
    running, side, a = scores0.clone(), torch.cuda.Stream(), torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    a @ a
    torch.cuda.synchronize()
    sizes = sorted({x.nbytes for x in want} | {16 << i for i in range(21)})
    filled = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    for _ in range(20):                                        # some 20 ms
        a @ a
    for x in filled:
        x.fill_(0xAB)
    filled = x = None
    got = list(calls(side, running))
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.gpu
def test_what_autograd_follows_is_refused_in_both_directions():
    """Tangents, outputs that require a gradient, a cache that came to be followed by what was copied into it."""
    from torch.autograd import forward_ad
    c = kv_cache(None, B=1, n=40, capacity=64)
    q, k = values((1, 4, 1, 128), 1).cuda(), values((1, 2, 1, 128), 2).cuda()
    lse, rows = torch.empty(1, 4, 1, device="cuda"), torch.empty(1, 2, 40, 128, dtype=torch.bfloat16, device="cuda")
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: c.attend(dual(q)), lambda: c.attend(dual(q), n_select=2), lambda: c.append(dual(k), k),
                     lambda: c.append(k, dual(k)), lambda: kv.kvcrush_attend(c.cache, q, lse=dual(lse)),
                     lambda: kv.kvcrush_attend(c.cache, q, out=dual(q)), lambda: kv.make_cache(dual(c.k), c.v, 40),
                     lambda: kv.kvcrush_cache_read(c.cache, n=40, k_out=dual(rows)), lambda: kv.make_cache(c.k, dual(c.v), 40)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        assert c.lengths.tolist() == [40] and c.bound == 40
        c.attend(q)                                            # (nothing is dual: as ever)
    for call in (lambda: kv.kvcrush_attend(c.cache, q, lse=lse.requires_grad_()),
                 lambda: kv.kvcrush_cache_read(c.cache, n=40, v_out=rows.requires_grad_()),
                 lambda: kv.kvcrush_block_bounds(c.cache, 16, c.bounds, c.bound_scales.detach().requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):
            call()
    d = decode_cache()
    d.attend(values((1, 4, 64), 1).cuda())
    with torch.no_grad():
        d.append(values((1, 4, 64), 1).cuda(), *(values((1, 2, 64), 2).cuda().requires_grad_() for _ in range(2)))
        d.attend(values((1, 4, 64), 1).cuda())
    d.append(values((1, 4, 64), 1).cuda(), *(values((1, 2, 64), 2).cuda().requires_grad_() for _ in range(2)))
    with pytest.raises(ValueError, match="gradient"):
        d.attend(values((1, 4, 64), 1).cuda())
    with torch.no_grad():
        out, _ = d.attend(values((1, 4, 64), 1).cuda())
    assert torch.isfinite(out).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [None, "i8"])
def test_counts_outside_their_range_count_as_its_ends(fmt):
    """More tokens than were given are as many as were given, less than none are none: lengths never pass what is written."""
    made = [kv_cache(fmt, B=3, n=20, capacity=64, unit=8) for _ in range(2)]
    k = values((3, 2, 4, 128), 9).cuda()
    counts = lambda *n: torch.tensor(n, dtype=torch.int32, device="cuda")  # noqa: E731
    for step in range(2):
        made[0].append(k, k, n_new=counts(7 + step, -3, 2 ** 31 - 1 - step))
        made[1].append(k, k, n_new=counts(4, 0, 4))
    given = counts(2, -5, -2 ** 31)
    made[0].drop(given)
    made[1].drop(counts(2, 0, 0))
    assert given.tolist() == [2, -5, -2 ** 31] and made[0].lengths.tolist() == made[1].lengths.tolist() == [26, 20, 28]
    q = values((3, 4, 1, 128), 3).cuda()
    for n_select in (0, 2):
        for x, y in zip(*(c.attend(q, n_select=n_select) for c in made)):
            assert torch.equal(x, y)
    with pytest.raises(ValueError):                            # a refused append takes back what it counted, no more
        made[0].append(k, k[:, :1], n_new=counts(9, -9, 1))
    assert made[0].lengths.tolist() == [26, 20, 28]


@pytest.mark.gpu
def test_a_drop_refreshes_the_bounds_of_the_last_block():
    """Taken back tokens have no say in which blocks are chosen, also before the next append."""
    B, Hkv, D, unit = 2, 2, 64, 8
    made = [KVCache(B, Hkv, 128, D, unit=unit) for _ in range(2)]
    k = values((B, Hkv, 60, D), 1).cuda()
    k[:, :, 43:] *= 50                                         # (blocks 5 to 7: what is dropped would win every choice)
    for c, n in zip(made, (60, 43)):
        c.append(k[:, :, :n], k[:, :, :n])
    made[0].drop(10)
    made[0].drop(torch.tensor([7, 7], dtype=torch.int32, device="cuda"))
    live = -(-43 // unit)
    assert torch.equal(made[0].bounds[:, :, :live], made[1].bounds[:, :, :live])
    assert torch.equal(made[0].bound_scales[:, :, :live], made[1].bound_scales[:, :, :live])
    q = values((B, 4, 1, D), 3).cuda()
    for x, y in zip(*(c.attend(q, n_select=2, n_sink=0, n_recent=0) for c in made)):
        assert torch.equal(x, y)
    made[0].drop(100)                                          # (nothing is left: no block to refresh)
    assert made[0].lengths.tolist() == [0, 0]


def test_caches_that_no_call_would_take_are_refused_at_once():
    """Before anything is allocated: no GPU is needed."""
    table = torch.zeros(1, 2, dtype=torch.int32)
    for change, match in ((dict(D=96), "64 or 128"), (dict(format="i8", dtype=torch.float32), "bfloat16 or float16"),
                          (dict(unit=1025), "unit"), (dict(unit=-1), "unit"), (dict(block_size=16, block_table=table), "n_blocks"),
                          (dict(block_size=8, block_table=table, n_blocks=9), "block_table")):
        with pytest.raises(ValueError, match=match):
            KVCache(1, 1, 32, **dict(dict(D=64, device="cpu"), **change))


@pytest.mark.gpu
def test_single_precision_rows_of_a_quantised_cache():
    c = KVCache(1, 2, 32, 64, format="i8")
    k = values((1, 2, 20, 64), 1, torch.float32).cuda()
    c.append(k, k)
    codes, par = ref.quantise(k.cpu().numpy(), "i8")
    assert torch.equal(c.read(dtype=torch.float32)[0].cpu(), torch.from_numpy(ref.values32(codes, par, "i8")))
    assert c.attend(values((1, 4, 1, 64), 2).cuda())[0].dtype == torch.bfloat16


@pytest.mark.gpu
def test_lists_without_entries_are_refused():
    c = kv_cache(None, n=40, capacity=64)
    q = values((2, 4, 1, 128), 1).cuda()
    with pytest.raises(ValueError, match="one entry"):
        kv.kvcrush_attend(c.cache, q, blocks=torch.empty(2, 2, 1, 0, dtype=torch.int32, device="cuda"), unit=16)
    out, lse = kv.kvcrush_attend(c.cache, q, blocks=torch.full((2, 2, 1, 1), -1, dtype=torch.int32, device="cuda"), unit=16)
    assert not out.any() and (lse == -float("inf")).all()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["k_param", "v_param"])
def test_a_backward_pass_notices_an_append_to_a_quantised_cache(name):
    c = KVCache(1, 2, 16, 64, format="i8")
    x = values((1, 2, 3, 64), 1).cuda()
    c.append(x, x)
    t = getattr(c, name)
    y = (torch.ones_like(t, requires_grad=True) * t).sum()
    c.append(x, x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.gpu
def test_a_drop_takes_any_whole_number():
    c = kv_cache(None, n=40, capacity=64)
    c.drop(np.int64(3))
    assert c.lengths.tolist() == [37, 37] and c.bound == 37
    with pytest.raises(TypeError):
        c.drop(2.5)
    with pytest.raises(ValueError, match="negative"):
        c.drop(np.int32(-1))
    assert c.lengths.tolist() == [37, 37] and c.bound == 37


@pytest.mark.gpu
@pytest.mark.parametrize("unit", [0, 8])
def test_a_block_table_wider_than_the_capacity(unit):
    table = torch.tensor([[3, 0, 5], [1, 4, 2]], dtype=torch.int32, device="cuda")
    c, plain = KVCache(2, 2, 32, 64, block_size=16, block_table=table, n_blocks=6, unit=unit), KVCache(2, 2, 32, 64, unit=unit)
    k, q = values((2, 2, 30, 64), 1).cuda(), values((2, 4, 1, 64), 2).cuda()
    for x in (c, plain):
        x.append(k, k)
    for n_select in {0, unit and 3}:
        for x, y in zip(*(m.attend(q, n_select=n_select) for m in (c, plain))):
            assert torch.equal(x, y)
    with pytest.raises(ValueError, match="capacity"):
        c.append(k, k)
