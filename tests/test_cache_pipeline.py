"""The classes that generate with a cache: DecodeCache.attend and KVCache against the plain references, step by step."""
import cache_reference as ref
import numpy as np
import pytest
import torch

from paper_2503_00022_amd import binding as kv
from paper_2503_00022_amd.pipeline import DecodeCache, KVCache


def values(shape, seed, dtype=torch.bfloat16):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype)


def near(got, want, lse, want_lse, absolute, dtype):
    """One rounding of the result; probabilities of 16 bits at least, fp32 sums of some hundred terms, logits of some tens:
    2^-14 of the sum of magnitudes; log-sum-exps as their logits, 2^-24 x 2 sqrt(128) x 40 + 2^-20."""
    half = torch.finfo(dtype).eps / 2
    far = np.abs(got.cpu().double().numpy() - want)
    assert (far <= half * np.abs(want) + 2.0 ** -14 * absolute).all(), far.max()
    assert (np.abs(lse.cpu().double().numpy() - want_lse) <= 1e-4).all()


@pytest.mark.gpu
@pytest.mark.parametrize("reduce_groups,Hq,Hkv,D", [(True, 8, 2, 128), (False, 4, 4, 64)])
def test_decode_cache_attends_through_evictions(reduce_groups, Hq, Hkv, D):
    B, budget, capacity = 2, 64, 80
    k, v = (values((B, Hkv, budget, D), i).cuda() for i in range(2))
    scores = torch.rand(B, Hkv if reduce_groups else Hq, budget, generator=torch.Generator().manual_seed(1)).cuda()
    cache = DecodeCache(k, v, scores, budget, 48, capacity, reduce_groups=reduce_groups)
    for step in range(50):
        q, kn, vn = (values((B, H, D), 100 * step + i).cuda() for i, H in enumerate((Hq, Hkv, Hkv)))
        n = cache.append(q, kn, vn)
        out, lse = cache.attend(q)
        assert out.shape == q.shape and lse.shape == q.shape[:2]
        if step % 7 and step not in (15, 16, 17, 49):
            continue
        want = ref.attend(q.cpu().double().numpy()[:, :, None], cache.k[:, :, :n].cpu().double().numpy(),
                          cache.v[:, :, :n].cpu().double().numpy(), [n] * B, [1] * B)
        near(out, want[0][:, :, 0], lse, want[1][:, :, 0], want[2][:, :, 0], torch.bfloat16)
    assert cache.evictions == 3


@pytest.mark.gpu
def test_decode_cache_refuses_other_queries():
    k = values((1, 2, 8, 64), 1).cuda()
    cache = DecodeCache(k, k, torch.rand(1, 2, 8).cuda(), 8, 4, 16)
    with pytest.raises(ValueError):
        cache.attend(torch.zeros(1, 4, 1, 64, device="cuda"))
    with pytest.raises(kv.KVCrushError):
        cache.attend(torch.zeros(1, 4, 64, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        cache.attend(torch.zeros(1, 4, 64, dtype=torch.bfloat16))


class Follower:
    """What a KVCache should hold, in 64 bits."""

    def __init__(self, B, Hkv, capacity, D, fmt):
        self.rows = {w: np.zeros((B, Hkv, capacity, D)) for w in "kv"}
        self.fmt, self.lengths = fmt, [0] * B

    def append(self, k, v, n_new):
        for b, n in enumerate(n_new):
            L = self.lengths[b]
            for w, x in (("k", k), ("v", v)):
                part = x[b, :, :n].float().numpy()
                codes, par = (part, None) if self.fmt is None else ref.quantise(part, self.fmt)
                self.rows[w][b, :, L:L + n] = ref.values64(codes, par, self.fmt)
            self.lengths[b] += n


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [None, "e4m3", "i8", "i4"])
@pytest.mark.parametrize("block_size", [0, 16])
def test_drafting_with_a_kv_cache(fmt, block_size):
    """A prompt, then rounds of drafts of which some are dropped again; attention over everything and over chosen blocks."""
    B, Hq, Hkv, D, capacity, unit = 2, 8, 2, 64, 256, 8
    table, n_blocks = None, 0
    if block_size:
        n_blocks = B * capacity // block_size + 5
        table = torch.from_numpy(np.random.RandomState(1).permutation(n_blocks)[:B * capacity // block_size].astype(np.int32))
        table = table.view(B, -1).cuda()
    c = KVCache(B, Hkv, capacity, D, format=fmt, block_size=block_size, block_table=table, n_blocks=n_blocks, unit=unit)
    f = Follower(B, Hkv, capacity, D, fmt)
    rng = np.random.RandomState(5)
    for step, T in enumerate([90, 1, 5, 1, 7, 5, 33]):
        k, v = (values((B, Hkv, T, D), 10 * step + i) for i in range(2))
        n_new = [T, T] if step in (0, 1) else [T, max(1, T - 2)]
        counts = None if n_new == [T, T] else torch.tensor(n_new, dtype=torch.int32, device="cuda")
        c.append(k.cuda(), v.cuda(), n_new=counts)
        f.append(k, v, n_new)
        assert c.lengths.tolist() == f.lengths and c.cache.S >= max(f.lengths)
        q = values((B, Hq, T, D), 10 * step + 5)
        seen = np.stack([ref.tree(T, rng) for _ in range(B)])
        mask = ref.mask_words(seen).cuda() if step % 2 == 0 else None
        out, lse = c.attend(q.cuda(), mask=mask, n_new=counts)
        want = ref.attend(q.double().numpy(), f.rows["k"], f.rows["v"], f.lengths, n_new, seen if step % 2 == 0 else None)
        live = np.isfinite(want[1])
        near(out, want[0], torch.where(torch.from_numpy(live), lse.cpu(), 0.0), np.where(live, want[1], 0), want[2], torch.bfloat16)
        assert (lse.cpu().numpy()[~live] == -np.inf).all()
        # over chosen blocks: all of them when there are as many places
        every = c.attend(q.cuda(), mask=mask, n_new=counts, n_select=capacity // unit)
        near(every[0], want[0], torch.where(torch.from_numpy(live), every[1].cpu(), 0.0), np.where(live, want[1], 0), want[2],
             torch.bfloat16)
        few = c.attend(q.cuda(), mask=mask, n_new=counts, n_select=4, n_recent=2)
        assert torch.isfinite(few[0]).all() and (few[1].cpu()[torch.from_numpy(live)] <= lse.cpu()[torch.from_numpy(live)] + 1e-4).all()
        rows = c.read(n=max(f.lengths), dtype=torch.float32 if fmt else None)
        for w, got in zip("kv", rows):
            for b in range(B):
                have = f.rows[w][b, :, :f.lengths[b]]
                assert (np.abs(got[b, :, :f.lengths[b]].cpu().double().numpy() - have) <= 2.0 ** -23 * (np.abs(have) + 8)).all()
        if T in (5, 7):                                        # two drafts of each sequence are not kept
            c.drop(2)
            f.lengths = [x - 2 for x in f.lengths]


@pytest.mark.gpu
def test_a_captured_step_of_a_kv_cache():
    """append and attend captured once, replayed for several tokens with eager work between: the eager cache's results."""
    B, Hq, Hkv, D = 2, 8, 2, 128
    made = [KVCache(B, Hkv, 512, D, format="i8", block_size=16, unit=16) for _ in range(2)]
    prompt = values((B, Hkv, 300, D), 1).cuda()
    k, q = torch.empty(B, Hkv, 1, D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, Hq, 1, D, dtype=torch.bfloat16, device="cuda")

    def step(c):
        c.append(k, k)
        return (*c.attend(q), *c.attend(q, n_select=6))

    k.copy_(values(k.shape, 2)), q.copy_(values(q.shape, 3))
    for c in made:
        c.append(prompt, prompt)
        step(c)
    torch.cuda.synchronize()
    made[0].bound = made[0].cache.S = 400                       # what the replays will need
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = step(made[0])
    made[1].bound = made[1].cache.S = 400
    for i in range(4):
        k.copy_(values(k.shape, 20 + i)), q.copy_(values(q.shape, 40 + i))
        graph.replay()
        torch.cuda.synchronize()
        made[1].bound = 400
        want = step(made[1])
        torch.cuda.synchronize()
        assert torch.equal(made[0].lengths, made[1].lengths) and made[0].lengths.tolist() == [302 + i] * 2
        for a, b in zip(got, want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
def test_a_refused_append_leaves_the_cache():
    c = KVCache(1, 2, 32, 64)
    good = values((1, 2, 3, 64), 1).cuda()
    c.append(good, good)
    with pytest.raises(ValueError):
        c.append(good, good[:, :1])
    with pytest.raises(kv.KVCrushError):
        c.append(good.half(), good.half())                      # a plain cache takes its own type
    with pytest.raises(ValueError, match="capacity"):
        c.append(values((1, 2, 30, 64), 2).cuda(), values((1, 2, 30, 64), 2).cuda())
    assert c.lengths.tolist() == [3] and c.bound == 3 and c.cache.S == 3
    with pytest.raises(ValueError, match="unit"):
        c.attend(values((1, 2, 1, 64), 1).cuda(), n_select=2)


@pytest.mark.gpu
def test_lengths_and_their_bound():
    """A bound that is set counts for every call; a drop of more than there is empties; a refused count changes nothing."""
    c = KVCache(2, 2, 64, 64)
    x = values((2, 2, 20, 64), 1).cuda()
    c.append(x, x)
    c.bound = 8
    assert c.read()[0].shape[2] == 8 and torch.equal(c.read()[0], x[:, :, :8])
    c.bound = 20
    with pytest.raises(RuntimeError):
        c.append(x, x, n_new=torch.ones(3, dtype=torch.int32, device="cuda"))
    assert c.bound == 20 and c.lengths.tolist() == [20, 20]
    with pytest.raises(ValueError, match="negative"):
        c.drop(-1)
    c.drop(torch.tensor([30, 4], dtype=torch.int32, device="cuda"))
    assert c.lengths.tolist() == [0, 16] and c.bound == 20
    c.append(x[:, :, :3], x[:, :, :3])
    assert c.lengths.tolist() == [3, 19] and c.bound == 23
    k = c.read()[0]
    assert torch.equal(k[0, :, :3], x[0, :, :3]) and torch.equal(k[1, :, :19], torch.cat([x[1, :, :16], x[1, :, :3]], 1))
    assert not k[0, :, 3:].any() and not k[1, :, 19:].any()
    c.drop(40)
    assert c.lengths.tolist() == [0, 0] and c.bound == 0
    out, lse = c.attend(values((2, 4, 1, 64), 2).cuda())
    assert not out.any() and (lse == -float("inf")).all()


@pytest.mark.gpu
def test_a_backward_pass_notices_an_append():
    c = KVCache(1, 2, 16, 64)
    x = values((1, 2, 3, 64), 1).cuda()
    c.append(x, x)
    w = torch.ones_like(c.k, requires_grad=True)
    y = (w * c.k).sum()
    c.append(x, x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_arguments_that_do_not_fit():
    with pytest.raises(ValueError, match="format"):
        KVCache(1, 1, 32, 64, format="fp4", device="cpu")
    with pytest.raises(ValueError, match="block_size"):
        KVCache(1, 1, 30, 64, block_size=16, device="cpu")
    with pytest.raises(ValueError, match="block_size"):
        KVCache(1, 1, 32, 64, block_table=torch.zeros(1, 2, dtype=torch.int32), device="cpu")
    with pytest.raises(ValueError, match="GPU memory"):
        KVCache(1, 1, 32, 64, device="cpu")
