"""Attention over a cache where weights and values differ by many orders: a key that takes nearly all of the softmax and
contributes nothing, V rows of very different size, infinities, NaN and values near their type's largest."""
import math

import cache_reference as ref
import numpy as np
import pytest
import torch
from test_cache_use import check_attention, q_type, values

from paper_2503_00022_amd import binding as kv

pytestmark = pytest.mark.gpu

# rows of a KV head that decide how the work is laid out: 4, 20 and 36 to 160 of them
ROWS = [(8, 2, 1), (40, 2, 1), (8, 2, 12), (8, 2, 40)]


def made(fmt, k, v, block_size=0):
    """A case whose rows are these (float32 [B,Hkv,L,D])."""
    B, Hkv, L, D = k.shape
    c = ref.Case(fmt, B, Hkv, [L] * B, D, block_size=block_size, seed=1)
    for w, x in (("k", k), ("v", v)):
        if fmt in ref.DTYPES:
            t, par = torch.from_numpy(x).to(ref.DTYPES[fmt]), None
            c.rows64[w] = t.double().numpy()
        else:
            codes, par = ref.quantise(x, fmt)
            t, c.rows64[w] = ref.store(codes, fmt), ref.values64(codes, par, fmt)
        for name, x in ((w, t), (w + "_param", None if par is None else torch.from_numpy(par))):
            if x is None:
                continue
            if block_size:       # the pool's other rows stay what no call may read
                raw = c.tensors[name].view(torch.uint8) if x.dtype == torch.float8_e4m3fn else c.tensors[name]
                x = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
                for b in range(B):
                    for i, blk in enumerate(c.table[b].tolist()):
                        part = x[b, :, i * block_size:(i + 1) * block_size].movedim(0, 1)
                        raw[blk, :len(part)] = part
            else:
                c.tensors[name] = x
    return c.cuda()


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("orders", [12, 17, 22, 26])
@pytest.mark.parametrize("L,D,block_size,rows", [(3000, 128, 0, ROWS[0]), (3000, 64, 16, ROWS[1]), (700, 128, 16, ROWS[2]), (500, 128, 0, ROWS[3])])
def test_many_small_weights_beside_a_large_one(fmt, orders, L, D, block_size, rows):
    """One key `orders` binary orders above all others, with V = 0; the others alike, so that no error averages out."""
    Hq, Hkv, T = rows
    rng = np.random.RandomState(orders)
    k, v = np.zeros((1, Hkv, L, D), dtype=np.float32), np.empty((1, Hkv, L, D), dtype=np.float32)
    v[:] = (rng.uniform(32, 64, (1, Hkv, 1, D)) * rng.choice([-1, 1], (1, Hkv, 1, D))).astype(np.float32)
    at = [0, L // 3][orders % 2]
    k[:, :, at], v[:, :, at] = orders * math.log(2) / math.sqrt(D), 0.0
    c = made(fmt, k, v, block_size)
    q = torch.ones(1, Hq, T, D).to(ref.DTYPES[q_type(fmt, "f16")])
    check_attention(c, q, kv.kvcrush_attend(c.make(kv), q.cuda()), [T])


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("orders", [15, 20, 40])
@pytest.mark.parametrize("rows", ROWS)
def test_one_large_row_that_hardly_counts(fmt, orders, rows):
    """A V row 2^orders times the others whose probability is e^-45 of theirs."""
    Hq, Hkv, T = rows
    D, L, rng = 128, 400, np.random.RandomState(orders)
    orders = min(orders, 15) if fmt == "f16" else orders
    k = (0.2 * rng.randn(1, Hkv, L, D)).astype(np.float32)
    v = rng.uniform(0.5, 1.0, (1, Hkv, L, D)).astype(np.float32)
    for at in (5, L - T - 1):
        k[:, :, at], v[:, :, at] = -45 / math.sqrt(D), v[:, :, at] * 2.0 ** orders
    c = made(fmt, k, v)
    q = torch.ones(1, Hq, T, D).to(ref.DTYPES[q_type(fmt, "f16")])
    check_attention(c, q, kv.kvcrush_attend(c.make(kv), q.cuda()), [T])


def near_or_alike(c, q, got, n_new, seen=None):
    """check_attention where the formula's results are finite, and its infinities and NaN elsewhere."""
    out = got[0].cpu().double().numpy()
    with np.errstate(invalid="ignore"):
        want = ref.attend(q.double().numpy(), c.rows64["k"], c.rows64["v"], c.lengths, n_new, seen)[0]
    odd = ~np.isfinite(want)
    assert odd.any() and np.array_equal(out[odd], want[odd], equal_nan=True)
    rows = {w: c.rows64[w].copy() for w in "kv"}
    plain = np.isfinite(c.rows64["v"])
    c.rows64["v"] = np.where(plain, c.rows64["v"], 0.0)          # (values of other columns than those that are compared)
    out[odd] = ref.attend(q.double().numpy(), c.rows64["k"], c.rows64["v"], c.lengths, n_new, seen)[0][odd]
    check_attention(c, q, (torch.from_numpy(out), got[1]), n_new, seen)
    c.rows64 = rows


@pytest.mark.parametrize("fmt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("block_size", [0, 16])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("L,D,orders", [(150, 128, 0), (150, 64, 5), (2500, 128, 130)])
def test_infinities_and_nan_reach_the_rows_that_see_them(fmt, block_size, rows, L, D, orders):
    """In old keys (all rows see them) and in drafts (some do): infinities of both signs, NaN, at keys of ordinary weight
    (orders = 0) and far below the largest."""
    Hq, Hkv, T = rows
    rng = np.random.RandomState(L + T)
    k, v = (rng.randn(1, Hkv, L, D).astype(np.float32) for _ in range(2))
    bad = [3, L // 2, L - 1] + ([L - T + 1] if T > 2 else [])
    k[:, :, bad[:2]] = -orders * math.log(2) / math.sqrt(D)
    v[:, :, bad[0], 3], v[:, :, bad[0], 7], v[:, :, bad[1], 7] = math.inf, -math.inf, -math.inf
    v[:, :, bad[1], 9], v[:, :, bad[0], 11], v[:, :, bad[1], 11] = math.nan, math.inf, -math.inf
    v[:, :, bad[2], 13] = math.inf
    if T > 2:
        v[:, :, bad[3], 15], v[:, 0, bad[3], 17] = -math.inf, math.nan
    seen = ref.tree(T, rng, roots=0.5)[None]
    c = made(fmt, k, v, block_size)
    q = torch.ones(1, Hq, T, D).to(ref.DTYPES[fmt])
    got = kv.kvcrush_attend(c.make(kv), q.cuda(), mask=ref.mask_words(seen).cuda())
    near_or_alike(c, q, got, [T], seen)


@pytest.mark.parametrize("fmt", ["e4m3", "i8", "i4"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("which", ["k", "v", "old"])
def test_rows_of_nan_reach_the_rows_that_see_them(fmt, rows, which):
    """A quantised row with a value that was not finite is NaN throughout, and so is what sees it, whole."""
    Hq, Hkv, T = rows
    L, D, rng = 200, 128, np.random.RandomState(T)
    k, v = (rng.randn(1, Hkv, L, D).astype(np.float32) for _ in range(2))
    at = 40 if which == "old" else L - T // 2 - 1
    (k if which == "k" else v)[:, -1, at, 5] = math.inf
    c = made(fmt, k, v)
    seen = ref.tree(T, rng, roots=0.5)[None]
    q = values((1, Hq, T, D), "bf16", 3)
    out, lse = kv.kvcrush_attend(c.make(kv), q.cuda(), mask=ref.mask_words(seen).cuda())
    sees = np.ones(T, dtype=bool) if which == "old" else seen[0, :, at - (L - T)]
    hit = np.zeros((Hq, T), dtype=bool)
    hit[Hq - Hq // Hkv:] = sees
    assert np.array_equal(torch.isnan(out[0]).cpu().numpy(), np.broadcast_to(hit[..., None], (Hq, T, D)))
    assert np.array_equal(torch.isnan(lse[0]).cpu().numpy(), hit if which == "k" else np.zeros_like(hit))
    hurt = c.rows64["v"][:, -1, at].copy(), c.rows64["k"][:, -1, at].copy()
    c.rows64["v"][:, -1, at] = c.rows64["k"][:, -1, at] = 0
    want = ref.attend(q.double().numpy(), c.rows64["k"], c.rows64["v"], [L], [T], seen)
    c.rows64["v"][:, -1, at], c.rows64["k"][:, -1, at] = hurt
    # (the rows that do not see it: one rounding, probabilities and logits as in check_attention, some tens of them)
    far = np.abs(out[0].cpu().double().numpy() - want[0][0])[~hit]
    assert (far <= 2.0 ** -8 * np.abs(want[0][0][~hit]) + 2.0 ** -14 * want[2][0][~hit]).all()


@pytest.mark.parametrize("fmt", ["bf16", "f16", "f32", "e4m3", "i8"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("L,lengths", [(90, False), (2500, False), (2500, True)])
def test_values_near_the_largest(fmt, rows, L, lengths):
    """Columns of one large value, of its negative and of both in turn, beside small ones."""
    Hq, Hkv, T = rows
    D, rng = 64, np.random.RandomState(L)
    top = 0.99 * torch.finfo(ref.DTYPES[fmt]).max if fmt in ref.DTYPES else 2.0 ** 127
    k = (0.1 * rng.randn(2, Hkv, L, D)).astype(np.float32)
    v = rng.randn(2, Hkv, L, D).astype(np.float32)
    v[..., 0], v[..., 1] = top, -top
    v[..., ::2, 2], v[..., 1::2, 2] = top, -top
    v[:, :, 5, 3] = top
    c = made(fmt, k, v)
    q = torch.ones(2, Hq, T, D).to(ref.DTYPES[q_type(fmt)])
    check_attention(c, q, kv.kvcrush_attend(c.make(kv, use_lengths=lengths), q.cuda()), [T, T])


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("level", [2.0 ** 40, -1e30, 2.0 ** 127])
def test_rows_without_a_range(rows, level):
    """4-bit rows of one value each: no scale, all of it in the lowest value."""
    Hq, Hkv, T = rows
    D, L, rng = 128, 300, np.random.RandomState(3)
    k = (0.1 * rng.randn(1, Hkv, L, D)).astype(np.float32)
    v = np.broadcast_to(np.float32(level) * rng.uniform(0.5, 1, (1, Hkv, L, 1)).astype(np.float32), k.shape).copy()
    c = made("i4", k, v)
    q = torch.ones(1, Hq, T, D).bfloat16()
    check_attention(c, q, kv.kvcrush_attend(c.make(kv), q.cuda()), [T])


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("T,lengths,Hq,Hkv,kind", [(1024, [1100], 2, 1, "tree"), (300, [300, 900], 4, 2, "chain"), (513, [800], 3, 3, "tree")])
def test_many_new_tokens(fmt, T, lengths, Hq, Hkv, kind):
    """Up to as many as a call takes: masks of several words, tiles of nothing but new tokens."""
    B, D = len(lengths), 64
    c = ref.Case(fmt, B, Hkv, lengths, D, block_size=16, seed=T).cuda()
    q, rng = values((B, Hq, T, D), q_type(fmt), 4), np.random.RandomState(T)
    seen = np.stack([ref.tree(T, rng) for _ in range(B)]) if kind == "tree" else None
    got = kv.kvcrush_attend(c.make(kv), q.cuda(), mask=None if seen is None else ref.mask_words(seen).cuda())
    check_attention(c, q, got, [min(T, n) for n in lengths], seen)


@pytest.mark.parametrize("fmt", ["bf16", "f16", "f32", "e4m3", "i8", "i4"])
@pytest.mark.parametrize("Hq,Hkv,T", [(8, 2, 3), (40, 2, 1)])
def test_infinities_in_chosen_and_other_blocks(fmt, Hq, Hkv, T):
    """Lists of blocks, lengths and counts on the device: the first token, in no list, is NaN; a chosen block holds an infinity
    (quantised: a row of NaN), which those rows that have it in their list see."""
    B, D, unit, lengths = 2, 64, 8, [300, 77]
    rng = np.random.RandomState(5)
    k, v = (rng.randn(B, Hkv, 300, D).astype(np.float32) for _ in range(2))
    v[:, :, 0] = math.nan
    v[:, 0, 3 * unit + 2, 5] = math.inf
    c = made(fmt, k, v, 16)
    c.lengths = lengths
    lists = [[[[3, 5, 9] if t % 2 else [2, 4, 7] for t in range(T)] if g == 0 else [[1, 6, 8]] * T for g in range(Hkv)] for _ in range(B)]
    q = values((B, Hq, T, D), q_type(fmt), 9)
    n_new = [T, max(T - 1, 1)]
    cache = c.make(kv)
    got = kv.kvcrush_attend(cache, q.cuda(), blocks=torch.tensor(lists, dtype=torch.int32).cuda(), unit=unit,
                            n_new=torch.tensor(n_new, dtype=torch.int32, device="cuda"))
    c.rows64["v"] = np.where(np.isfinite(c.rows64["v"]), c.rows64["v"], 0.0)
    out = got[0].cpu().double().numpy()
    want = ref.attend(q.double().numpy(), c.rows64["k"], c.rows64["v"], lengths, n_new, None, None, lists, unit)[0]
    for b in range(B):
        for t in range(1, n_new[b], 2):                        # (those that have block 3)
            hit = out[b, :Hq // Hkv, t]
            assert (hit[:, 5] == math.inf).all() if fmt in ref.DTYPES else np.isnan(hit).all()
            at = 5 if fmt in ref.DTYPES else slice(None)
            out[b, :Hq // Hkv, t, at] = want[b, :Hq // Hkv, t, at]
    check_attention(c, q, (torch.from_numpy(out), got[1]), n_new, lists=lists, unit=unit)


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("L", [50, 2500])
def test_logits_far_below_zero(fmt, rows, L):
    """All of a row's logits are about -10^33 but for one of half that: it is all of the softmax, not a row that sees nothing."""
    Hq, Hkv, T = rows
    D, rng = 64, np.random.RandomState(L)
    big = 6e4 if fmt == "f16" else 2.0 ** 56
    k, v = np.full((1, Hkv, L, D), -big, dtype=np.float32), rng.randn(1, Hkv, L, D).astype(np.float32)
    k[:, :, L // 3] = -big / 2
    c = made(fmt, k, v)
    q = torch.full((1, Hq, T, D), 2.0 ** 15 if fmt == "f16" else 2.0 ** 53).to(ref.DTYPES[q_type(fmt)])
    out, lse = kv.kvcrush_attend(c.make(kv), q.cuda())
    want = ref.attend(q.double().numpy(), c.rows64["k"], c.rows64["v"], [L], [T])
    # (other keys' weights are 0 in any arithmetic; lse: the logit's own rounding, D products and their sum)
    half = torch.finfo(q.dtype).eps / 2
    assert (np.abs(out.cpu().double().numpy() - want[0]) <= (half + 2.0 ** -16) * np.abs(want[0]) + 2.0 ** -17 * np.abs(c.rows64["v"]).max()).all()
    assert (np.abs(lse.cpu().double().numpy() / want[1] - 1) <= 2.0 ** -18).all()


@pytest.mark.parametrize("fmt", ["bf16", "f32", "e4m3", "i8", "i4"])
@pytest.mark.parametrize("rows", ROWS[1:3])
@pytest.mark.parametrize("orders,scale", [(118, None), (-118, None), (60, 2.0 ** -110), (57, 2.0 ** -114)])
def test_queries_and_keys_of_opposite_sizes(fmt, rows, orders, scale):
    """Tiny queries and huge keys, the other way round, and huge ones of both with a tiny scale: ordinary logits."""
    Hq, Hkv, T = rows
    D, L, rng = 64, 300, np.random.RandomState(3)
    k = (rng.randn(1, Hkv, L, D) * 2.0 ** orders).astype(np.float32)
    v = rng.randn(1, Hkv, L, D).astype(np.float32)
    if scale is None and orders < 0 and fmt in ("e4m3", "i8", "i4"):
        k *= 2.0 ** 25                                         # (rows below 2^-100 are stored as zero)
    c = made(fmt, k, v)
    small = -orders if scale is None else -orders - math.log2(scale) - 3
    q = (torch.from_numpy(rng.randn(1, Hq, T, D)) * 2.0 ** small).to(ref.DTYPES[q_type(fmt)])
    check_attention(c, q, kv.kvcrush_attend(c.make(kv), q.cuda(), scale=scale or 0.0), [T], scale=scale)


@pytest.mark.parametrize("fmt", ["e4m3", "i8", "i4"])
@pytest.mark.parametrize("rows", ROWS)
def test_small_codes_beside_a_large_one(fmt, rows):
    """Each row of K has one value that makes its scale and that no query looks at; the logits are those of its smallest codes."""
    Hq, Hkv, T = rows
    D, L, rng = 128, 300, np.random.RandomState(4)
    top = {"e4m3": 448.0, "i8": 127.0, "i4": 15.0}[fmt]
    step = 2.0 ** -9 if fmt == "e4m3" else 1.0
    k = (rng.randint(0, 8, (1, Hkv, L, D)) * step).astype(np.float32)
    k[..., 0], k[..., 1] = top, 0.0
    v = (rng.randint(0, 8, (1, Hkv, L, D)) * step).astype(np.float32)
    v[..., 0], v[..., 1] = top, 0.0
    c = made(fmt, k, v)
    assert np.array_equal(c.rows64["k"], k) and np.array_equal(c.rows64["v"], v)
    q = values((1, Hq, T, D), "bf16", 8, 0.3 / step)
    q[..., 0] = 0
    check_attention(c, q, kv.kvcrush_attend(c.make(kv), q.cuda()), [T])
