"""The calls that use a KV cache against plain references: rows written and read back (equal to the last bit), attention
of new tokens, 8-bit block bounds and the choice of blocks (equal), attention over chosen blocks, and all of them together."""
import math

import cache_reference as ref
import numpy as np
import pytest
import torch

from paper_2503_00022_amd import binding as kv

pytestmark = pytest.mark.gpu


def values(shape, dtype, seed, magnitude=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * magnitude).to(ref.DTYPES[dtype])


def bits(t):
    return t.contiguous().view(torch.uint8)


def same(a, b):
    """Equal, NaN to NaN."""
    a, b = a.cpu(), b.cpu()
    return a.dtype == b.dtype and torch.equal(torch.nan_to_num(a.float(), nan=1e30), torch.nan_to_num(b.float(), nan=1e30))


# ------------------------------------------------------------------------------------------------ rows
@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("src", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,Hkv,lengths,T,D,block_size", [
    (1, 1, [1], 1, 64, 0), (2, 3, [5, 17], 1, 128, 0), (3, 2, [70, 33, 64], 33, 128, 16), (2, 2, [40, 3], 7, 64, 10),
    (1, 2, [300], 300, 128, 32), (2, 1, [130, 129], 129, 64, 0)])
def test_rows_are_written_and_read_back(fmt, src, B, Hkv, lengths, T, D, block_size):
    if fmt in ref.DTYPES and src != fmt:
        pytest.skip("a plain cache takes its own type")
    c = ref.Case(fmt, B, Hkv, lengths, D, block_size=block_size, seed=T, room=9).cuda()
    before = {w: c.dense(w) for w in c.tensors}
    cache = c.make(kv)
    new = {w: values((B, Hkv, T, D), src, 7 + i, 3.0) for i, w in enumerate("kv")}
    new["k"][0, 0, 0] = 0                                       # a row of zeros
    new["v"][-1, -1, -1] = 2.5                                  # a row without a range
    kv.kvcrush_cache_write(cache, new["k"].cuda(), new["v"].cuda())
    got = dict(zip("kv", kv.kvcrush_cache_read(cache, n=c.capacity, dtype=ref.DTYPES[src])))
    for w in "kv":
        stored, par = c.dense(w), c.dense(w + "_param")
        for b in range(B):
            n = min(T, lengths[b])
            at = slice(lengths[b] - n, lengths[b])
            x = new[w][b, :, :n].float().numpy()
            codes, p = (x, None) if fmt in ref.DTYPES else ref.quantise(x, fmt)
            assert torch.equal(bits(stored[b, :, at]), bits(ref.store(codes, fmt)))
            if p is not None:
                assert torch.equal(par[b, :, at], torch.from_numpy(p))
            # every other row is what it was
            rest = [i for i in range(c.capacity) if not at.start <= i < at.stop]
            assert torch.equal(bits(stored[b, :, rest]), bits(before[w][b, :, rest]))
            old = ref.load(stored[b], fmt)[:, :lengths[b]]
            want = torch.from_numpy(ref.values32(old, None if par is None else par[b, :, :lengths[b]].numpy(), fmt))
            assert same(got[w][b, :, :lengths[b]], want.to(ref.DTYPES[src]))
            assert (got[w][b, :, lengths[b]:] == 0).all()


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("block_size", [0, 16])
def test_chosen_rows_and_rows_a_sequence_does_not_have(fmt, block_size):
    lengths = [90, 0, 41]
    c = ref.Case(fmt, 3, 2, lengths, 128, block_size=block_size, seed=3).cuda()
    cache = c.make(kv)
    dt = torch.float32 if fmt not in ("bf16", "f16") else ref.DTYPES[fmt]
    idx = torch.tensor([[0, 5, 5, 89, 89], [0, 1, 2, 3, 4], [40, 3, -7, 41, 10 ** 6]], dtype=torch.int32)
    k_out, v_out = (torch.full((3, 2, 5, 128), 7.0, dtype=dt, device="cuda") for _ in range(2))
    kv.kvcrush_cache_read(cache, idx=idx.cuda(), k_out=k_out, v_out=v_out)
    for w, got in (("k", k_out), ("v", v_out)):
        rows = ref.values32(ref.load(c.dense(w), fmt), None if fmt in ref.DTYPES else c.dense(w + "_param").numpy(), fmt)
        for b in (0, 2):
            at = idx[b].clamp(0, lengths[b] - 1).numpy()
            assert same(got[b], torch.from_numpy(rows[b][:, at]).to(dt))
        assert (got[1] == 7).all()                              # an empty sequence has no rows
    n = 60
    k_out.resize_(3, 2, n, 128).fill_(7.0), v_out.resize_(3, 2, n, 128).fill_(7.0)
    kv.kvcrush_cache_read(cache, n=n, k_out=k_out, v_out=v_out)
    assert (k_out[2, :, 41:] == 7).all() and (v_out[1] == 7).all() and not (k_out[2, :, :41] == 7).all()


@pytest.mark.parametrize("fmt", ["e4m3", "i8", "i4"])
@pytest.mark.parametrize("src", ["bf16", "f16", "f32"])
def test_rows_that_are_not_finite_tiny_or_huge(fmt, src):
    top = torch.finfo(ref.DTYPES[src]).max
    tiny = torch.finfo(ref.DTYPES[src]).tiny
    x = values((1, 1, 10, 64), src, 5)
    x[0, 0, 0, 3] = math.nan
    x[0, 0, 1, 63] = math.inf
    x[0, 0, 2, 0] = -math.inf
    x[0, 0, 3], x[0, 0, 3, 1] = top, -top                       # (a difference beyond fp32 for i4 of f32 and bf16)
    x[0, 0, 4] *= tiny
    x[0, 0, 5] = 0
    x[0, 0, 6] = -0.0
    x[0, 0, 7] = top
    x[0, 0, 8] = tiny
    c = ref.Case(fmt, 1, 1, [10], 64).cuda()
    cache = c.make(kv)
    kv.kvcrush_cache_write(cache, x.cuda(), x.cuda())
    codes, par = ref.quantise(x[0].float().numpy(), fmt)
    for w in "kv":
        assert torch.equal(bits(c.dense(w)[0]), bits(ref.store(codes, fmt)))
        assert same(c.dense(w + "_param")[0], torch.from_numpy(par))
    got, _ = kv.kvcrush_cache_read(cache, dtype=torch.float32)
    assert same(got[0], torch.from_numpy(ref.values32(codes, par, fmt)))
    # (127 times the rounded scale of a row that reaches fp32's largest value may be the next power of two: infinity, by
    # the definition as well, so rows 3 and 7 are left to the comparison above)
    assert torch.isnan(got[0, 0, :3]).all() and torch.isfinite(got[0, 0, [4, 5, 6, 8, 9]]).all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "i4"])
def test_padded_new_tokens_and_views_as_sources(fmt):
    lengths, T, D = [20, 9, 5, 0], 6, 128
    n_new = [6, 2, 0, 6]                                       # the last sequence is empty: nothing of it is new
    c = ref.Case(fmt, 4, 3, lengths, D, room=4).cuda()
    cache = c.make(kv)
    before = {w: c.dense(w) for w in "kv"}
    wide = values((4, T + 2, 3, 2 * D), "bf16", 1).cuda()      # token-major projections, K beside V
    k_new, v_new = (wide[:, 1:T + 1, :, i * D:(i + 1) * D].transpose(1, 2) for i in range(2))
    kv.kvcrush_cache_write(cache, k_new, v_new, n_new=torch.tensor(n_new, dtype=torch.int32, device="cuda"))
    for w, x in (("k", k_new.cpu()), ("v", v_new.cpu())):
        got = c.dense(w)
        for b in range(4):
            n = min(n_new[b], lengths[b])
            codes = x[b, :, :n].float().numpy()
            codes = codes if fmt == "bf16" else ref.quantise(codes, fmt)[0]
            at = slice(lengths[b] - n, lengths[b])
            if n:
                assert torch.equal(bits(got[b, :, at]), bits(ref.store(codes, fmt)))
            rest = [i for i in range(c.capacity) if not at.start <= i < at.stop]
            assert torch.equal(bits(got[b, :, rest]), bits(before[w][b, :, rest]))


# ------------------------------------------------------------------------------------------- attention
def check_attention(c, q, got, n_new, seen=None, scale=None, lists=None, unit=1):
    """Bounds.  Logits: products are exact, D fp32 roundings of at most 2^-24 X each, taken as independent, on both the
    logit and the normaliser, 2^-21 for exponentials and (quantised) the parameters' products: e.  Probabilities:
    two values of 8 (bf16) or 11 bits: 2^-16 or 2^-22; fp32 sums of n terms: 2^-24 sqrt(n) of the sum of magnitudes.
    The result is rounded once."""
    out, lse = (x.cpu().double().numpy() for x in got)
    q64 = q.cpu().double().numpy()
    want, wlse, absolute, size = ref.attend(q64, c.rows64["k"], c.rows64["v"], c.lengths, n_new, seen, scale, lists, unit)
    D, n = c.D, max(max(c.lengths), 1)
    X = size * (4 if c.fmt == "i4" else 1)                      # (i4: codes and lowest value apart, larger than their sum)
    e = 2 * math.sqrt(D) * 2.0 ** -24 * X + 2.0 ** -21
    half = torch.finfo(q.dtype).eps / 2
    p = 2.0 ** -16 if c.fmt == "bf16" else 2.0 ** -21
    allowed = half * np.abs(want) + (2 * e + p + 2.0 ** -23 * math.sqrt(n))[..., None] * absolute * (1 + half)
    empty = np.isinf(wlse)
    assert (out[empty] == 0).all() and (lse[empty] == -np.inf).all()
    assert np.isfinite(out).all()
    assert (np.abs(out - want) <= allowed + 1e-37).all(), np.max((np.abs(out - want) - allowed))
    far = np.abs(lse[~empty] - wlse[~empty])
    assert (far <= e[~empty] + 2.0 ** -23 * np.abs(wlse[~empty]) + 2.0 ** -23 * math.sqrt(n)).all(), far.max()


def q_type(fmt, other="bf16"):
    return fmt if fmt in ref.DTYPES else other


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("B,Hq,Hkv,lengths,D,block_size", [
    (1, 1, 1, [1], 64, 0), (2, 8, 2, [2, 31], 128, 0), (3, 6, 2, [32, 33, 64], 64, 16), (1, 9, 1, [127], 128, 24),
    (2, 4, 4, [700, 129], 128, 16), (1, 40, 1, [300], 64, 0), (4, 8, 8, [0, 1, 513, 96], 128, 1), (1, 70, 1, [257], 128, 0)])
def test_one_token(fmt, B, Hq, Hkv, lengths, D, block_size):
    c = ref.Case(fmt, B, Hkv, lengths, D, block_size=block_size, seed=Hq).cuda()
    q = values((B, Hq, 1, D), q_type(fmt, "f16" if Hq % 2 else "bf16"), 3)
    got = kv.kvcrush_attend(c.make(kv), q.cuda())
    check_attention(c, q, got, [min(1, x) for x in lengths])


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("B,Hq,Hkv,lengths,T,D,block_size,kind", [
    (2, 4, 2, [50, 9], 2, 128, 0, "chain"), (2, 8, 2, [300, 40], 7, 64, 16, "tree"), (1, 6, 2, [133], 33, 128, 0, "tree"),
    (2, 4, 4, [70, 260], 70, 64, 16, "tree"), (1, 8, 1, [200], 130, 128, 32, "chain"), (3, 4, 2, [20, 3, 12], 12, 128, 0, "chain"),
    (2, 2, 1, [65, 64], 64, 64, 8, "tree")])
def test_drafted_tokens(fmt, B, Hq, Hkv, lengths, T, D, block_size, kind):
    c = ref.Case(fmt, B, Hkv, lengths, D, block_size=block_size, seed=T).cuda()
    q = values((B, Hq, T, D), q_type(fmt, "f16" if T % 2 else "bf16"), 4)
    rng = np.random.RandomState(T)
    n_new = [min(T, x) for x in lengths]
    seen = np.stack([ref.tree(T, rng) for _ in range(B)]) if kind == "tree" else None
    mask = None if seen is None else ref.mask_words(seen).cuda()
    got = kv.kvcrush_attend(c.make(kv), q.cuda(), mask=mask)
    check_attention(c, q, got, n_new, seen)


@pytest.mark.parametrize("fmt", ref.FORMATS)
def test_rows_that_see_nothing_padding_and_a_shared_mask(fmt):
    """Sequences of nothing but drafts whose mask leaves rows empty; fewer real drafts than T; a query axis in the middle."""
    lengths, T, Hq, Hkv, D = [5, 40, 7, 0], 5, 6, 3, 64
    n_new = [5, 3, 0, 0]
    c = ref.Case(fmt, 4, Hkv, lengths, D, seed=1).cuda()
    seen = np.zeros((T, T), dtype=bool)
    seen[1, 0] = seen[1, 1] = seen[3, 1] = seen[4, 4] = True    # rows 0 and 2 see no draft
    q = values((4, T, Hq, D), q_type(fmt), 9).transpose(1, 2)
    out = torch.full((4, T, Hq, D), 5.0, dtype=q.dtype, device="cuda").transpose(1, 2)
    got = kv.kvcrush_attend(c.make(kv), q.cuda(), mask=ref.mask_words(seen).cuda(), out=out,
                            n_new=torch.tensor([5, 3, 0, 4], dtype=torch.int32, device="cuda"))
    assert got[0] is out
    check_attention(c, q, got, n_new, np.broadcast_to(seen, (4, T, T)))


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("block_size", [0, 16])
def test_unseen_values_have_no_influence(fmt, block_size):
    """Drafts that a query does not see hold NaN, infinities or huge rows; those that see them are not looked at."""
    B, Hq, Hkv, T, D, L = 1, 8, 2, 6, 128, 75
    c = ref.Case(fmt, B, Hkv, [L], D, block_size=block_size, seed=2)
    rows = {w: c.rows64[w].copy() for w in "kv"}
    seen = np.tri(T, dtype=bool)
    seen[:, 2] = seen[:, 4] = False                             # drafts 2 and 4 are dead branches
    seen[2, 2] = seen[4, 4] = True
    for j, bad in ((2, math.nan), (4, math.inf)):
        pos = L - T + j
        for w in "kv":
            t, par = c.tensors[w], c.tensors[w + "_param"]
            at = (0, slice(None), pos) if not block_size else (int(c.table[0, pos // block_size]), pos % block_size)
            if par is not None:
                par[at] = bad
                t.view(torch.uint8)[at] = 0x7F
            else:
                t[at] = bad
    c.cuda()
    q = values((B, Hq, T, D), q_type(fmt), 6)
    out, lse = kv.kvcrush_attend(c.make(kv), q.cuda(), mask=ref.mask_words(seen).cuda())
    good = [0, 1, 3, 5]
    c.rows64 = rows
    sub = seen.copy()
    sub[[2, 4]] = False                                         # (rows 2 and 4 are not compared)
    want = ref.attend(q.double().numpy(), rows["k"], rows["v"], [L], [T], sub[None])
    assert torch.isfinite(out[:, :, good]).all() and torch.isfinite(lse[:, :, good]).all()
    far = (out.cpu().double().numpy() - want[0])[:, :, good]
    half = torch.finfo(q.dtype).eps / 2
    assert (np.abs(far) <= half * np.abs(want[0][:, :, good]) + 2.0 ** -14 * want[2][:, :, good]).all()
    assert torch.isnan(out[:, :, 2]).all() if fmt not in ("i8", "i4", "e4m3") else True


@pytest.mark.parametrize("fmt", ["bf16", "f16", "f32", "i8", "i4"])
def test_large_logits_and_scales(fmt):
    """Peaked rows (logits of some hundreds), rows of very different size, the caller's own scale."""
    B, Hq, Hkv, D, L = 2, 8, 2, 128, 333
    c = ref.Case(fmt, B, Hkv, [L, 200], D, seed=8)
    size = np.exp(2.0 * np.random.RandomState(1).randn(B, Hkv, L, 1))
    for w in ("k", "v"):
        x = (np.random.RandomState(5).randn(B, Hkv, L, D) * size).astype(np.float32)
        if fmt in ref.DTYPES:
            t = torch.from_numpy(x).to(ref.DTYPES[fmt])
            c.tensors[w], c.rows64[w] = t, t.double().numpy()
        else:
            codes, par = ref.quantise(x, fmt)
            c.tensors[w], c.tensors[w + "_param"], c.rows64[w] = ref.store(codes, fmt), torch.from_numpy(par), ref.values64(codes, par, fmt)
    c.cuda()
    q = values((B, Hq, 1, D), q_type(fmt), 6, 3.0)
    for scale in (0.0, 0.7, 0.001):
        got = kv.kvcrush_attend(c.make(kv), q.cuda(), scale=scale)
        check_attention(c, q, got, [1, 1], scale=scale or None)


@pytest.mark.parametrize("fmt,B,Hq,Hkv,lengths,T,D,block_size", [
    ("bf16", 1, 8, 2, [5000], 1, 128, 0), ("f32", 1, 4, 2, [3001], 2, 128, 16), ("e4m3", 2, 16, 2, [4097, 2500], 5, 128, 16),
    ("i4", 1, 8, 1, [9001], 3, 64, 0), ("i8", 3, 4, 2, [3100, 1, 2049], 1, 64, 16), ("f16", 1, 32, 4, [2600], 12, 64, 64)])
def test_long_caches_in_pieces(fmt, B, Hq, Hkv, lengths, T, D, block_size):
    c = ref.Case(fmt, B, Hkv, lengths, D, block_size=block_size, seed=11).cuda()
    q = values((B, Hq, T, D), q_type(fmt), 12)
    got = kv.kvcrush_attend(c.make(kv), q.cuda())
    check_attention(c, q, got, [min(T, x) for x in lengths])
    again = kv.kvcrush_attend(c.make(kv), q.cuda())
    assert torch.equal(bits(got[0]), bits(again[0])) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("fmt,B,Hq,Hkv,lengths,T,D", [
    ("i8", 1, 21, 3, [1500], 101, 64), ("bf16", 3, 14, 2, [900, 40, 700], 51, 128), ("f32", 1, 27, 3, [600], 77, 128),
    ("i4", 2, 30, 2, [0, 1400], 71, 64)])
def test_pieces_of_many_rows(fmt, B, Hq, Hkv, lengths, T, D):
    """More than 2048 rows, no multiple of a workgroup's, whose pieces each group of lanes merges by itself: equal cuts of one
    sequence, cuts by length of several, sequences that have no piece to merge."""
    assert B * Hq * T > 2048 and B * Hq * T % 8
    c = ref.Case(fmt, B, Hkv, lengths, D, seed=T, room=70).cuda()
    q, cache = values((B, Hq, T, D), q_type(fmt), 5).cuda(), c.make(kv)
    assert kv.kvcrush_attend_workspace(cache, Hq, T, q.dtype) > 0
    check_attention(c, q, kv.kvcrush_attend(cache, q), [min(T, n) for n in lengths])


# ---------------------------------------------------------------------------------------------- blocks
def reference_bounds(c, unit):
    nb = -(-c.capacity // unit)
    out = []
    for b in range(c.B):
        codes = ref.load(c.dense("k"), c.fmt)[b]
        par = None if c.fmt in ref.DTYPES else c.dense("k_param")[b].numpy()
        out.append(ref.bounds(ref.values32(codes, par, c.fmt), c.lengths[b], unit, nb))
    return np.stack([x[0] for x in out]), np.stack([x[1] for x in out])


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("D,unit,block_size", [(128, 16, 0), (64, 32, 16), (128, 7, 16), (64, 1, 0), (128, 200, 24)])
def test_block_bounds(fmt, D, unit, block_size):
    c = ref.Case(fmt, 3, 2, [130, 0, 77], D, block_size=block_size, seed=unit, room=40).cuda()
    cache = c.make(kv)
    want = reference_bounds(c, unit)
    got = kv.kvcrush_block_bounds(cache, unit)
    assert np.array_equal(got[0].cpu().numpy(), want[0]) and np.array_equal(got[1].cpu().numpy(), want[1])
    # new tokens: their blocks change, the others stay what they are
    new = values((3, 2, 9, D), q_type(fmt), 2, 4.0).cuda()
    n_new = [9, 0, 5]
    counts = torch.tensor([9, 9, 5], dtype=torch.int32, device="cuda")
    kv.kvcrush_cache_write(cache, new, new, n_new=counts)
    want = reference_bounds(c, unit)
    marked = [x.clone() for x in got]
    for b in range(3):
        first = (c.lengths[b] - n_new[b]) // unit
        marked[0][b, :, :first] = 77
        want[0][b, :, :first] = 77
        if not n_new[b]:
            marked[0][b], want[0][b] = 55, 55
    kv.kvcrush_block_bounds(cache, unit, marked[0], marked[1], T=9, n_new=counts)
    assert np.array_equal(marked[0].cpu().numpy(), want[0]) and np.array_equal(marked[1].cpu().numpy(), want[1])


def reference_lists(c, q, want, unit, n_select, n_sink, n_recent, n_new):
    G = q.shape[1] // c.Hkv
    q = q.float().numpy()
    return [[[ref.choose(q[b, g * G:(g + 1) * G, t], want[0][b, g], want[1][b, g], c.lengths[b], unit, n_select, n_sink, n_recent)
              if t < n_new[b] else [] for t in range(q.shape[2])] for g in range(c.Hkv)] for b in range(c.B)]


def padded(lists, n):
    return torch.tensor([[[x + [-1] * (n - len(x)) for x in g] for g in b] for b in lists], dtype=torch.int32)


@pytest.mark.parametrize("qt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,Hq,Hkv,lengths,T,D,unit,n_select,n_sink,n_recent", [
    (1, 4, 2, [300], 1, 128, 16, 5, 1, 1), (3, 6, 2, [700, 40, 0], 3, 64, 8, 12, 0, 2), (1, 40, 1, [513], 2, 128, 4, 100, 3, 0),
    (2, 2, 2, [2100, 999], 1, 64, 2, 512, 0, 0), (1, 3, 1, [5000], 1, 64, 1, 37, 5, 7), (2, 8, 8, [64, 65], 1, 128, 64, 1, 0, 1),
    (1, 1, 1, [9000], 1, 64, 1, 4500, 0, 0), (1, 2, 1, [64], 2, 64, 16, 4, 2, 2)])
def test_block_selection(qt, B, Hq, Hkv, lengths, T, D, unit, n_select, n_sink, n_recent):
    c = ref.Case("f32", B, Hkv, lengths, D, seed=n_select).cuda()
    cache = c.make(kv)
    want = reference_bounds(c, unit)
    q = values((B, Hq, T, D), qt, 21)
    n_new = [min(max(T - b, 0), lengths[b]) for b in range(B)]
    counts = torch.tensor([T - b for b in range(B)], dtype=torch.int32, device="cuda")
    bnd = kv.kvcrush_block_bounds(cache, unit)
    got = kv.kvcrush_block_select(cache, q.cuda(), *bnd, unit, n_select, n_sink, n_recent, n_new=counts)
    lists = reference_lists(c, q, want, unit, n_select, n_sink, n_recent, n_new)
    assert torch.equal(got.cpu(), padded(lists, n_select))


@pytest.mark.parametrize("n_select", [1, 2, 63, 64, 65, 200])
def test_block_selection_ties(n_select):
    """Equal keys everywhere, a few distinct ones, queries of zeros: ties go to the lower block."""
    c = ref.Case("f32", 2, 2, [800, 800], 64, seed=1)
    c.tensors["k"][:, :, :] = c.tensors["k"][0, 0, 0]
    c.tensors["k"][0, 0, 400:402] *= 2
    c.cuda()
    cache = c.make(kv)
    q = values((2, 4, 1, 64), "f32", 5)
    q[1, 0:2] = 0
    want = reference_bounds(c, 4)
    bnd = kv.kvcrush_block_bounds(cache, 4)
    for ends in ((0, 0), (0, 1), (1, 0)):
        got = kv.kvcrush_block_select(cache, q.cuda(), *bnd, 4, n_select, *ends)
        assert torch.equal(got.cpu(), padded(reference_lists(c, q, want, 4, n_select, *ends, [1, 1]), n_select))


@pytest.mark.parametrize("fmt", ref.FORMATS)
@pytest.mark.parametrize("B,Hq,Hkv,lengths,T,D,unit,n_select,block_size", [
    (1, 4, 2, [300], 1, 128, 16, 5, 16), (2, 6, 2, [700, 40], 3, 64, 8, 12, 0), (1, 33, 1, [513], 2, 128, 32, 4, 16),
    (1, 8, 2, [3000], 1, 64, 16, 100, 24), (3, 4, 4, [96, 0, 5], 4, 128, 5, 3, 0), (1, 64, 1, [200], 1, 64, 64, 2, 64)])
def test_attention_over_chosen_blocks(fmt, B, Hq, Hkv, lengths, T, D, unit, n_select, block_size):
    c = ref.Case(fmt, B, Hkv, lengths, D, block_size=block_size, seed=unit).cuda()
    cache = c.make(kv)
    q = values((B, Hq, T, D), q_type(fmt), 31)
    n_new = [min(T, x) for x in lengths]
    rng = np.random.RandomState(T)
    seen = np.stack([ref.tree(T, rng) for _ in range(B)])
    bnd = kv.kvcrush_block_bounds(cache, unit)
    blocks = kv.kvcrush_block_select(cache, q.cuda(), *bnd, unit, n_select, n_sink=1, n_recent=1)
    lists = reference_lists(c, q, reference_bounds(c, unit), unit, n_select, 1, 1, n_new)
    assert torch.equal(blocks.cpu(), padded(lists, n_select))
    got = kv.kvcrush_attend(cache, q.cuda(), mask=ref.mask_words(seen).cuda(), blocks=blocks, unit=unit)
    check_attention(c, q, got, n_new, seen, lists=lists, unit=unit)


def test_lists_with_entries_that_count_for_nothing():
    c = ref.Case("bf16", 1, 1, [100], 64, seed=4).cuda()
    cache = c.make(kv)
    q = values((1, 2, 2, 64), "bf16", 1)
    blocks = torch.tensor([[[[-1, 0, 0, 3, 2, 3, 9, 10 ** 9], [-5, -1, 10, 7, 2 ** 31 - 1, -1, 3, 3]]]], dtype=torch.int32)
    # ascending ones: the first list's 0, 3, (2 is behind 3), 3 behind 2 again, 9; a repeated one counts once
    blocks[0, 0, 0] = torch.tensor([-1, 0, 0, 3, 3, 9, 10, 10 ** 9])
    got = kv.kvcrush_attend(cache, q.cuda(), blocks=blocks.cuda(), unit=10)
    # (query 1: nothing before 10, which is beyond the sequence; 7 is not larger than 10; 3 is larger than -1, the second 3 not)
    check_attention(c, q, got, [2], lists=[[[[0, 3, 9], [3]]]], unit=10)


# -------------------------------------------------------------------------------------------- together
def test_a_generation_with_a_quantised_cache_step_by_step():
    """Prompt, then drafts written, attended to with chosen blocks, some of them kept: the cache, its bounds and the
    results follow the reference throughout."""
    fmt, B, Hq, Hkv, D, unit, bs, T = "i8", 2, 8, 2, 64, 8, 16, 4
    c = ref.Case(fmt, B, Hkv, [0, 0], D, capacity=160, block_size=bs).cuda()
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    cache = kv.make_cache(c.tensors["k"], c.tensors["v"], 160, c.tensors["k_param"], c.tensors["v_param"], lengths, c.table.cuda())
    bnd = kv.kvcrush_block_bounds(cache, unit)
    rows = {w: np.zeros((B, Hkv, 160, D)) for w in "kv"}
    rng = np.random.RandomState(3)
    at = [0, 0]
    for step, n in enumerate([50, 4, 4, 1, 4, 30, 4]):
        n_new = [n, max(n - step % 3, 1)]
        at = [a + x for a, x in zip(at, n_new)]
        lengths.copy_(torch.tensor(at, dtype=torch.int32))
        counts = torch.tensor(n_new, dtype=torch.int32, device="cuda")
        new = {w: values((B, Hkv, n, D), "bf16", 100 * step + i) for i, w in enumerate("kv")}
        kv.kvcrush_cache_write(cache, new["k"].cuda(), new["v"].cuda(), n_new=counts)
        kv.kvcrush_block_bounds(cache, unit, *bnd, T=n, n_new=counts)
        for w in "kv":
            for b in range(B):
                codes, par = ref.quantise(new[w][b, :, :n_new[b]].float().numpy(), fmt)
                rows[w][b, :, at[b] - n_new[b]:at[b]] = ref.values64(codes, par, fmt)
        c.lengths, c.rows64 = list(at), rows
        want = reference_bounds(c, unit)
        assert np.array_equal(bnd[0].cpu().numpy(), want[0]) and np.array_equal(bnd[1].cpu().numpy(), want[1])
        q = values((B, Hq, n, D), "bf16", 100 * step + 50)
        seen = np.stack([ref.tree(n, rng) for _ in range(B)])
        mask = ref.mask_words(seen).cuda()
        blocks = kv.kvcrush_block_select(cache, q.cuda(), *bnd, unit, 6, 1, 2, n_new=counts)
        lists = reference_lists(c, q, want, unit, 6, 1, 2, n_new)
        assert torch.equal(blocks.cpu(), padded(lists, 6))
        check_attention(c, q, kv.kvcrush_attend(cache, q.cuda(), mask=mask, n_new=counts, blocks=blocks, unit=unit), n_new, seen,
                        lists=lists, unit=unit)
        check_attention(c, q, kv.kvcrush_attend(cache, q.cuda(), mask=mask, n_new=counts), n_new, seen)
        if n == T:                                              # the last draft is not kept
            at = [a - 1 for a in at]


def test_a_step_in_a_graph_replayed_on_changing_inputs():
    """Write, bounds, choice and attention captured once: every replay, with eager work between, gives the eager result."""
    fmt, B, Hq, Hkv, D, unit, T = "e4m3", 2, 8, 2, 128, 16, 3
    made = [ref.Case(fmt, B, Hkv, [600, 600], D, capacity=640, block_size=16, seed=5).cuda() for _ in range(2)]
    lengths = torch.tensor([400, 333], dtype=torch.int32, device="cuda")
    caches = [kv.make_cache(c.tensors["k"], c.tensors["v"], 640, c.tensors["k_param"], c.tensors["v_param"], lengths, c.table.cuda())
              for c in made]
    bnds = [kv.kvcrush_block_bounds(c, unit) for c in caches]
    new = torch.empty(B, Hkv, T, D, dtype=torch.bfloat16, device="cuda")
    q = torch.empty(B, Hq, T, D, dtype=torch.bfloat16, device="cuda")
    counts = torch.empty(B, dtype=torch.int32, device="cuda")
    ws = [torch.empty(1 << 24, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(cache, bnd):
        kv.kvcrush_cache_write(cache, new, new, n_new=counts)
        kv.kvcrush_block_bounds(cache, unit, *bnd, T=T, n_new=counts)
        blocks = kv.kvcrush_block_select(cache, q, *bnd, unit, 8, n_new=counts, workspace=ws[0])
        sparse = kv.kvcrush_attend(cache, q, n_new=counts, blocks=blocks, unit=unit, workspace=ws[1])
        full = kv.kvcrush_attend(cache, q, n_new=counts, workspace=ws[1])
        rows = kv.kvcrush_cache_read(cache, n=600, dtype=torch.bfloat16)
        return (blocks, *sparse, *full, *rows)

    def inputs(i):
        new.copy_(values(new.shape, "bf16", i))
        q.copy_(values(q.shape, "bf16", 50 + i))
        counts.copy_(torch.tensor([1 + i % 3, 3 - i % 3], dtype=torch.int32))
        lengths.copy_(torch.tensor([400 + 3 * i, 590 - i], dtype=torch.int32))

    inputs(0)
    step(caches[0], bnds[0])
    step(caches[1], bnds[1])
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = step(caches[0], bnds[0])
    for i in range(1, 5):
        inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        want = step(caches[1], bnds[1])
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(bits(x), bits(y))
        for x, y in zip(bnds[0], bnds[1]):
            assert torch.equal(x, y)


def test_calls_on_another_stream():
    c = ref.Case("i8", 2, 2, [900, 800], 128, seed=3).cuda()
    cache = c.make(kv)
    q = values((2, 8, 4, 128), "bf16", 2).cuda()
    bnd = kv.kvcrush_block_bounds(cache, 16)
    want_b = kv.kvcrush_block_select(cache, q, *bnd, 16, 10)
    want = kv.kvcrush_attend(cache, q, blocks=want_b, unit=16)
    rows = kv.kvcrush_cache_read(cache)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        bnd2 = kv.kvcrush_block_bounds(cache, 16, stream=side)
        blocks = kv.kvcrush_block_select(cache, q, *bnd2, 16, 10, stream=side)
        got = kv.kvcrush_attend(cache, q, blocks=blocks, unit=16, stream=side)
        rows2 = kv.kvcrush_cache_read(cache, stream=side)
        side.synchronize()
        assert torch.equal(blocks, want_b) and torch.equal(bits(got[0]), bits(want[0])) and torch.equal(got[1], want[1])
        assert all(torch.equal(bits(x), bits(y)) for x, y in zip(rows, rows2))


def test_gradients_are_refused():
    """The calls are for inference: a tensor that autograd follows is turned down rather than cut off from its gradient."""
    c = ref.Case("bf16", 1, 2, [20], 64, seed=3).cuda()
    cache = c.make(kv)
    q = values((1, 4, 1, 64), "bf16", 1).cuda().requires_grad_()
    k = values((1, 2, 1, 64), "bf16", 2).cuda().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        kv.kvcrush_attend(cache, q)
    with pytest.raises(ValueError, match="gradient"):
        kv.kvcrush_cache_write(cache, k, k.detach())
    with pytest.raises(ValueError, match="gradient"):
        kv.make_cache(c.tensors["k"].requires_grad_(), c.tensors["v"], 20)
    with torch.no_grad():
        kv.kvcrush_cache_write(cache, k, k)
        out, _ = kv.kvcrush_attend(cache, q)
    assert torch.isfinite(out).all() and not out.requires_grad
    with pytest.raises(ValueError, match="shape"):
        kv.kvcrush_attend(cache, q.detach(), out=torch.empty(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError, match="blocks"):
        kv.kvcrush_attend(cache, q.detach(), blocks=torch.zeros(1, 1, 1, 4, dtype=torch.int32, device="cuda"), unit=16)
    with pytest.raises(ValueError, match="mask"):
        kv.kvcrush_attend(cache, q.detach(), mask=torch.zeros(1, 2, 1, dtype=torch.int64, device="cuda"))
    with pytest.raises(kv.KVCrushError):
        kv.kvcrush_attend(cache, q.detach().half())


@pytest.mark.parametrize("n_new,lengths", [([3, 3], [2, 40]), ([-5, 100], [30, 3]), ([2 ** 31 - 1, -2 ** 31], [10, 10])])
def test_counts_and_lengths_outside_their_ranges_are_pulled_into_them(n_new, lengths):
    """n_new beyond T or the length, negative ones, lengths beyond S: as the header says, clamped."""
    B, T, D = 2, 3, 64
    c = ref.Case("i8", B, 2, lengths, D, capacity=64, seed=6).cuda()
    given = torch.tensor([L if L != 40 else 10 ** 9 for L in lengths], dtype=torch.int32, device="cuda")
    cache = kv.make_cache(c.tensors["k"], c.tensors["v"], max(lengths), c.tensors["k_param"], c.tensors["v_param"], given)
    q = values((B, 4, T, D), "bf16", 8)
    real = [min(max(n, 0), T, L) for n, L in zip(n_new, lengths)]
    counts = torch.tensor(n_new, dtype=torch.int32, device="cuda")
    check_attention(c, q, kv.kvcrush_attend(cache, q.cuda(), n_new=counts), real)
    bnd = kv.kvcrush_block_bounds(cache, 8)
    got = kv.kvcrush_block_select(cache, q.cuda(), *bnd, 8, 3, 1, 1, n_new=counts)
    assert torch.equal(got.cpu(), padded(reference_lists(c, q, reference_bounds(c, 8), 8, 3, 1, 1, real), 3))


def test_block_tables_that_name_blocks_outside_the_pool():
    """Such entries are pulled into the pool, never followed: results are those of the pulled table."""
    c = ref.Case("bf16", 1, 2, [60], 64, block_size=16, seed=2)
    n = c.n_blocks
    good = torch.tensor([[0, n - 1, 1, n - 1]], dtype=torch.int32)
    bad = torch.tensor([[-7, n, 1, 2 ** 31 - 1]], dtype=torch.int32)
    c.tensors = {w: None if t is None else torch.nan_to_num(t, nan=0.5) for w, t in c.tensors.items()}
    c.cuda()
    q = values((1, 4, 1, 64), "bf16", 3).cuda()
    results = []
    for table in (good, bad):
        cache = kv.make_cache(c.tensors["k"], c.tensors["v"], 60, block_table=table.cuda())
        results.append((*kv.kvcrush_attend(cache, q), *kv.kvcrush_cache_read(cache), *kv.kvcrush_block_bounds(cache, 8)))
    for a, b in zip(*results):
        assert torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("fmt", ["bf16", "i4"])
def test_sequences_of_very_different_lengths_share_the_pieces(fmt):
    """Lengths on the device, many sequences: pieces dealt by length, some sequences with one piece, empty ones among them."""
    lengths = [4000, 1, 0, 700, 33, 2500, 5, 64] + [7] * 13
    B = len(lengths)
    c = ref.Case(fmt, B, 1, lengths, 64, seed=5).cuda()
    q = values((B, 4, 2, 64), "bf16", 4)
    check_attention(c, q, kv.kvcrush_attend(c.make(kv), q.cuda()), [min(2, x) for x in lengths])


def test_more_sequences_than_a_wave_has_lanes():
    lengths = [(37 * i) % 300 for i in range(70)]
    c = ref.Case("i8", 70, 1, lengths, 64, seed=5).cuda()
    q = values((70, 2, 1, 64), "f16", 4)
    check_attention(c, q, kv.kvcrush_attend(c.make(kv), q.cuda()), [min(1, x) for x in lengths])


@pytest.mark.parametrize("fmt,rows", [("i8", 2_400_000), ("bf16", 1_200_000)])
def test_offsets_beyond_32_bits(fmt, rows):
    """A pool of more than 4 GiB whose last blocks are used."""
    D, Hkv, bs = 128, 16, 4
    n_blocks = rows // bs
    k, v = (torch.zeros(n_blocks, bs, Hkv, D, dtype=ref.STORED[fmt], device="cuda") for _ in range(2))
    assert k.numel() * k.element_size() > 2 ** 32
    k_param, v_param = (torch.zeros(n_blocks, bs, Hkv, device="cuda") if fmt == "i8" else None for _ in range(2))
    table = torch.tensor([[n_blocks - 1, 0, n_blocks - 2, n_blocks // 2 + 1]], dtype=torch.int32)
    cache = kv.make_cache(k, v, 13, k_param, v_param, block_table=table.cuda())
    new = {w: values((1, Hkv, 13, D), "bf16", i) for i, w in enumerate("kv")}
    kv.kvcrush_cache_write(cache, new["k"].cuda(), new["v"].cuda())
    c = ref.Case(fmt, 1, Hkv, [13], D)
    for w in "kv":
        x = new[w].float().numpy()
        codes, par = (x, None) if fmt == "bf16" else ref.quantise(x, fmt)
        c.rows64[w] = ref.values64(codes, par, fmt)
    q = values((1, 32, 1, D), "bf16", 9)
    check_attention(c, q, kv.kvcrush_attend(cache, q.cuda()), [1])
    got = kv.kvcrush_cache_read(cache, dtype=torch.bfloat16)
    for w, x in zip("kv", got):
        assert (np.abs(x.cpu().double().numpy() - c.rows64[w]) <= 2.0 ** -8 * np.abs(c.rows64[w])).all()
    tokens = lambda t: torch.stack([t[int(table[0, i // bs]), i % bs] for i in range(12)]).transpose(0, 1)  # noqa: E731
    bnd = kv.kvcrush_block_bounds(cache, 4)
    par = None if fmt == "bf16" else tokens(k_param).cpu().numpy()
    want = ref.bounds(ref.values32(ref.load(tokens(k), fmt), par, fmt), 12, 4, 3)
    assert np.array_equal(bnd[0][0, :, :3].cpu().numpy(), want[0]) and np.array_equal(bnd[1][0, :, :3].cpu().numpy(), want[1])
