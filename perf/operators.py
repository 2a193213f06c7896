"""The operators that use a KV cache, as timed and compared cases.

A serving program holds a layer's cache in fewer bits (it is quantised as it is written, and read back where the
values themselves are needed), attends to it with one new token or with a tree of drafted ones, and on long caches
attends only to the blocks that a cheap score picks for each query.  Four kinds of case:

  write    kvcrush_cache_write of T new tokens, which are then read back (kvcrush_cache_read of their positions)
  read     kvcrush_cache_read of a whole cache, or of the tokens that a selection kept
  attend   kvcrush_attend: T new tokens, already in the cache, attend to it (T = 1: an ordinary decoding step)
  sparse   kvcrush_block_bounds of the new tokens' blocks, kvcrush_block_select, kvcrush_attend on the chosen blocks

Caches are dense [B,Hkv,capacity,D] or paged pools [n_blocks,16,Hkv,D], in bf16, f16, f32, e4m3, 8-bit or 4-bit integers;
`own` = False computes the same in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16                                    # tokens per block of a paged pool
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BITS = {"bf16": 16, "f16": 16, "f32": 32, "e4m3": 8, "i8": 8, "i4": 4}
PARAMS = {"bf16": 0, "f16": 0, "f32": 0, "e4m3": 4, "i8": 4, "i4": 8}  # bytes per row beside the codes
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8, "i4": torch.uint8}
TINY = 2.0 ** -100                            # rows (or ranges) below this are stored as zero


def listed():
    return [
        # one generated token of a few sequences enters an 8-bit cache: latency
        {"name": "write_t1_i8", "kind": "write", "B": 8, "Hkv": 8, "S": 2048, "T": 1, "D": 128, "dtype": "bf16", "format": "i8",
         "paged": False, "ragged": False},
        # a batch of long prompts goes into a paged cache after prefill
        {"name": "write_t8192_e4m3_paged", "kind": "write", "B": 8, "Hkv": 8, "S": 8192, "T": 8192, "D": 128, "dtype": "bf16",
         "format": "e4m3", "paged": True, "ragged": False},
        # the tokens that a selection kept of a 4-bit cache, as values
        {"name": "read_i4_4096_of_16384", "kind": "read", "B": 1, "Hkv": 8, "S": 16384, "n": 4096, "D": 128, "dtype": "bf16",
         "format": "i4", "paged": False, "ragged": False},
        # whole caches of different lengths, as values
        {"name": "read_e4m3_s7839", "kind": "read", "B": 4, "Hkv": 8, "S": 7839, "n": 0, "D": 128, "dtype": "f16",
         "format": "e4m3", "paged": True, "ragged": True},
        # the smallest attention: a short cache of two sequences
        {"name": "attend_b2_s160", "kind": "attend", "B": 2, "Hq": 8, "Hkv": 2, "S": 160, "T": 1, "D": 128, "dtype": "bf16",
         "format": "bf16", "paged": False, "ragged": False},
        # a single-precision model without shared heads
        {"name": "attend_mha8_s512_f32", "kind": "attend", "B": 1, "Hq": 8, "Hkv": 8, "S": 512, "T": 1, "D": 64, "dtype": "f32",
         "format": "f32", "paged": False, "ragged": False},
        # generation on a compressed cache, a batch of sequences
        {"name": "attend_b8_s2048", "kind": "attend", "B": 8, "Hq": 32, "Hkv": 8, "S": 2048, "T": 1, "D": 128, "dtype": "bf16",
         "format": "bf16", "paged": False, "ragged": False},
        # generation on long paged 8-bit caches of different lengths: the largest read
        {"name": "attend_b4_s32768_e4m3", "kind": "attend", "B": 4, "Hq": 32, "Hkv": 8, "S": 32768, "T": 1, "D": 128,
         "dtype": "bf16", "format": "e4m3", "paged": True, "ragged": True},
        # a small draft tree on one long prompt
        {"name": "tree16_s16384", "kind": "attend", "B": 1, "Hq": 32, "Hkv": 8, "S": 16384, "T": 16, "D": 128, "dtype": "bf16",
         "format": "bf16", "paged": False, "ragged": False},
        # a large tree over the average prompt, ragged: the most arithmetic for a byte read
        {"name": "tree64_b2_s7839_i8", "kind": "attend", "B": 2, "Hq": 32, "Hkv": 8, "S": 7839, "T": 64, "D": 128, "dtype": "f16",
         "format": "i8", "paged": False, "ragged": True},
        # one token on a very long 4-bit cache, 64 of its 2048 blocks
        {"name": "sparse_s32768_i4", "kind": "sparse", "B": 1, "Hq": 32, "Hkv": 8, "S": 32768, "T": 1, "D": 128, "dtype": "bf16",
         "format": "i4", "paged": True, "ragged": False, "unit": 16, "n_select": 64},
        # a short draft on a batch of long caches, larger blocks
        {"name": "sparse_b4_s16384_t4", "kind": "sparse", "B": 4, "Hq": 32, "Hkv": 8, "S": 16384, "T": 4, "D": 128, "dtype": "bf16",
         "format": "bf16", "paged": True, "ragged": True, "unit": 32, "n_select": 48},
    ]


# --------------------------------------------------------------------------------- drawing
HEADS = [(32, 8), (32, 32), (8, 8), (8, 2), (12, 4), (16, 16), (24, 8), (4, 4)]
MOST_BYTES = 2.2e8                            # the largest listed attention; a third of the largest write
MOST_FLOPS = 1.4e10


def _size(rng, lo, hi):
    """Spread over the logarithm; one in four a multiple of 64, the others as they fall."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, n // 64 * 64) if rng.random() < 0.25 else n


def draw(rng):
    kind = rng.choice(["write", "read", "attend", "attend", "attend", "sparse"])
    Hq, Hkv = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    quantised = rng.choice(["e4m3", "i8", "i4"])
    c = {"kind": kind, "B": rng.choice([1, 2, 3, 4, 8, 16]), "Hkv": Hkv, "D": rng.choice([64, 128, 128]), "dtype": dtype,
         "paged": rng.random() < 0.5, "ragged": rng.random() < 0.5}
    if kind == "write":
        T = _size(rng, 1, 8192)
        c.update(S=T + _size(rng, 1, 8192), T=T, format=quantised, dtype=rng.choice(["bf16", "f16", "f32"]))
    elif kind == "read":
        S = _size(rng, 100, 32768)
        c.update(S=S, n=rng.choice([0, max(1, S // rng.randint(2, 9))]), format=quantised,
                 dtype=rng.choice(["bf16", "f16", "f32"]))
    else:
        c.update(Hq=Hq, format=rng.choice([dtype, quantised, quantised]))
        if kind == "attend":
            T = rng.choice([1, 1, _size(rng, 2, 128)])
            c.update(S=T + _size(rng, 100, 32768 - 128), T=T)
            if rng.random() < 0.15:
                c.update(dtype="f32", format="f32", T=rng.randint(1, 8))
        else:
            unit = rng.choice([16, 32, 64])
            c["B"] = min(c["B"], 64 // Hkv)
            c.update(S=_size(rng, 2000, 32768), T=rng.choice([1, 1, 2, 4]), unit=unit, n_select=_size(rng, 8, 1536 // unit))
    while c["B"] > 1 and (work(c)["bytes"] > MOST_BYTES or work(c)["flops"] > MOST_FLOPS):
        c["B"] -= 1
    while work(c)["bytes"] > MOST_BYTES or work(c)["flops"] > MOST_FLOPS:
        c["S"] = c["S"] * 3 // 4
        c["T"] = min(c["T"], max(1, c["S"] // 2)) if "T" in c else 1
        c["n"] = min(c.get("n", 0), c["S"])
    return c


# ---------------------------------------------------------------- the plain forms' parts
def _over(a, b):
    """a / b of a number and a tensor, rounded once (torch makes a reciprocal and a product of it, rounded twice)."""
    return torch.full_like(b, a) / b if isinstance(a, float) else a / torch.full_like(a, b)


def _pack4(codes):
    """4-bit codes, the even position in the low half of its byte."""
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack4(packed):
    return torch.stack((packed & 15, packed >> 4), dim=-1).flatten(-2)


def _quantise(x, fmt):
    """Rows of fp32 values -> (codes, parameters): e4m3 and i8 with one scale a row, i4 with scale and lowest value."""
    if fmt == "i4":
        lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
        span = hi - lo
        flat = span < TINY
        inv = torch.where(flat, 0.0, _over(15.0, span))
        codes = ((x - lo) * inv).round().to(torch.uint8)
        return _pack4(codes), torch.cat((torch.where(flat, 0.0, _over(span, 15.0)), lo), -1)
    top = 448.0 if fmt == "e4m3" else 127.0
    a = x.abs().amax(-1, keepdim=True)
    zero = a < TINY
    y = x * torch.where(zero, 0.0, _over(top, a))
    return (y.to(torch.float8_e4m3fn) if fmt == "e4m3" else y.round().to(torch.int8)), torch.where(zero, 0.0, _over(a, top))[..., 0]


def _values(codes, par, fmt):
    """What the codes stand for, in fp32."""
    if fmt == "i4":  # (the product of a scale and a small integer is exact in 64 bits: one rounding)
        return (_unpack4(codes).double() * par[..., :1].double() + par[..., 1:].double()).float()
    return codes.float() * par[..., None] if fmt in CODES else codes.float()


def _rows(st, which, index):
    """Rows of the cache's K or V at token positions index [B,n] as fp32 [B,Hkv,n,D]."""
    codes, par, fmt = st[which], st[which + "_param"], st["format"]
    raw = codes.view(torch.uint8) if fmt in CODES else codes
    if st["table"] is None:
        at = (torch.arange(index.shape[0], device=index.device)[:, None], slice(None), index)   # -> [B,n,Hkv,..]
    else:
        block = st["table"].gather(1, index // BLOCK).long()
        at = (block, index % BLOCK)
    got = raw[at].transpose(1, 2)
    got = got.view(codes.dtype) if fmt in CODES else got
    return _values(got, None if par is None else par[at].transpose(1, 2), fmt)


def _store(st, which, index, codes, par):
    """Codes [B,Hkv,n,..] go to the token positions index [B,n] of the cache."""
    dst = st[which].view(torch.uint8)
    if st["table"] is None:
        at = (torch.arange(index.shape[0], device=index.device)[:, None], slice(None), index)
    else:
        at = (st["table"].gather(1, index // BLOCK).long(), index % BLOCK)
    dst[at] = codes.view(torch.uint8).transpose(1, 2)
    st[which + "_param"][at] = par.transpose(1, 2)


def _visible(st, pos):
    """[B,..,n] truth values: whether query t sees the token at pos [B,T,n] (or [B,H,T,n])."""
    mask, T = st["mask"], st["T"]
    n, L = st["n_new"], st["lengths"]
    shape = [-1] + [1] * (pos.dim() - 1)
    first = (L - n).long().view(shape)
    draft = pos - first
    t = torch.arange(T, device=pos.device)[:, None]
    if mask is None:
        seen = draft <= t
    else:
        bits = ((mask[..., None] >> torch.arange(64, device=mask.device)) & 1).flatten(-2)[..., :T].bool()   # [B,T,T]
        bits = bits if pos.dim() == 3 else bits[:, None].expand(-1, pos.shape[1], -1, -1)
        seen = (draft < 0) | bits.gather(-1, draft.clamp(0, T - 1))
    return seen & (pos >= 0) & (pos < L.long().view(shape)) & (t < n.long().view(shape))


def _softmax_product(x, seen, v):
    """softmax of the seen logits x [..,n], times v [..,n,D]; rows that see nothing give 0 and -inf."""
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total == 0, 1.0, total)
    return out, (m + torch.log(total))[..., 0]


def _attend(st, q, index=None):
    """q [B,Hq,T,D]; index: the positions [B,Hkv,T,n] to attend to (all tokens without)."""
    B, Hq, T, D = q.shape
    Hkv = st["Hkv"]
    G = Hq // Hkv
    q = q.float() / math.sqrt(D)
    if index is None:
        pos = torch.arange(st["S"], device=q.device).expand(B, -1)
        k, v = _rows(st, "k", pos), _rows(st, "v", pos)
        x = (q.reshape(B, Hkv, G * T, D) @ k.transpose(-1, -2)).view(B, Hkv, G, T, -1)
        seen = _visible(st, pos[:, None].expand(-1, T, -1))[:, None, None]
        out, lse = _softmax_product(x.reshape(B, Hkv, G * T, -1), seen.expand(-1, Hkv, G, -1, -1).reshape(B, Hkv, G * T, -1), v)
        return out.view(B, Hq, T, D), lse.view(B, Hq, T)
    n = index.shape[-1]
    head = torch.arange(Hkv, device=q.device)[None, :, None].expand(B, -1, T * n)
    flat = index.clamp(min=0).reshape(B, Hkv, T * n)
    batch = torch.arange(B, device=q.device)[:, None, None]
    if st["table"] is None:
        at = (batch, head, flat)
    else:
        block = st["table"].long()[batch, flat // BLOCK]
        at = (block, flat % BLOCK, head)
    k, v = (_values((st[w].view(torch.uint8)[at].view(st[w].dtype) if st["format"] in CODES else st[w][at]),
                    None if st[w + "_param"] is None else st[w + "_param"][at], st["format"]).view(B, Hkv, T, n, D)
            for w in ("k", "v"))
    x = q.reshape(B, Hkv, G, T, D).transpose(2, 3) @ k.transpose(-1, -2)                       # [B,Hkv,T,G,n]
    out, lse = _softmax_product(x, _visible(st, index)[..., None, :], v)
    return out.transpose(2, 3).reshape(B, Hq, T, D), lse.transpose(2, 3).reshape(B, Hq, T)


def _bounds_of(k, live):
    """k [..,unit,D] fp32, live [..,unit] -> 8-bit lowest and highest values [..,2,D] of each block, and its scale."""
    lo = torch.where(live[..., None], k, math.inf).amin(-2)
    hi = torch.where(live[..., None], k, -math.inf).amax(-2)
    lo, hi = (torch.where(live.any(-1)[..., None], x, 0.0) for x in (lo, hi))
    both = torch.stack((lo, hi), -2)
    a = both.abs().amax((-1, -2))
    zero = a < TINY
    codes = (both * torch.where(zero, 0.0, _over(127.0, a))[..., None, None]).round().to(torch.int8)
    return codes, torch.where(zero, 0.0, _over(a, 127.0))


def _refresh(st):
    """The bounds of the blocks that hold the last T tokens."""
    unit, T, B = st["unit"], st["T"], st["q"].shape[0]
    nb = (T - 1) // unit + 2
    last = (st["lengths"].long() - 1) // unit
    block = (last[:, None] - torch.arange(nb - 1, -1, -1, device=last.device)).clamp(min=0)       # [B,nb]
    pos = (block[..., None] * unit + torch.arange(unit, device=last.device)).view(B, -1)
    k = _rows(st, "k", pos.clamp(max=st["S"] - 1)).view(B, st["Hkv"], nb, unit, -1)
    live = (pos < st["lengths"].long()[:, None]).view(B, 1, nb, unit).expand(-1, st["Hkv"], -1, -1)
    codes, scale = _bounds_of(k, live)
    at = (torch.arange(B, device=last.device)[:, None], slice(None), block)
    st["bounds"][at] = codes.transpose(1, 2)
    st["bound_scales"][at] = scale.transpose(1, 2)


def _choose(st):
    """The n_select blocks of each query: the first, the last, and the best by 8-bit bounds; ascending, -1 behind."""
    q, Hkv, T, unit, n = st["q"].float(), st["Hkv"], st["T"], st["unit"], st["n_select"]
    B, Hq, _, D = q.shape
    a = q.abs().amax(-1, keepdim=True)
    zero = a < TINY
    q8 = (q * torch.where(zero, 0.0, _over(127.0, a))).round().reshape(B, Hkv, -1, D)
    sq = torch.where(zero, 0.0, _over(a, 127.0)).reshape(B, Hkv, -1, 1)
    lo, hi = st["bounds"].float().unbind(-2)
    whole = q8.clamp(min=0) @ hi.transpose(-1, -2) + q8.clamp(max=0) @ lo.transpose(-1, -2)       # integers below 2^24
    score = ((whole * st["bound_scales"][..., None, :]) * sq).view(B, Hkv, Hq // Hkv, T, -1).amax(2)   # [B,Hkv,T,Nb]
    nb = ((st["lengths"].long() + unit - 1) // unit).view(-1, 1, 1, 1)
    block = torch.arange(score.shape[-1], device=q.device)
    score = torch.where((block < 1) | (block >= nb - 1), math.inf, score)
    score = torch.where(block < nb, score, -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :n]
    live = (best < nb) & (torch.arange(T, device=q.device)[:, None] < st["n_new"].view(-1, 1, 1, 1))
    got = torch.where(live, best, 1 << 30).sort(-1).values
    got = torch.where(got == 1 << 30, -1, got)
    pad = torch.full((*got.shape[:-1], n - got.shape[-1]), -1, dtype=got.dtype, device=got.device)
    return torch.cat((got, pad), -1).to(torch.int32)


# ------------------------------------------------------------------------------- preparing
def _tree(B, T, g):
    """Random draft trees: each token follows one of those before it; words [B,T,ceil(T/64)] of its ancestors and itself."""
    rng = np.random.RandomState(g)
    seen = np.zeros((B, T, -(-T // 64) * 64), dtype=bool)
    for b in range(B):
        for t in range(T):
            if t and rng.rand() < 0.95:
                seen[b, t] = seen[b, rng.randint(max(0, t - 6), t)]
            seen[b, t, t] = True
    words = np.packbits(seen.reshape(B, T, -1, 64), axis=-1, bitorder="little").view(np.int64)[..., 0]
    return torch.from_numpy(words.copy()).cuda()


def prepare(case, seed):
    c = case
    B, Hkv, S, D, fmt = c["B"], c["Hkv"], c["S"], c["D"], c["format"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    T = c.get("T", 1)
    lengths = torch.full((B,), S, dtype=torch.int32, device="cuda")
    n_new = torch.full((B,), T, dtype=torch.int32, device="cuda")
    if c["ragged"]:
        low = max(T, S // 2)
        lengths[1:] = torch.randint(low, S + 1, (B - 1,), generator=g, device="cuda", dtype=torch.int32)
        if T > 1:
            n_new[1:] = torch.randint(1, T + 1, (B - 1,), generator=g, device="cuda", dtype=torch.int32)
    capacity = -(-S // BLOCK) * BLOCK if c["paged"] else S
    channel = torch.exp(0.5 * torch.randn(2, 1, Hkv, 1, D, generator=g, device="cuda"))   # some channels are larger
    st = {"case": c, "kind": c["kind"], "format": fmt, "Hkv": Hkv, "S": S, "T": T, "D": D, "lengths": lengths, "n_new": n_new,
          "ragged": c["ragged"], "table": None, "mask": None, "dtype": TYPES[c["dtype"]]}
    if c["paged"]:
        blocks = capacity // BLOCK
        st["table"] = torch.randperm(B * blocks, generator=g, device="cuda").to(torch.int32).view(B, blocks)
    for i, w in enumerate(("k", "v")):
        x = torch.randn(B, Hkv, capacity, D, generator=g, device="cuda") * channel[i]
        if c["kind"] == "write":
            st[w + "_new"] = (torch.randn(B, Hkv, T, D, generator=g, device="cuda") * channel[i]).to(TYPES[c["dtype"]])
        if fmt in CODES:
            codes, par = _quantise(x, fmt)
        else:
            codes, par = x.to(TYPES[fmt]), None
        if c["paged"]:
            where = st["table"].view(-1).long()

            def pool(t):
                src = t.view(B, Hkv, blocks, BLOCK, *t.shape[3:]).movedim(1, 3).flatten(0, 1)
                out = torch.empty_like(src, memory_format=torch.contiguous_format)
                out[where] = src
                return out

            codes = pool(codes.view(torch.uint8)).view(codes.dtype) if fmt in CODES else pool(codes)
            par = None if par is None else pool(par)
        st[w], st[w + "_param"] = codes.contiguous(), None if par is None else par.contiguous()
    if c["kind"] == "write":
        first = (lengths - n_new).long()[:, None]
        st["idx"] = torch.minimum(first + torch.arange(T, device="cuda"), lengths.long()[:, None] - 1).to(torch.int32)
    elif c["kind"] == "read":
        st["idx"] = None
        if c["n"]:   # ascending, as a selection leaves them
            order = torch.rand(B, S, generator=g, device="cuda").argsort(1)[:, :c["n"]].sort(1).values
            st["idx"] = (order * lengths.long()[:, None] // S).to(torch.int32)
        shape = (B, Hkv, c["n"] or S, D)
        st["k_out"], st["v_out"] = (torch.zeros(shape, dtype=st["dtype"], device="cuda") for _ in range(2))
    else:
        st["q"] = torch.randn(B, T, c["Hq"], D, generator=g, device="cuda").to(st["dtype"]).transpose(1, 2)  # as projected
        st["mask"] = _tree(B, T, seed % (1 << 31)) if T > 1 else None
    if c["kind"] == "sparse":
        unit = c["unit"]
        nb = -(-capacity // unit)
        st.update(unit=unit, n_select=c["n_select"])
        pos = torch.arange(nb * unit, device="cuda").expand(B, -1)
        k = _rows(st, "k", pos.clamp(max=capacity - 1)).view(B, Hkv, nb, unit, D)
        live = (pos < (lengths - n_new)[:, None]).view(B, 1, nb, unit).expand(-1, Hkv, -1, -1)   # before the new tokens
        st["bounds"], st["bound_scales"] = _bounds_of(k, live)
    return st


# --------------------------------------------------------------------------------- running
def _handle(st):
    """The cache's description and the workspaces, which a program makes once and keeps beside the cache."""
    from paper_2503_00022_amd import binding as kv
    ragged = st["ragged"]
    h = {"kv": kv, "cache": kv.make_cache(st["k"], st["v"], st["S"], k_param=st["k_param"], v_param=st["v_param"],
                                          lengths=st["lengths"] if ragged else None, block_table=st["table"])}
    h["n_new"] = st["n_new"] if ragged and st["T"] > 1 else None
    if st["kind"] in ("attend", "sparse"):
        Hq = st["q"].shape[1]
        n_list = st["n_select"] if st["kind"] == "sparse" else 0
        need = kv.kvcrush_attend_workspace(h["cache"], Hq, st["T"], st["dtype"], n_list=n_list, unit=st.get("unit", 0))
        h["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    if st["kind"] == "sparse":
        need = kv.kvcrush_block_select_workspace(h["cache"], Hq, st["T"], st["dtype"], st["unit"], st["n_select"])
        h["select_ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return h


def _run_own(st):
    h = st.get("handle") or st.setdefault("handle", _handle(st))
    kv, cache, kind = h["kv"], h["cache"], st["kind"]
    if kind == "write":
        kv.kvcrush_cache_write(cache, st["k_new"], st["v_new"], n_new=h["n_new"])
        k, v = kv.kvcrush_cache_read(cache, idx=st["idx"], dtype=st["dtype"])
        return {"k": k, "v": v, "k_param": st["k_param"], "v_param": st["v_param"]}
    if kind == "read":
        k, v = kv.kvcrush_cache_read(cache, idx=st["idx"], k_out=st["k_out"], v_out=st["v_out"])
        return {"k": k, "v": v}
    blocks = None
    if kind == "sparse":
        kv.kvcrush_block_bounds(cache, st["unit"], bounds=st["bounds"], scales=st["bound_scales"], T=st["T"], n_new=h["n_new"])
        blocks = kv.kvcrush_block_select(cache, st["q"], st["bounds"], st["bound_scales"], st["unit"], st["n_select"], n_sink=1,
                                         n_recent=1, n_new=h["n_new"], workspace=h["select_ws"])
    out, lse = kv.kvcrush_attend(cache, st["q"], mask=st["mask"], n_new=h["n_new"], blocks=blocks, unit=st.get("unit", 0),
                                 workspace=h["ws"])
    if kind == "attend":
        return {"out": out, "lse": lse}
    return {"out": out, "lse": lse, "blocks": blocks, "bounds": st["bounds"], "bound_scales": st["bound_scales"]}


def run(st):
    if own:
        return _run_own(st)
    kind, dt = st["kind"], st["dtype"]
    if kind == "write":
        T = st["T"]
        t = torch.arange(T, device="cuda")
        real = st["n_new"].long()[:, None] - 1
        t = torch.minimum(t, real)                             # (padding repeats the last new token's row)
        pos = st["lengths"].long()[:, None] - 1 - real + t
        for w in ("k", "v"):
            x = st[w + "_new"].float().gather(2, t[:, None, :, None].expand(-1, st["Hkv"], -1, st["D"]))
            _store(st, w, pos, *_quantise(x, st["format"]))
        return {"k": _rows(st, "k", st["idx"].long()).to(dt), "v": _rows(st, "v", st["idx"].long()).to(dt),
                "k_param": st["k_param"], "v_param": st["v_param"]}
    if kind == "read":
        B, Hkv, n, D = st["k_out"].shape
        if st["idx"] is not None:
            pos, live = st["idx"].long(), None
        else:
            pos = torch.arange(n, device="cuda").expand(B, -1)
            live = (pos < st["lengths"][:, None])[:, None, :, None]
        for w in ("k", "v"):
            x = _rows(st, w, pos).to(dt)
            st[w + "_out"].copy_(x if live is None else torch.where(live, x, st[w + "_out"]))
        return {"k": st["k_out"], "v": st["v_out"]}
    if kind == "attend":
        out, lse = _attend(st, st["q"])
        return {"out": out.to(dt), "lse": lse}
    _refresh(st)
    blocks = _choose(st)
    pos = blocks.long()[..., None] * st["unit"] + torch.arange(st["unit"], device="cuda")
    pos = torch.where(blocks[..., None] < 0, -1, pos).flatten(-2)
    out, lse = _attend(st, st["q"], torch.where(pos < st["S"], pos, -1))
    return {"out": out.to(dt), "lse": lse, "blocks": blocks, "bounds": st["bounds"], "bound_scales": st["bound_scales"]}


# ----------------------------------------------------------------------- the same in 64 bits
def _exact_row_values(x, fmt):
    """What rows x hold after quantising, and their parameters, in 64 bits.  Which code a value gets is by definition
    settled by an fp32 product (many a bf16 value lies right between two codes); the rest is not rounded."""
    x = x.float()
    if fmt == "i4":
        lo, hi = x.aminmax(dim=-1, keepdim=True)
        y = ((x - lo) * _over(15.0, hi - lo)).double()
        step = (hi.double() - lo) / 15
        return lo + step * torch.round(y), torch.cat((step, lo.double()), -1)
    a = torch.linalg.vector_norm(x, math.inf, dim=-1, keepdim=True)
    y, a = (x * _over(448.0 if fmt == "e4m3" else 127.0, a)).double(), a.double()
    if fmt == "i8":
        return torch.round(y) * a / 127, (a / 127)[..., 0]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * a / 448, (a / 448)[..., 0]


def _exact_cache(st, which, b):
    """The tokens of sequence b, [Hkv,S,D] in 64 bits."""
    fmt = st["format"]
    x, par = st[which], st[which + "_param"]
    if st["table"] is not None:
        order = st["table"][b].long()
        x = (x.view(torch.uint8)[order].view(x.dtype) if fmt in CODES else x[order]).flatten(0, 1).transpose(0, 1)
        par = None if par is None else par[order].flatten(0, 1).transpose(0, 1)
    else:
        x, par = x[b], None if par is None else par[b]
    if fmt == "i4":
        low, high = x % 16, x // 16
        x = torch.stack((low, high), -1).reshape(*x.shape[:-1], -1)
        return x.double() * par[..., 0:1].double() + par[..., 1:2].double()
    return x.double() if par is None else x.to(torch.float32).double() * par.unsqueeze(-1).double()


def exact(case, seed):
    c = case
    B, Hkv, S, D, fmt = c["B"], c["Hkv"], c["S"], c["D"], c["format"]
    if c["kind"] == "sparse" and B * Hkv * S * D > 1 << 28:
        return None                                            # (the scores of so many blocks take the CPU too long)
    st = prepare(case, seed)
    T = st["T"]
    L, N = st["lengths"].tolist(), st["n_new"].tolist()
    if c["kind"] in ("write", "read"):
        got = {"k": [], "v": []}
        pars = {}
        for w in ("k", "v"):
            if c["kind"] == "write":
                values, par = _exact_row_values(st[w + "_new"], fmt)
                pars[w + "_param"] = st[w + "_param"].double()
            for b in range(B):
                x = _exact_cache(st, w, b)
                if c["kind"] == "write":
                    at = slice(L[b] - N[b], L[b])
                    x[:, at] = values[b, :, :N[b]]
                    got[w].append(x[:, st["idx"][b].long()])
                    p = pars[w + "_param"]
                    tokens = torch.arange(at.start, at.stop, device="cuda")
                    if st["table"] is None:
                        p[b, :, tokens] = par[b, :, :N[b]]
                    else:
                        p[st["table"][b, tokens // BLOCK].long(), tokens % BLOCK] = par[b, :, :N[b]].transpose(0, 1)
                elif st["idx"] is not None:
                    got[w].append(x[:, st["idx"][b].long()])
                else:
                    x = x[:, :S].clone()
                    x[:, L[b]:] = 0
                    got[w].append(x)
        return {"k": torch.stack(got["k"]), "v": torch.stack(got["v"]), **pars}
    q = st["q"].double()
    Hq = q.shape[1]
    G = Hq // Hkv
    out = torch.zeros(B, Hq, T, D, dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device="cuda")
    blocks = _exact_blocks(st) if c["kind"] == "sparse" else None
    for b in range(B):
        k, v = _exact_cache(st, "k", b), _exact_cache(st, "v", b)
        seen = torch.zeros(T, S, dtype=torch.bool, device="cuda")
        first = L[b] - N[b]
        seen[:N[b], :first] = True
        among = np.tri(N[b], dtype=bool)
        if st["mask"] is not None:
            words = st["mask"][b].cpu().numpy().view(np.uint8).reshape(T, -1)
            among = np.unpackbits(words, axis=1, bitorder="little")[:N[b], :N[b]].astype(bool)
        seen[:N[b], first:L[b]] = torch.from_numpy(among).cuda()
        for h in range(Hq):
            see = seen
            if blocks is not None:
                see = seen.clone()
                for t in range(T):
                    chosen = blocks[b][h // G][t]
                    keep = torch.zeros(S, dtype=torch.bool, device="cuda")
                    for x in chosen:
                        keep[x * c["unit"]:(x + 1) * c["unit"]] = True
                    see[t] &= keep
            x = (q[b, h] @ k[h // G, :S].t()) / math.sqrt(D)
            x = x.masked_fill(~see, -math.inf)
            total = torch.logsumexp(x, 1)
            p = torch.exp(x - total.clamp(min=-1e300)[:, None])
            out[b, h], lse[b, h] = p @ v[h // G, :S], total
    if blocks is None:
        return {"out": out, "lse": lse}
    return {"out": out, "lse": lse, "blocks": None, "bounds": None, "bound_scales": st["exact_scales"]}


def _exact_blocks(st):
    """Lists of the chosen blocks by sequence, KV head and query; the scores are fp32 values by definition (an exact
    integer times two scales), and so they are formed here."""
    unit, D, Hkv, T = st["unit"], st["D"], st["Hkv"], st["T"]
    q = st["q"].cpu().numpy() if st["dtype"] == torch.float32 else st["q"].float().cpu().numpy()
    G = q.shape[1] // Hkv
    a = np.abs(q).max(-1, keepdims=True)
    q8, sq = np.rint(q * (np.float32(127) / a)).astype(np.int64), (a / np.float32(127))[..., 0]
    chosen = []
    st["exact_scales"] = st["bound_scales"].double()
    for b in range(st["lengths"].numel()):
        L, N = int(st["lengths"][b]), int(st["n_new"][b])
        nb = -(-L // unit)
        k = _exact_cache(st, "k", b)[:, :L].float().cpu().numpy()
        bounds = st["bounds"][b].cpu().numpy().astype(np.int64)
        scales = st["bound_scales"][b].cpu().numpy().copy()
        for n in range((L - N) // unit, nb):
            part = k[:, n * unit:(n + 1) * unit]
            lo, hi = part.min(1), part.max(1)
            top = np.maximum(np.abs(lo), np.abs(hi)).max(-1)
            bounds[:, n, 0], bounds[:, n, 1] = (np.rint(x * (np.float32(127) / top)[:, None]).astype(np.int64) for x in (lo, hi))
            scales[:, n] = top / np.float32(127)
            st["exact_scales"][b, :, n] = torch.from_numpy(top.astype(np.float64) / 127).cuda()
        rows = []
        for g in range(Hkv):
            row = []
            for t in range(T):
                x = q8[b, g * G:(g + 1) * G, t]
                whole = np.maximum(x, 0) @ bounds[g, :nb, 1].T + np.minimum(x, 0) @ bounds[g, :nb, 0].T     # [G,nb]
                score = ((whole.astype(np.float32) * scales[g, :nb]) * sq[b, g * G:(g + 1) * G, t, None]).max(0)
                score[0] = score[nb - 1] = np.inf
                row.append(sorted(np.argsort(-score, kind="stable")[:st["n_select"]].tolist()) if t < N else [])
            rows.append(row)
        chosen.append(rows)
    return chosen


# ------------------------------------------------------------------------------------ work
def work(case):
    c = case
    B, Hkv, S, D, fmt = c["B"], c["Hkv"], c["S"], c["D"], c["format"]
    T = c.get("T", 1)
    value = BITS[c["dtype"]] / 8
    row = D * BITS[fmt] / 8 + PARAMS[fmt]                      # bytes of a cached row
    tokens = S if not c["ragged"] or B == 1 else (S + (B - 1) * (max(T, S // 2) + S) / 2) / B
    if c["kind"] == "write":                                   # values in, rows out and in again, values out
        new = T if not c["ragged"] or B == 1 or T == 1 else (T + (B - 1) * (T + 1) / 2) / B
        return {"bytes": 2 * B * Hkv * new * 2 * (D * value + row), "flops": 0}
    if c["kind"] == "read":
        n = c["n"] or tokens
        return {"bytes": 2 * B * Hkv * n * (D * value + row), "flops": 0}
    Hq = c["Hq"]
    ends = B * Hq * T * (2 * D * value + 4)                    # q, out, lse
    if c["kind"] == "attend":
        return {"bytes": 2 * B * Hkv * tokens * row + ends, "flops": 4 * B * Hq * T * tokens * D}
    n = min(c["n_select"] * c["unit"], tokens)
    blocks = tokens / c["unit"]
    return {"bytes": B * Hkv * (2 * T * n * row + blocks * (2 * D + 4) + 4 * T * c["n_select"]) + ends,
            "flops": 4 * B * Hq * T * (n * D + blocks * D)}
