"""What the calls that use a KV cache compute, in plain numpy / torch on the CPU: rows by their definition (fp32, one
rounding per operation), attention and block scores in 64 bits.  Nothing of the library is used."""
import math

import numpy as np
import torch

FORMATS = ["bf16", "f16", "f32", "e4m3", "i8", "i4"]
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
STORED = {**DTYPES, "e4m3": torch.float8_e4m3fn, "i8": torch.int8, "i4": torch.uint8}
F = np.float32
TINY = F(2.0 ** -100)


def quantise(x, fmt):
    """x float32 array [.., D] -> (whole codes or e4m3 values as float32 [.., D], parameters [..] or [.., 2])."""
    x = np.asarray(x, dtype=F)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(x).all(-1)
        if fmt == "i4":
            lo, hi = x.min(-1), x.max(-1)
            d = hi - lo
            bad |= ~np.isfinite(d)
            flat = d < TINY
            inv = np.where(flat | bad, F(0), F(15) / d)
            codes = np.where(bad[..., None], F(0), np.rint((x - lo[..., None]) * inv[..., None]))
            par = np.stack((np.where(flat, F(0), d / F(15)), lo), -1)
            par[bad] = np.nan
            return codes.astype(F), par.astype(F)
        top = F(448) if fmt == "e4m3" else F(127)
        a = np.abs(x).max(-1)
        zero = a < TINY
        inv = np.where(zero | bad, F(0), top / a)
        y = np.where(bad[..., None], F(0), x * inv[..., None]).astype(F)
        codes = np.rint(y) if fmt == "i8" else torch.from_numpy(y).to(torch.float8_e4m3fn).float().numpy()
        par = np.where(zero, F(0), a / top)
        par[bad] = np.nan
        return codes.astype(F), par.astype(F)


def values32(codes, par, fmt):
    """The rows' values in fp32, rounded once."""
    if fmt == "i4":
        with np.errstate(all="ignore"):
            return (codes.astype(np.float64) * par[..., :1] + par[..., 1:]).astype(F)
    return codes if par is None else (codes * par[..., None]).astype(F)


def values64(codes, par, fmt):
    codes = codes.astype(np.float64)
    if fmt == "i4":
        return codes * par[..., :1].astype(np.float64) + par[..., 1:].astype(np.float64)
    return codes if par is None else codes * par[..., None].astype(np.float64)


def store(codes, fmt):
    """Codes as the cache holds them."""
    t = torch.from_numpy(codes)
    if fmt == "i4":
        c = t.to(torch.uint8)
        return c[..., 0::2] | (c[..., 1::2] << 4)
    return t.to(STORED[fmt])


def load(t, fmt):
    """The codes (or values) of stored rows, float32."""
    t = t.cpu()
    if fmt == "i4":
        t = torch.stack((t & 15, t >> 4), -1).flatten(-2)
    return t.float().numpy()


class Case:
    """A cache with random rows: dense or paged, its true rows kept beside it.  Everything that no call may read (rows at and
    beyond a length, blocks of no sequence) holds NaN or, as codes, 0x7F bytes."""

    def __init__(self, fmt, B, Hkv, lengths, D, capacity=None, block_size=0, seed=0, magnitude=1.0, room=0):
        rng = np.random.RandomState(seed)
        self.fmt, self.B, self.Hkv, self.D, self.lengths, self.block_size = fmt, B, Hkv, D, list(lengths), block_size
        capacity = max(max(lengths), 1) + room if capacity is None else capacity
        if block_size:
            capacity = -(-capacity // block_size) * block_size
        self.capacity = capacity
        self.table = None
        tensors, self.rows64 = {}, {}
        if block_size:
            per = capacity // block_size
            self.n_blocks = B * per + 3
            self.table = torch.from_numpy(rng.permutation(self.n_blocks)[:B * per].astype(np.int32)).view(B, per)
        for w in ("k", "v"):
            x = (rng.randn(B, Hkv, capacity, D) * magnitude * np.exp(0.5 * rng.randn(1, Hkv, 1, D))).astype(F)
            if fmt in DTYPES:
                x = torch.from_numpy(x).to(DTYPES[fmt]).float().numpy()
                codes, par = x, None
            else:
                codes, par = quantise(x, fmt)
            self.rows64[w] = values64(codes, par, fmt)
            t, p = store(codes, fmt), None if par is None else torch.from_numpy(par)
            self._poison(t, p)
            if block_size:
                t, p = self._pool(t), None if p is None else self._pool(p)
            tensors[w], tensors[w + "_param"] = t, p
        self.tensors = tensors

    def _poison(self, t, p, only=None):
        for b in range(self.B):
            rows = slice(self.lengths[b], None) if only is None else only[b]
            if t.dtype.is_floating_point and t.dtype != torch.float8_e4m3fn:
                t[b, :, rows] = math.nan
            else:
                t.view(torch.uint8)[b, :, rows] = 0x7F
            if p is not None:
                p[b, :, rows] = math.nan

    def _pool(self, t):
        raw = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
        pool = torch.zeros(self.n_blocks, self.block_size, self.Hkv, *raw.shape[3:], dtype=raw.dtype)
        pool.fill_(math.nan) if raw.dtype.is_floating_point else pool.fill_(0x7F)
        for b in range(self.B):
            for i, blk in enumerate(self.table[b].tolist()):
                pool[blk] = raw[b, :, i * self.block_size:(i + 1) * self.block_size].movedim(0, 1)
        return pool.view(t.dtype)

    def dense(self, name):
        """The tensor `name` (k, v, k_param, v_param) as the dense layout shows it, from wherever it is now."""
        t = self.tensors[name]
        t = None if t is None else t.cpu()
        if t is None or self.table is None:
            return t
        raw = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
        out = torch.stack([raw[self.table[b].long()].flatten(0, 1).movedim(1, 0) for b in range(self.B)])
        return out.view(t.dtype)

    def cuda(self):
        self.tensors = {k: None if t is None else t.cuda() for k, t in self.tensors.items()}
        return self

    def make(self, kv, use_lengths=True, S=None):
        t = self.tensors
        lengths = torch.tensor(self.lengths, dtype=torch.int32, device="cuda") if use_lengths else None
        S = S if S is not None else self.capacity if use_lengths else self.lengths[0]
        table = None if self.table is None else self.table.cuda()
        return kv.make_cache(t["k"], t["v"], S, t["k_param"], t["v_param"], lengths, table)


def tree(T, rng, roots=0.1):
    """A draft tree as truth values [T,T]: each token sees its ancestors and itself."""
    seen = np.zeros((T, T), dtype=bool)
    for t in range(T):
        if t and rng.rand() > roots:
            seen[t] = seen[rng.randint(max(0, t - 5), t)]
        seen[t, t] = True
    return seen


def mask_words(seen):
    """Truth values [.., T, T] -> int64 words [.., T, ceil(T / 64)]."""
    T = seen.shape[-1]
    wide = np.zeros((*seen.shape[:-1], -(-T // 64) * 64), dtype=bool)
    wide[..., :T] = seen
    words = np.packbits(wide, axis=-1, bitorder="little").view(np.int64)
    return torch.from_numpy(words.copy())


def attend(q, k, v, lengths, n_new, seen=None, scale=None, lists=None, unit=1):
    """q [B,Hq,T,D], k and v [B,Hkv,capacity,D] (64 bits) -> out, lse, and sum of probability x |v|, |logits| at most.
    lists[b][kv head][t]: blocks, or None."""
    B, Hq, T, D = q.shape
    G = Hq // k.shape[1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, absolute = np.zeros((B, Hq, T, D)), np.zeros((B, Hq, T, D))
    lse, size = np.full((B, Hq, T), -np.inf), np.zeros((B, Hq, T))
    for b in range(B):
        L, n = lengths[b], n_new[b]
        for t in range(n):
            see = np.zeros(L, dtype=bool)
            see[:L - n] = True
            see[L - n:] = (seen[b, t, :n] if seen is not None else np.arange(n) <= t)
            for h in range(Hq):
                at = np.nonzero(see)[0]
                if lists is not None:
                    at = at[np.isin(at // unit, lists[b][h // G][t])]
                if not len(at):
                    continue
                x = scale * (k[b, h // G, at] @ q[b, h, t])
                size[b, h, t] = scale * (np.abs(k[b, h // G, at]) @ np.abs(q[b, h, t])).max()
                m = x.max()
                p = np.exp(x - m)
                lse[b, h, t] = m + math.log(p.sum())
                p /= p.sum()
                out[b, h, t] = p @ v[b, h // G, at]
                absolute[b, h, t] = p @ np.abs(v[b, h // G, at])
    return out, lse, absolute, size


def bounds(k32, length, unit, n_blocks):
    """k32 [Hkv,capacity,D] float32 -> (int8 values [Hkv,n_blocks,2,D], scales): blocks without tokens are zero."""
    Hkv, _, D = k32.shape
    out, scales = np.zeros((Hkv, n_blocks, 2, D), dtype=np.int64), np.zeros((Hkv, n_blocks), dtype=F)
    for i in range(-(-length // unit)):
        part = k32[:, i * unit:min((i + 1) * unit, length)]
        both = np.stack((part.min(1), part.max(1)), 1)                     # [Hkv,2,D]
        a = np.abs(both).max((1, 2))
        inv = np.where(a < TINY, F(0), F(127) / np.maximum(a, TINY))
        out[:, i] = np.rint(both * inv[:, None, None])
        scales[:, i] = np.where(a < TINY, F(0), a / F(127))
    return out, scales


def choose(q32, bnd, scales, length, unit, n_select, n_sink, n_recent):
    """q32 [G,D] float32 of one query and KV head, its blocks' bounds [Nb,2,D] and scales -> ascending list."""
    nb = -(-length // unit)
    a = np.abs(q32).max(-1)
    inv = np.where(a < TINY, F(0), F(127) / np.maximum(a, TINY))
    sq = np.where(a < TINY, F(0), a / F(127))
    q8 = np.rint(q32 * inv[:, None]).astype(np.int64)
    whole = np.maximum(q8, 0) @ bnd[:nb, 1].T + np.minimum(q8, 0) @ bnd[:nb, 0].T
    score = ((whole.astype(F) * scales[None, :nb]) * sq[:, None]).max(0)
    score[:n_sink] = np.inf
    if n_recent:
        score[max(nb - n_recent, 0):] = np.inf
    return sorted(np.argsort(-score, kind="stable")[:n_select].tolist())
