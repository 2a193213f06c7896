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
