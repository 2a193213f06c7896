"""Host-side refusals of the calls that use a KV cache: bad arguments are turned down before anything is launched, through
the C entry points and through the binding (no call here reaches a launch; no GPU is needed)."""
import ctypes

import pytest
import torch

from paper_2503_00022_amd import binding as kv

FAKE = 0x10000                       # aligned, never dereferenced
ODD = 0x10008
BIG = 1 << 50
OK, INVALID, UNSUPPORTED, WORKSPACE = kv.OK, kv.ERR_INVALID_ARG, kv.ERR_UNSUPPORTED, kv.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    from paper_2503_00022_amd import build
    build.ensure_built()
    return kv.load()


GOOD = dict(B=2, Hkv=2, S=100, D=128, capacity=128, format=kv.I8, block_size=0, n_blocks=0, k=FAKE, v=FAKE, k_param=FAKE,
            v_param=FAKE, lengths=None, block_table=None)
PAGED = dict(GOOD, block_table=FAKE, block_size=16, n_blocks=50)


def cache(base=GOOD, **kw):
    d = dict(base, **kw)
    return kv.Cache(*(d[n] for n, _ in kv.Cache._fields_))


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def write(lib, c=None, T=4, dtype=kv.BF16, k=FAKE, v=FAKE, ks=None, vs=None, **kw):
    return lib.kvcrush_cache_write(ctypes.byref(cache(**kw) if c is None else c), T, dtype, k, v, ks, vs, None, None)


def read(lib, n=4, idx=FAKE, dtype=kv.BF16, k=FAKE, v=FAKE, **kw):
    return lib.kvcrush_cache_read(ctypes.byref(cache(**kw)), n, idx, dtype, k, v, None)


def attend_args(Hq=4, T=4, dtype=kv.BF16, scale=0.0, q_stride=(0, 0, 0), out_stride=(0, 0, 0), mask=None, mask_stride=0, n_new=None,
                blocks=None, n_list=0, unit=0):
    return kv.AttendArgs(Hq, T, dtype, scale, strides(*q_stride), strides(*out_stride), mask, mask_stride, n_new, blocks, n_list, unit)


def attend(lib, c=None, args=None, q=FAKE, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=BIG, **kw):
    return lib.kvcrush_attend(ctypes.byref(c or cache()), ctypes.byref(args or attend_args(**kw)), q, out, lse, ws, ws_bytes, None)


BAD_CACHES = [
    (dict(B=0), INVALID), (dict(Hkv=0), INVALID), (dict(S=-1), INVALID), (dict(S=129), INVALID), (dict(capacity=0, S=0), INVALID),
    (dict(format=6), INVALID), (dict(format=-1), INVALID), (dict(D=0), INVALID), (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED), (dict(capacity=(1 << 29) + 1), UNSUPPORTED),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=ODD), INVALID), (dict(v=ODD), INVALID), (dict(k_param=None), INVALID),
    (dict(v_param=None), INVALID), (dict(v_param=ODD), INVALID)]
BAD_PAGED = [(dict(block_size=0), INVALID), (dict(n_blocks=0), INVALID), (dict(block_size=24), INVALID),
             (dict(n_blocks=1 << 27), UNSUPPORTED)]


@pytest.mark.parametrize("base,change,status", [(GOOD, c, s) for c, s in BAD_CACHES] + [(PAGED, c, s) for c, s in BAD_PAGED])
def test_caches_that_are_refused(lib, base, change, status):
    c = cache(base, **change)
    assert write(lib, c) == status
    assert lib.kvcrush_cache_read(ctypes.byref(c), 4, FAKE, kv.BF16, FAKE, FAKE, None) == status
    args = attend_args()
    assert attend(lib, c, args) == status
    assert lib.kvcrush_attend_workspace(ctypes.byref(c), ctypes.byref(args)) == 0
    assert lib.kvcrush_block_bounds(ctypes.byref(c), 16, 0, None, FAKE, FAKE, None) == status
    assert lib.kvcrush_block_select(ctypes.byref(c), ctypes.byref(args), 16, 4, 1, 1, FAKE, FAKE, FAKE, FAKE, FAKE, BIG, None) == status
    assert lib.kvcrush_block_select_workspace(ctypes.byref(c), ctypes.byref(args), 16, 4) == 0


def test_null_structs(lib):
    assert lib.kvcrush_cache_write(None, 4, kv.BF16, FAKE, FAKE, None, None, None, None) == INVALID
    assert lib.kvcrush_cache_read(None, 4, None, kv.BF16, FAKE, FAKE, None) == INVALID
    assert lib.kvcrush_attend(None, ctypes.byref(attend_args()), FAKE, FAKE, FAKE, FAKE, BIG, None) == INVALID
    assert lib.kvcrush_attend(ctypes.byref(cache()), None, FAKE, FAKE, FAKE, FAKE, BIG, None) == INVALID
    assert lib.kvcrush_block_select(ctypes.byref(cache()), None, 16, 4, 1, 1, FAKE, FAKE, FAKE, FAKE, FAKE, BIG, None) == INVALID


def test_write_and_read_refusals(lib):
    assert write(lib, T=-1) == INVALID and write(lib, dtype=3) == INVALID
    assert write(lib, k=None) == INVALID and write(lib, v=ODD) == INVALID
    assert write(lib, T=0, k=None, v=None) == OK                                  # nothing to do
    assert write(lib, S=0, k=None, v=None) == OK
    assert read(lib, n=(1 << 29) + 1) == UNSUPPORTED
    assert write(lib, ks=strides(512, 128, 130)) == INVALID                       # not a multiple of 16 bytes
    assert write(lib, vs=strides(512, -128, 128)) == INVALID
    assert write(lib, vs=strides(1 << 42, 128, 128)) == INVALID
    assert write(lib, format=kv.BF16, dtype=kv.F16) == INVALID                    # a plain cache takes its own type
    assert write(lib, B=40000) == UNSUPPORTED and write(lib, Hkv=70000) == UNSUPPORTED
    assert read(lib, n=-1) == INVALID and read(lib, n=129, idx=None) == INVALID and read(lib, dtype=5) == INVALID
    assert read(lib, k=None) == INVALID and read(lib, v=ODD) == INVALID
    assert read(lib, format=kv.F32, dtype=kv.BF16) == INVALID
    assert read(lib, n=0, k=None, v=None) == OK
    assert read(lib, B=40000) == UNSUPPORTED


def test_attend_refusals(lib):
    assert attend(lib, Hq=5) == INVALID and attend(lib, Hq=0) == INVALID and attend(lib, T=0) == INVALID
    assert attend(lib, T=1025) == UNSUPPORTED and attend(lib, cache(B=5000), T=1024) == UNSUPPORTED
    assert attend(lib, dtype=kv.F32) == INVALID                                   # float queries on a quantised cache
    assert attend(lib, cache(format=kv.F16), dtype=kv.BF16) == INVALID
    assert attend(lib, dtype=4) == INVALID
    assert attend(lib, scale=-1.0) == INVALID and attend(lib, scale=float("nan")) == INVALID and attend(lib, scale=1e9) == INVALID
    assert attend(lib, q=None) == INVALID and attend(lib, out=None) == INVALID and attend(lib, q=ODD) == INVALID
    assert attend(lib, out=ODD) == INVALID and attend(lib, lse=ODD) == INVALID
    assert attend(lib, q_stride=(2048, 512, 12)) == INVALID
    assert attend(lib, out_stride=(2048, 512, 0)) == INVALID                      # rows of an output must not overlap
    assert attend(lib, out_stride=(2048, 512, 64)) == INVALID
    assert attend(lib, mask=FAKE, mask_stride=-1) == INVALID
    assert attend(lib, blocks=FAKE, n_list=0, unit=16) == INVALID and attend(lib, blocks=FAKE, n_list=4, unit=0) == INVALID
    assert attend(lib, blocks=FAKE, n_list=1 << 20, unit=1 << 10) == UNSUPPORTED
    assert attend(lib, cache(B=70000)) == UNSUPPORTED
    long = cache(S=100000, capacity=100000)
    need = lib.kvcrush_attend_workspace(ctypes.byref(long), ctypes.byref(attend_args()))
    assert need > 0
    assert attend(lib, long, ws=None) == WORKSPACE and attend(lib, long, ws=ODD) == WORKSPACE
    assert attend(lib, long, ws_bytes=need - 1) == WORKSPACE
    sizes = [lib.kvcrush_attend_workspace(ctypes.byref(cache(S=s, capacity=100000)), ctypes.byref(attend_args()))
             for s in (0, 1, 100, 1000, 10000, 50000, 100000)]
    assert sizes == sorted(sizes)                                                 # a growing cache needs no less


@pytest.mark.parametrize("B,Hkv,Hq,T,D,fmt,lengths", [
    (1, 8, 32, 1, 128, kv.BF16, None), (3, 5, 10, 1, 64, kv.I4, FAKE), (1, 1, 4, 40, 128, kv.I8, None), (7, 8, 8, 3, 128, kv.E4M3, FAKE),
    (40, 4, 8, 1, 64, kv.F16, FAKE), (2, 2, 64, 5, 128, kv.F32, None)])
def test_a_growing_cache_never_needs_less_scratch_memory(lib, B, Hkv, Hq, T, D, fmt, lengths):
    """A workspace sized for the capacity serves every length on the way there."""
    args = attend_args(Hq=Hq, T=T, dtype=kv.BF16 if fmt > 2 else fmt)
    sizes = [lib.kvcrush_attend_workspace(ctypes.byref(cache(B=B, Hkv=Hkv, D=D, format=fmt, S=s, capacity=40000, lengths=lengths)),
                                          ctypes.byref(args)) for s in [*range(0, 6000, 7), *range(6000, 40000, 331)]]
    assert sizes == sorted(sizes) and sizes[-1] > 0


def test_block_refusals(lib):
    def bounds(c=None, unit=16, T=0, b=FAKE, s=FAKE):
        return lib.kvcrush_block_bounds(ctypes.byref(c or cache()), unit, T, None, b, s, None)

    def select(c=None, unit=16, n=4, sink=1, recent=1, q=FAKE, b=FAKE, s=FAKE, out=FAKE, ws=FAKE, ws_bytes=BIG, **kw):
        return lib.kvcrush_block_select(ctypes.byref(c or cache()), ctypes.byref(attend_args(**kw)), unit, n, sink, recent, q, b, s, out,
                                        ws, ws_bytes, None)

    assert bounds(unit=0) == INVALID and bounds(T=-1) == INVALID and bounds(b=None) == INVALID and bounds(s=ODD) == INVALID
    assert bounds(unit=1025) == UNSUPPORTED and bounds(cache(B=70000)) == UNSUPPORTED
    big = dict(base=dict(GOOD, B=1, Hkv=1, S=0, capacity=1 << 29))                  # 2^26 and 2^25 blocks
    assert bounds(cache(**big), unit=8) == UNSUPPORTED and bounds(cache(**big), unit=16) == OK
    assert select(n=32769) == UNSUPPORTED and select(n=2 ** 31 - 1) == UNSUPPORTED
    assert bounds(cache(S=0)) == OK                                               # an empty cache has no blocks
    assert select(unit=0) == INVALID and select(n=0) == INVALID and select(sink=-1) == INVALID and select(sink=3, recent=2) == INVALID
    assert select(sink=2 ** 31 - 1, recent=2 ** 31 - 1) == INVALID
    assert select(q=None) == INVALID and select(b=ODD) == INVALID and select(s=None) == INVALID and select(out=ODD) == INVALID
    assert select(Hq=3) == INVALID and select(T=1025) == UNSUPPORTED and select(q_stride=(1, 1, 1)) == INVALID
    assert select(cache(Hkv=1), Hq=1025) == UNSUPPORTED and select(cache(B=2000), T=1024) == UNSUPPORTED
    assert select(cache(S=40000, capacity=40000), unit=1) == UNSUPPORTED
    need = lib.kvcrush_block_select_workspace(ctypes.byref(cache()), ctypes.byref(attend_args()), 1, 4)
    assert need >= 2 * 2 * 4 * 100 * 4
    assert select(unit=1, ws=None) == WORKSPACE and select(unit=1, ws_bytes=need - 1) == WORKSPACE and select(unit=1, ws=ODD) == WORKSPACE


def test_one_row_for_all_is_not_taken_for_a_packed_tensor():
    """Three zero strides mean packed to the library, which would read far behind the row."""
    row = torch.zeros(1, 1, 1, 64)
    with pytest.raises(ValueError, match="contiguous"):
        kv._strides(row.expand(2, 3, 4, 64))
    assert kv._strides(row.expand(2, 3, 1, 64)) == (0, 0, 64)       # an axis of one element has its packed stride
    assert kv._strides(row.expand(1, 3, 4, 64)) == (3 * 4 * 64, 0, 0)
    assert kv._strides(row) is None


def test_scratch_memory_is_as_large_as_it_says():
    one = torch.zeros(1, dtype=torch.uint8)
    with pytest.raises(ValueError, match="contiguous"):
        kv._scratch(one.expand(1 << 20), one.get_device())
    with pytest.raises(ValueError, match="GPU memory"):
        kv._scratch(one, 0)
    kv._scratch(one, one.get_device())


def test_binding_refuses_host_memory_and_wrong_shapes():
    k = torch.zeros(2, 2, 32, 64, dtype=torch.int8)
    with pytest.raises(ValueError, match="GPU memory"):
        kv.make_cache(k, k, 10)
    c = cache()
    c.tensors, c.device, c.index, c.value_dtype, c.per_sequence = (), torch.device("cuda", 0), 0, torch.bfloat16, (2,)
    with pytest.raises(ValueError, match="GPU memory"):
        kv.kvcrush_attend(c, torch.zeros(2, 4, 1, 128))
    with pytest.raises(ValueError, match="GPU memory"):
        kv.kvcrush_cache_write(c, torch.zeros(2, 2, 1, 128), torch.zeros(2, 2, 1, 128))
    with pytest.raises(ValueError, match="GPU memory"):
        kv.kvcrush_cache_read(c, idx=torch.zeros(2, 3))
    with pytest.raises(ValueError, match="unit"):
        kv.kvcrush_block_bounds(c, 0)
    with pytest.raises(ValueError, match="together"):
        kv.kvcrush_block_bounds(c, 16, T=3)
