"""What the norms, rotations and the attention of new tokens refuse, and sizes: host code alone, on a context and buffers that are never used."""
import ctypes
import math

import pytest

import paper_1910_00178_amd as ng

INVALID, SHAPE, SMALL = ng.NGEMM_ERR_INVALID_ARG, ng.NGEMM_ERR_BAD_SHAPE, ng.NGEMM_ERR_BUFFER_TOO_SMALL
HERE = 0x10000                                           # an address that nothing reads: all calls below are refused or have nothing to do


class Context(ctypes.Structure):                         # the head of the library's own
    _fields_ = [("magic", ctypes.c_uint32), ("device", ctypes.c_int), ("rest", ctypes.c_char * 256)]


def context(device=0):
    c = Context(0x4e47454d, device)
    return c, ctypes.c_void_p(ctypes.addressof(c))


@pytest.fixture
def ctx():
    c, p = context()
    yield p
    del c


def refused(status, fn, *args):
    with pytest.raises(ng.binding.NgemmError) as e:
        fn(*args)
    assert e.value.status == status


def test_rotation(ctx):
    assert ng.ngemm_rotation_bytes(100, 64) == 100 * 64 * 4 and ng.ngemm_rotation_bytes(1 << 30, 256) == 1 << 40
    create = ng.ngemm_rotation_create
    for positions, dim in ((0, 64), (-1, 64), ((1 << 30) + 1, 64), (100, 0), (100, 8), (100, 24), (100, 272), (100, -16)):
        assert ng.ngemm_rotation_bytes(positions, dim) == 0
        refused(SHAPE, create, ctx, positions, dim, 0, HERE, 1 << 60)
    refused(INVALID, create, None, 100, 64, 0, HERE, 25600)
    refused(INVALID, create, ctx, 100, 64, 2, HERE, 25600)
    refused(INVALID, create, ctx, 100, 64, -1, HERE, 25600)
    refused(INVALID, create, ctx, 100, 64, 0, None, 25600)
    refused(INVALID, create, ctx, 100, 64, 0, HERE + 4, 25600)
    refused(SMALL, create, ctx, 100, 64, 0, HERE, 25599)
    r = create(ctx, 100, 64, 1, HERE, 25600)
    ng.ngemm_rotation_free(r)
    ng.ngemm_rotation_free(None)
    refused(INVALID, ng.ngemm_rotation_free, ctx)


def test_norm_rotate(ctx):
    r = ng.ngemm_rotation_create(ctx, 100, 64, 0, HERE, 25600)
    _keep, other = context(1)
    elsewhere = ng.ngemm_rotation_create(other, 100, 64, 0, HERE, 25600)

    def call(ctx=ctx, type=ng.NGEMM_BF16, dim=64, tokens=8, hq=4, q=HERE, qt=256, qh=64, wq=HERE, hk=2, k=HERE, kt=128, kh=64, wk=HERE, eps=1e-6, r=r, at=HERE,
             qo=HERE, qot=256, qoh=64, ko=HERE, kot=128, koh=64):
        return ng.ngemm_qk_norm_rotate, ctx, type, dim, tokens, hq, q, qt, qh, wq, hk, k, kt, kh, wk, eps, r, at, qo, qot, qoh, ko, kot, koh, HERE

    for status, bad in ((INVALID, {"ctx": None}), (INVALID, {"type": 3}), (INVALID, {"type": -1}), (SHAPE, {"dim": 24}), (SHAPE, {"dim": 272}), (SHAPE, {"dim": 0}),
                        (SHAPE, {"tokens": -1}), (SHAPE, {"tokens": 1 << 31}), (SHAPE, {"hq": -1}), (SHAPE, {"hk": 65537}), (INVALID, {"q": None}), (INVALID, {"k": None}),
                        (INVALID, {"qo": None}), (INVALID, {"ko": None}), (INVALID, {"q": HERE + 1}), (INVALID, {"ko": HERE + 1}), (INVALID, {"wq": HERE + 2}),
                        (INVALID, {"wk": HERE + 1}), (SHAPE, {"qt": -1}), (SHAPE, {"kh": -1}), (SHAPE, {"qot": 64}), (SHAPE, {"koh": 0}), (SHAPE, {"qoh": 63}),
                        (SHAPE, {"qt": (1 << 40) + 1}), (SHAPE, {"tokens": 1 << 30, "qt": 1 << 31}), (INVALID, {"eps": -1e-6}), (INVALID, {"eps": math.nan}),
                        (INVALID, {"eps": math.inf}), (INVALID, {"at": None}), (INVALID, {"r": ctx}), (INVALID, {"r": elsewhere}), (SHAPE, {"dim": 48}),
                        (SHAPE, {"tokens": 1 << 30, "hq": 65536, "qt": 0, "qh": 0, "qot": 65536 * 64})):
        refused(status, *call(**bad))
    for nothing in ({"tokens": 0}, {"hq": 0, "hk": 0}, {"tokens": 0, "q": None, "k": None, "qo": None, "ko": None, "at": None}):
        fn, *args = call(**nothing)
        fn(*args)
    # a side without heads: its weights are not looked at (what is refused is the other side's size)
    for unused in ({"hk": 0, "wk": HERE + 1}, {"hq": 0, "hk": 65536, "wq": HERE + 1}):
        refused(SHAPE, *call(**({"tokens": 1 << 30, "hq": 65536, "qt": 0, "qh": 0, "kt": 0, "kh": 0, "qot": 65536 * 64, "kot": 65536 * 64} | unused)))
    for x in (r, elsewhere):
        ng.ngemm_rotation_free(x)


def cache_of(ctx, kv_heads=2, head_dim=64):
    size = ng.ngemm_kv_cache_bytes(4, 16, kv_heads, head_dim)
    return ng.ngemm_kv_cache_create(ctx, 4, 16, kv_heads, head_dim, HERE, size)


def test_write(ctx):
    c = cache_of(ctx)
    r, wide = (ng.ngemm_rotation_create(ctx, 100, dim, 0, HERE, 1 << 20) for dim in (64, 80))
    _keep, other = context(1)
    elsewhere = ng.ngemm_rotation_create(other, 100, 64, 0, HERE, 25600)

    def call(ctx=ctx, c=c, type=ng.NGEMM_BF16, batch=1, tokens=8, k=HERE, kt=128, kh=64, v=HERE, vt=128, vh=64, w=HERE, eps=1e-6, r=r, off=HERE, pages=HERE, stride=1):
        return ng.ngemm_kv_write_rotated, ctx, c, type, batch, tokens, k, kt, kh, v, vt, vh, w, eps, r, off, None, pages, stride, HERE

    for status, bad in ((INVALID, {"ctx": None}), (INVALID, {"c": None}), (INVALID, {"c": ctx}), (INVALID, {"ctx": other}), (INVALID, {"type": 3}), (SHAPE, {"batch": -1}),
                        (SHAPE, {"batch": 0}), (SHAPE, {"tokens": -1}), (SHAPE, {"tokens": 1 << 31}), (INVALID, {"k": None}), (INVALID, {"v": None}), (INVALID, {"off": None}),
                        (INVALID, {"pages": None}), (SHAPE, {"kt": -1}), (SHAPE, {"vh": -64}), (SHAPE, {"stride": -1}), (INVALID, {"k": HERE + 1}), (INVALID, {"w": HERE + 1}),
                        (INVALID, {"eps": -1.0}), (INVALID, {"eps": math.nan}), (INVALID, {"r": c}), (INVALID, {"r": elsewhere}), (SHAPE, {"r": wide})):
        refused(status, *call(**bad))
    fn, *args = call(tokens=0)
    fn(*args)
    for x in (r, wide, elsewhere):
        ng.ngemm_rotation_free(x)
    ng.ngemm_kv_cache_free(c)


def test_chunk(ctx):
    c = cache_of(ctx)
    _keep, other = context(1)

    def call(ctx=ctx, c=c, type=ng.NGEMM_BF16, batch=2, heads=4, tokens=8, q=HERE, qt=256, qh=64, off=HERE, start=HERE, new=8, longest=16, pages=HERE, stride=1,
             window=0, sinks=0, scale=0.1, o=HERE, ot=256, oh=64, ws=HERE, wsb=1 << 40):
        return (ng.ngemm_attention_chunk, ctx, c, type, batch, heads, tokens, q, qt, qh, off, start, new, longest, pages, stride, window, sinks, scale, o, ot, oh, ws, wsb, HERE)

    for status, bad in ((INVALID, {"ctx": None}), (INVALID, {"c": None}), (INVALID, {"ctx": other}), (INVALID, {"type": ng.NGEMM_F32}), (INVALID, {"type": 9}),
                        (SHAPE, {"batch": -1}), (SHAPE, {"batch": 0}), (SHAPE, {"heads": 3}), (SHAPE, {"heads": 0}), (SHAPE, {"heads": 131072}), (SHAPE, {"tokens": -1}),
                        (SHAPE, {"tokens": 1 << 31}), (INVALID, {"q": None}), (INVALID, {"o": None}), (INVALID, {"q": HERE + 1}), (SHAPE, {"qt": -1}), (SHAPE, {"ot": 64}),
                        (SHAPE, {"oh": 63}), (INVALID, {"off": None}), (SHAPE, {"new": -1}), (SHAPE, {"longest": -1}), (SHAPE, {"longest": (1 << 30) + 1}),
                        (INVALID, {"pages": None}), (SHAPE, {"stride": -2}), (SHAPE, {"window": -1}), (SHAPE, {"window": (1 << 30) + 1}), (SHAPE, {"sinks": -1}),
                        (SHAPE, {"sinks": (1 << 30) + 1}), (INVALID, {"scale": math.nan}), (INVALID, {"scale": math.inf}), (SHAPE, {"batch": 1 << 25})):
        refused(status, *call(**bad))
    for nothing in ({"tokens": 0}, {"new": 0}, {"tokens": 0, "batch": 0, "q": None, "o": None, "off": None}):
        fn, *args = call(**nothing)
        fn(*args)
    for more in ({"longest": 100000}, {"longest": 100000, "new": 4, "tokens": 4}, {"longest": 100000, "tokens": 200, "new": 200}, {"longest": 100000, "window": 60000}):
        need = ng.ngemm_attention_chunk_workspace_bytes(2, 4, 2, 64, more.get("tokens", 8), more.get("new", 8), 100000, more.get("window", 0), 0)
        assert need > 0
        refused(SMALL, *call(**more, wsb=need - 1))
        refused(INVALID, *call(**more, ws=None))
        refused(INVALID, *call(**more, ws=HERE + 8, wsb=need))
    for bad in ((0, 4, 2, 64, 8, 8, 100000, 0, 0), (2, 3, 2, 64, 8, 8, 100000, 0, 0), (2, 4, 2, 72, 8, 8, 100000, 0, 0), (2, 4, 2, 64, 0, 8, 100000, 0, 0),
                (2, 4, 2, 64, 8, 0, 100000, 0, 0), (2, 4, 2, 64, 8, 8, -1, 0, 0), (2, 4, 2, 64, 8, 8, 100000, -1, 0), (2, 4, 2, 64, 8, 8, 16, 0, 0)):
        assert ng.ngemm_attention_chunk_workspace_bytes(*bad) == 0
    ng.ngemm_kv_cache_free(c)


def test_workspace_stays_small(ctx):
    """Splitting the keys serves few rows: its workspace does not grow with the batch or the prompts."""
    most = 0
    for batch in (1, 2, 7, 64, 1000, 100000):
        for new in (1, 2, 16, 100, 3000, 70000):
            for heads, kv, dim in ((32, 8, 128), (12, 12, 64), (64, 1, 256), (16, 1, 16)):
                tokens = batch * new
                if (tokens + 256 * batch) * heads < 1 << 31:
                    for longest in (new, new + 1000, 1 << 20, 1 << 30):
                        most = max(most, ng.ngemm_attention_chunk_workspace_bytes(batch, heads, kv, dim, tokens, new, longest, 0, 0))
    assert 0 < most < 1 << 30
