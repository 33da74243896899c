"""Norms and rotations of rows, and of keys on their way into the cache, against the plain 64-bit implementation."""
import math

import pytest
import torch

import paper_1910_00178_amd as ng
from attention_ref import Cache, quantise
from test_gpu_attention import BF16, F16, F32, Strided, ctx, gen, handle, ints, number, page_table, sums  # noqa: F401
from turn_ref import ARITHMETIC, check_rows, table, turned

pytestmark = pytest.mark.gpu

HALVES, NEIGHBOURS = ng.NGEMM_PAIRS_HALVES, ng.NGEMM_PAIRS_NEIGHBOURS


class Rotation:
    def __init__(self, ctx, positions, dim, pairs):
        self.host = table(positions, dim)
        self.dev = self.host.cuda()
        self.handle = ng.ngemm_rotation_create(ctx, positions, dim, pairs, self.dev, self.dev.numel() * 4)
        self.pairs = pairs

    def close(self):
        ng.ngemm_rotation_free(self.handle)


def turn(ctx, q, k, wq, wk, eps, rotation, positions, how="packed", in_place=False, stream=None):
    n, Hq, D = q.shape
    qs, ks = Strided(q, how, fill=9.0), Strided(k, how, fill=9.0)
    qo, ko = (qs, ks) if in_place else (Strided(torch.full_like(q, 5), how, fill=9.0), Strided(torch.full_like(k, 5), how, fill=9.0))
    dev = [None if w is None else w.float().cuda() for w in (wq, wk)]
    ng.ngemm_qk_norm_rotate(ctx, number(q.dtype), D, n, Hq, *qs.args, dev[0], k.shape[1], *ks.args, dev[1], eps, rotation and rotation.handle,
                            None if positions is None else positions.int().cuda(), *qo.args, *ko.args, stream)
    torch.cuda.synchronize()
    assert qo.gaps_untouched() and ko.gaps_untouched()
    return qo.window.clone(), ko.window.clone()


def check_turn(ctx, q, k, wq, wk, eps, rotation, positions, **how):
    got = turn(ctx, q, k, wq, wk, eps, rotation, positions, **how)
    for out, x, w in zip(got, (q, k), (wq, wk)):
        check_rows(out, *turned(x, w, eps, rotation and rotation.host, positions, rotation and rotation.pairs == NEIGHBOURS))
    return got


SIZES = [  # heads of Q and K, D, rotated, tokens
    (1, 1, 16, 16, 1),
    (3, 1, 32, 32, 5),
    (12, 12, 64, 64, 33),
    (32, 8, 128, 128, 7),
    (5, 2, 80, 48, 65),
    (40, 8, 96, 96, 9),
    (2, 2, 96, 16, 3),
    (6, 1, 256, 64, 17),
    (1, 3, 240, 240, 20),
    (32, 8, 128, 112, 700),                              # enough rows for four heads an item, heads that are no multiple of four:
    (9, 2, 64, 32, 12000),
    (5, 3, 208, 208, 6000),
]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("pairs", [None, HALVES, NEIGHBOURS])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_rows(ctx, size, pairs, dtype):  # noqa: F811
    Hq, Hk, D, rotated, n = size
    g = gen(D + n)
    q, k = (torch.randn(n, h, D, generator=g).mul(2).to(dtype) for h in (Hq, Hk))
    wq, wk = (1 + torch.randn(D, generator=g) / 4 for _ in range(2))
    positions = torch.randint(0, 5000, (n,), generator=g)
    rotation = None if pairs is None else Rotation(ctx, 5000, rotated, pairs)
    check_turn(ctx, q, k, wq, wk, 1e-6, rotation, positions)
    if pairs is not None:
        check_turn(ctx, q, k, None, wk, 1e-6, rotation, positions)
        rotation.close()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("how", ["gaps", "odd", "heads_first"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_strides_and_places(ctx, dtype, how, in_place):  # noqa: F811
    for D, n, pairs in ((64, 40, HALVES), (128, 2100, NEIGHBOURS), (256, 3, HALVES), (128, 2100, HALVES)):
        g = gen(D)
        q, k = (torch.randn(n, h, D, generator=g).to(dtype) for h in (6, 2))
        rotation = Rotation(ctx, 100, D // 2, pairs)
        check_turn(ctx, q, k, torch.rand(D, generator=g), None, 1e-5, rotation, torch.arange(n) % 100, how=how, in_place=in_place)
        rotation.close()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("eps", [0.0, 1e-12, 1e-6, 1.0])
def test_rows_of_any_size(ctx, dtype, eps):  # noqa: F811
    """Squares far outside of the floats' range on either side, rows of zeros, single large elements."""
    g = gen(3)
    sizes = [1.0, 0.0, 6e-8, 1e-5, 6e4] if dtype is F16 else [1.0, 0.0, 1e-38, 1e-30, 1e-22, 1e-18, 1e-15, 1e15, 1e18, 1e20, 1e30, 1e37]
    q = torch.stack([torch.randn(2, 128, generator=g).clamp(-1, 1).double() * s for s in sizes]).to(dtype)
    q[0, 1, 1:] = 0
    k = q[:, :1].clone()
    got = check_turn(ctx, q, k, torch.ones(128), torch.rand(128, generator=g), eps, None, None)
    assert not got[0][1].any() and bool(torch.isfinite(got[0].float()).all())


def test_rows_that_are_not_numbers(ctx):  # noqa: F811
    q = torch.ones(4, 2, 64)
    q[1, 0, 5], q[2, 1, 7] = math.inf, math.nan
    got, _ = turn(ctx, q, q[:, :1], torch.ones(64), None, 1e-6, None, None)
    want = torch.ones(4, 2, 64)
    want[1, 0], want[1, 0, 5], want[2, 1] = 0, math.nan, math.nan
    assert torch.allclose(got.cpu(), want, equal_nan=True)


@pytest.mark.parametrize("pairs", [HALVES, NEIGHBOURS])
def test_positions_without_angles(ctx, pairs):  # noqa: F811
    g = gen(6)
    rotation = Rotation(ctx, 50, 32, pairs)
    positions = torch.tensor([0, 49, 50, -1, 1 << 30, -(1 << 31), 7])
    q = torch.randn(7, 3, 64, generator=g)
    got = check_turn(ctx, q, q[:, :2].clone(), None, torch.rand(64, generator=g), 1e-6, rotation, positions)
    assert bool(torch.isnan(got[0][2:6]).all()) and not torch.isnan(got[0][[0, 1, 6]]).any()
    rotation.close()


def test_one_side_and_shared_rows(ctx):  # noqa: F811
    """Q or K alone; an input whose heads are one row; nothing to do."""
    g = gen(8)
    D, n = 64, 9
    rotation = Rotation(ctx, 100, D, HALVES)
    positions = torch.arange(n)
    row = torch.randn(n, D, generator=g).to(BF16)
    dev, out, at = row.cuda(), torch.full((n, 4, D), 3.0, dtype=BF16, device="cuda"), ints(list(range(n)))
    args = (dev, D, 0, None)
    ng.ngemm_qk_norm_rotate(ctx, ng.NGEMM_BF16, D, n, 4, *args, 0, None, 0, 0, None, 0.0, rotation.handle, at, out, 4 * D, D, None, 0, 0)
    torch.cuda.synchronize()
    check_rows(out, *turned(row[:, None].expand(n, 4, D), None, 0.0, rotation.host, positions, False))
    k_out = torch.full_like(out, 3.0)
    ng.ngemm_qk_norm_rotate(ctx, ng.NGEMM_BF16, D, n, 0, None, 0, 0, None, 4, *args, 0.0, rotation.handle, at, None, 0, 0, k_out, 4 * D, D)
    torch.cuda.synchronize()
    assert torch.equal(out, k_out)
    for tokens, heads in ((0, 4), (n, 0)):
        ng.ngemm_qk_norm_rotate(ctx, ng.NGEMM_BF16, D, tokens, heads, *args, 0, None, 0, 0, None, 0.0, rotation.handle, at, k_out, 4 * D, D, None, 0, 0)
    torch.cuda.synchronize()
    assert torch.equal(out, k_out)
    rotation.close()


# ---- into the cache ----

WRITES = [  # page, heads, D, rotated, new tokens, starts
    (16, 1, 16, 16, [1], [0]),
    (16, 2, 64, 64, [1, 1, 1, 1], [0, 15, 16, 33]),
    (64, 3, 128, 128, [17, 0, 40, 1, 100], [5, 3, 0, 63, 31]),
    (48, 2, 80, 32, [16, 32, 15], [16, 0, 1]),
    (32, 1, 256, 256, [50, 3], [0, 14]),
    (16, 5, 96, 96, [33], [7]),
    (16, 2, 240, 16, [20, 1], [3, 9]),
    (64, 8, 128, 128, [3000, 1500, 5000], [100, 0, 3]),  # two heads a workgroup
]


def check_write(ctx, shape, dtype, pairs, norm, how, k=None, positions=200):  # noqa: F811
    page, H, D, rotated, new, starts = shape
    g = gen(D + len(new))
    per = max((a + n + page - 1) // page for a, n in zip(starts, new))
    pool = len(new) * per + 2
    pages = page_table(g, len(new), per, pool, spare=1)
    want = Cache(pool, page, H, D, fill=0x33)
    raw = want.raw.cuda()
    off = sums(new)
    at = torch.cat([torch.arange(a, a + n) for a, n in zip(starts, new)])
    if k is None:
        k = (torch.randn(off[-1], H, D, generator=g) * torch.rand(off[-1], H, 1, generator=g) * 7).to(dtype)
    v = (torch.randn(off[-1], H, D, generator=g) * 3).to(dtype)
    weight = 1 + torch.randn(D, generator=g) / 4 if norm else None
    rotation = None if pairs is None else Rotation(ctx, max(positions, int(at.max()) + 1) if positions else 30, rotated, pairs)
    y, size = turned(k, weight, 1e-6, rotation and rotation.host, at, pairs == NEIGHBOURS)
    seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new))
    place = (pages[seq, at // page].long(), slice(None), at % page // 16, at % 16)
    views = want.views()
    views[0][place], views[2][place] = quantise(y)
    views[1][place], views[3][place] = quantise(v)
    c = handle(ctx, want, raw)
    ks, vs = Strided(k, how), Strided(v, how)
    ng.ngemm_kv_write_rotated(ctx, c, number(dtype), len(new), off[-1], *ks.args, *vs.args, None if weight is None else weight.cuda(), 1e-6,
                              rotation and rotation.handle, ints(off), ints(starts), pages.cuda(), pages.shape[1])
    torch.cuda.synchronize()
    ng.ngemm_kv_cache_free(c)
    if rotation:
        rotation.close()
    got = Cache(pool, page, H, D)
    got.raw = raw.cpu()
    codes, scales = got.views()[0][place].double(), got.views()[2][place].double()
    # K: an element is off by ARITHMETIC times its size, the largest too; 127 y / amax by both, and by the roundings of the product, the quotient and amax / 127
    most = y.abs().amax(-1, keepdim=True)
    assert torch.equal(torch.isnan(scales), torch.isnan(most[..., 0]))
    fine = ~torch.isnan(scales)
    most_off = ARITHMETIC * size.amax(-1, keepdim=True)
    assert bool(((scales - most[..., 0] / 127).abs() <= most_off[..., 0] / 127 + 2.0 ** -22 * most[..., 0] / 127 + 2.0 ** -149)[fine].all())
    exact = torch.where(most > 0, 127 * y / torch.where(most > 0, most, 1), 0.0)
    by = torch.where(most > 0, 127 * (ARITHMETIC * size + most_off) / torch.where(most > 0, most, 1), 0.0) + 2.0 ** -15
    assert bool(((codes - exact).abs() <= 0.5 + by)[fine].all()) and not codes[~fine].any()
    # V, and every byte that was not to be written
    a, b = got.views(), want.views()
    a[0][place], a[2][place] = b[0][place], b[2][place]
    assert torch.equal(got.raw, want.raw)
    return codes, scales


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("pairs", [None, HALVES, NEIGHBOURS])
@pytest.mark.parametrize("shape", WRITES, ids=lambda s: "x".join(map(str, s[:4])))
def test_write(ctx, shape, pairs, dtype):  # noqa: F811
    if dtype is F32:                                     # (V's codes of f32 rows may differ near ties: those of bf16 numbers are exact)
        g = gen(1)
        k = torch.randn(sum(shape[4]), shape[1], shape[2], generator=g)
        check_write_f32(ctx, shape, pairs, k)
        return
    check_write(ctx, shape, dtype, pairs, True, "packed")
    check_write(ctx, shape, dtype, pairs, False, "packed")


def check_write_f32(ctx, shape, pairs, k):  # noqa: F811
    """K in f32 against the same rows in the plain implementation; V's rows hold few bits, so that their codes are certain."""
    page, H, D, rotated, new, starts = shape
    torch_randn = torch.randn

    def few_bits(*a, **kw):
        return torch_randn(*a, **kw).to(BF16).float()
    torch.randn = few_bits
    try:
        check_write(ctx, shape, F32, pairs, True, "packed", k=k)
    finally:
        torch.randn = torch_randn


@pytest.mark.parametrize("how", ["gaps", "odd", "heads_first"])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_write_strides(ctx, dtype, how):  # noqa: F811
    check_write(ctx, WRITES[2], dtype, HALVES, True, how)
    check_write(ctx, WRITES[3], dtype, NEIGHBOURS, False, how)


def test_write_as_kv_write(ctx):  # noqa: F811
    """Without norm and rotation: the bytes of ngemm_kv_write."""
    page, H, D, n = 32, 4, 128, 1000
    g = gen(2)
    k, v = (torch.randn(n, H, D, generator=g).to(BF16).cuda() for _ in range(2))
    pages = page_table(g, 2, 17, 40).cuda()
    size = ng.ngemm_kv_cache_bytes(40, page, H, D)
    raws = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    for raw, fn, more in zip(raws, (ng.ngemm_kv_write, ng.ngemm_kv_write_rotated), ((), (None, 0.0, None))):
        c = ng.ngemm_kv_cache_create(ctx, 40, page, H, D, raw, size)
        fn(ctx, c, ng.NGEMM_BF16, 2, n, k, H * D, D, v, H * D, D, *more, ints([0, 477, n]), ints([5, 0]), pages, 17)
        torch.cuda.synchronize()
        ng.ngemm_kv_cache_free(c)
    # 127 x / amax from 16-bit rows and from the same numbers as floats: the next code near a tie
    a, b = (r[:size].view(torch.int8).view(40, H, page // 16, 32 * D + 128).cpu() for r in raws)
    assert torch.equal(a[..., 16 * D:], b[..., 16 * D:]) and int((a.int() - b.int())[..., :16 * D].abs().max()) <= 1
    assert int((a != b).sum()) < 100


def test_write_positions_without_angles(ctx):  # noqa: F811
    """Positions that the table does not have: K's rows are NaN, V's are written."""
    codes, scales = check_write(ctx, (16, 2, 64, 64, [20, 40], [5, 0]), BF16, HALVES, True, "packed", positions=0)
    assert bool(torch.isnan(scales[50:]).all()) and not torch.isnan(scales[20:50]).any()


def test_write_places_that_do_not_exist(ctx):  # noqa: F811
    """Positions before 0, past the pages and in pages that are not there: nothing is written, and nothing faults."""
    page, H, D = 16, 2, 64
    cache = Cache(3, page, H, D, fill=0x11)
    raw = cache.raw.cuda()
    c = handle(ctx, cache, raw)
    rotation = Rotation(ctx, 100, D, HALVES)
    g = gen(1)
    k, v = (torch.randn(60, H, D, generator=g).to(F16).cuda() for _ in range(2))
    pages = ints([[5, 1], [-1, 2], [0, 1 << 30]])
    ng.ngemm_kv_write_rotated(ctx, c, ng.NGEMM_F16, 3, 60, k, H * D, D, v, H * D, D, None, 0.0, rotation.handle, ints([0, 20, 40, 60]), ints([10, -40, 25]), pages, 2)
    torch.cuda.synchronize()
    now = raw.cpu()
    touched = (now != 0x11).flatten(1).any(1)
    assert touched.tolist() == [False, True, False]                            # sequence 0's second page
    assert bool((now[1, :, 0, :14 * D] != 0x11).any())
    ng.ngemm_kv_cache_free(c)
    rotation.close()


def test_stream_and_graph(ctx):  # noqa: F811
    """On a stream of their own, captured, and replayed with other inputs: the eager results every time."""
    n, Hq, H, D, page = 50, 8, 2, 64, 16
    rotation = Rotation(ctx, 100, D, HALVES)
    raw = torch.zeros(ng.ngemm_kv_cache_bytes(8, page, H, D), dtype=torch.int8, device="cuda")
    c = ng.ngemm_kv_cache_create(ctx, 8, page, H, D, raw, raw.numel())
    q, k, v = (torch.empty(n, h, D, dtype=BF16, device="cuda") for h in (Hq, H, H))
    qo, ko, w = torch.empty_like(q), torch.empty_like(k), torch.rand(D, device="cuda")
    at, off, pages = ints(list(range(n))), ints([0, n]), ints([[3, 1, 5, 7]])

    def calls():
        ng.ngemm_qk_norm_rotate(ctx, ng.NGEMM_BF16, D, n, Hq, q, Hq * D, D, w, H, k, H * D, D, w, 1e-6, rotation.handle, at, qo, Hq * D, D, ko, H * D, D)
        ng.ngemm_kv_write_rotated(ctx, c, ng.NGEMM_BF16, 1, n, k, H * D, D, v, H * D, D, w, 1e-6, rotation.handle, off, None, pages, 4)

    def fill(seed):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen(seed)).to(BF16))
        torch.cuda.synchronize()

    outs, eager = (qo, ko, raw), []
    for seed in range(3):
        fill(seed)
        calls()
        torch.cuda.synchronize()
        eager.append([x.clone() for x in outs])
    side = torch.cuda.Stream()
    fill(0)
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, eager[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (1, 2, 0, 1):
        fill(seed)
        for x in outs:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager[seed]))
        torch.randn(1000, device="cuda").sum().item()
    ng.ngemm_kv_cache_free(c)
    rotation.close()
