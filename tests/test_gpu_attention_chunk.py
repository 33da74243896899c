"""Attention of new tokens over the cache's pages, with and without a window, against the plain 64-bit implementation."""
import math

import pytest
import torch

import paper_1910_00178_amd as ng
from attention_ref import Cache, attend, check, quantise
from test_gpu_attention import BF16, F16, Strided, ctx, filled_cache, gen, handle, ints, number, sums  # noqa: F401

pytestmark = pytest.mark.gpu


def run(ctx, cache, table, q, new, starts, window=0, sinks=0, scale=0.125, how="packed", most=None, longest=None, behind=0, o_how=None):  # noqa: F811
    """`behind`: rows of Q behind the last sequence's."""
    H, D = cache.shape[2:]
    raw = cache.raw.cuda()
    c = handle(ctx, cache, raw)
    q = torch.cat([q, torch.full((behind, *q.shape[1:]), math.nan, dtype=q.dtype)]) if behind else q
    n, Hq = q.shape[:2]
    qs, os_ = Strided(q, how), Strided(torch.full_like(q, 77), o_how or how, fill=55.0)
    most = max(new) if most is None else most
    longest = max([a + b for a, b in zip(new, starts)] + [0]) if longest is None else longest
    size = ng.ngemm_attention_chunk_workspace_bytes(len(new), Hq, H, D, n, most, longest, window, sinks)
    ws = torch.full((size + 32,), 0x7f, dtype=torch.uint8, device="cuda")
    out = []
    for _ in range(2):
        ng.ngemm_attention_chunk(ctx, c, number(q.dtype), len(new), Hq, n, *qs.args, ints(sums(new)), ints(starts), most, longest, table.cuda(), table.shape[1],
                                 window, sinks, scale, *os_.args, ws, size)
        torch.cuda.synchronize()
        out.append(os_.window.cpu().clone())
    assert os_.gaps_untouched() and bool((ws[size:] == 0x7f).all())
    assert torch.equal(out[0].nan_to_num(1e4), out[1].nan_to_num(1e4))
    assert not behind or bool((out[0][n - behind:] == 77).all())
    ng.ngemm_kv_cache_free(c)
    return out[0][:n - behind]


def seen(n, start, m, window, sinks):
    at = torch.arange(start, start + n).unsqueeze(1)
    key = torch.arange(m)
    return (key <= at) & ((key > at - window) | (key < sinks)) if window else key <= at


def wanted(cache, table, q, new, starts, window=0, sinks=0, scale=0.125, longest=1 << 30):
    outs, sizes, T, first = [], [], cache.shape[1], 0
    for b, (n, start) in enumerate(zip(new, starts)):
        m = max(0, min(start + n, longest))
        k, v = cache.rows(table[b, :(m + T - 1) // T].tolist(), m) if m else (torch.zeros(0, *cache.shape[2:]).double(),) * 2
        o, s = attend(q[first:first + n].double(), k, v, scale, seen(n, start, m, window, sinks))
        outs.append(o)
        sizes.append(s)
        first += n
    return torch.cat(outs), torch.cat(sizes)


def make(seed, heads, new, starts, dtype, page=48, spread=1.0):
    Hq, H, D = heads
    g = gen(seed)
    cache, table = filled_cache(g, [max(0, a + b) for a, b in zip(new, starts)], page, H, D)
    return cache, table, (torch.randn(sum(new), Hq, D, generator=g) * spread).to(dtype)


def weights(heads, new, dtype):
    """The type that a bound on the weights' rounding may count: bf16 alone for bf16 rows of sequences of many rows."""
    return BF16 if dtype is BF16 and max(new) * heads[0] // heads[1] > 16 else F16


HEADS = [(1, 1, 16), (2, 1, 64), (4, 4, 80), (8, 2, 128), (16, 1, 128), (10, 2, 96), (24, 1, 128), (40, 1, 64), (6, 2, 256), (3, 3, 240), (5, 1, 176)]
LENGTHS = [  # new tokens, starts
    ([1, 1, 1, 1, 1], [0, 15, 16, 63, 300]),
    ([3, 1, 4, 2], [0, 700, 61, 64]),
    ([0, 5, 0, 33, 1, 130, 7], [9, 60, 0, 31, 200, 100, 0]),
    ([257], [0]),
    ([129, 64], [511, 0]),
]
WINDOWS = [(0, 0), (1, 0), (50, 4), (64, 64), (200, 1), (17, 100)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", WINDOWS, ids=lambda w: "x".join(map(str, w)))
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "x".join(map(str, x[0])))
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_chunk(ctx, heads, lengths, window, dtype):  # noqa: F811
    new, starts = lengths
    cache, table, q = make(heads[0] + heads[2], heads, new, starts, dtype)
    scale = 1 / math.sqrt(heads[2])
    got = run(ctx, cache, table, q, new, starts, *window, scale, how="gaps" if heads[0] % 3 == 0 else "packed", behind=len(new) % 2)
    check(got, *wanted(cache, table, q, new, starts, *window, scale), dtype, weights=weights(heads, new, dtype))


@pytest.mark.parametrize("window", [(0, 0), (3000, 70)], ids=["all", "window"])
@pytest.mark.parametrize("lengths", [([1], [20000]), ([4, 2], [9000, 300]), ([100, 1, 1], [70, 12000, 5]), ([96, 96], [16000, 2000]), ([1] * 70, [100 * i for i in range(70)])],
                         ids=["1", "4", "mixed", "96", "70"])
@pytest.mark.parametrize("heads", [(8, 2, 128), (12, 12, 64), (2, 1, 256)], ids=lambda h: "x".join(map(str, h)))
def test_long(ctx, heads, lengths, window):  # noqa: F811
    """Few rows behind long texts: the work is split over their length; more sequences than are looked up together."""
    new, starts = lengths
    cache, table, q = make(7, heads, new, starts, BF16, page=64)
    got = run(ctx, cache, table, q, new, starts, *window, 0.1)
    check(got, *wanted(cache, table, q, new, starts, *window, 0.1), BF16, weights=weights(heads, new, BF16))


@pytest.mark.parametrize("how", ["gaps", "odd", "heads_first"])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_strides(ctx, dtype, how):  # noqa: F811
    for heads, new, starts in (((6, 2, 64), [2, 5], [33, 70]), ((6, 2, 64), [90, 200, 1], [33, 0, 5]), ((4, 1, 176), [40, 3], [10, 100])):
        cache, table, q = make(5, heads, new, starts, dtype, page=16)
        got = run(ctx, cache, table, q, new, starts, how=how)
        check(got, *wanted(cache, table, q, new, starts), dtype, weights=weights(heads, new, dtype))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.5, 1.0, 30.0])
def test_scores(ctx, dtype, scale):  # noqa: F811
    """Weights that are all equal, falling the other way, and so far apart that one key takes everything."""
    for new, starts in (([2, 1], [300, 64]), ([150, 70], [40, 0])):
        cache, table, q = make(9, (8, 2, 128), new, starts, dtype, page=32)
        got = run(ctx, cache, table, q, new, starts, scale=scale)
        want, size = wanted(cache, table, q, new, starts, scale=scale)
        # scores up to some thousands: a float's roundoff of the largest sum of |q k| moves an exponent by that much
        k = max(float(cache.rows(table[b, :(m + 31) // 32].tolist(), m)[0].abs().max()) for b, m in enumerate(a + b for a, b in zip(new, starts)))
        slack = 128 * float(q.abs().max()) * k * abs(scale) * 2.0 ** -21
        check(got, want, size * (1 + slack / 2.0 ** -11), dtype, weights=weights((8, 2), new, dtype))


@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_query_sizes(ctx, size):  # noqa: F811
    for new, starts in (([2, 1], [300, 64]), ([150, 70], [40, 0])):
        cache, table, q = make(10, (4, 2, 64), new, starts, BF16, page=32)
        big = (q.double() * size).to(BF16)
        got = run(ctx, cache, table, big, new, starts, scale=0.1 / size)
        check(got, *wanted(cache, table, big, new, starts, scale=0.1 / size), BF16)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_value_sizes(ctx, dtype):  # noqa: F811
    """Values of very different sizes in one sequence: a token of large values and little weight does not take the others' bits."""
    for new, starts in (([2, 1], [300, 64]), ([150, 70], [40, 0])):
        cache, table, q = make(11, (4, 2, 64), new, starts, dtype, page=32)
        k, v, ks, vs = cache.views()
        at = torch.arange(vs.numel()).view(vs.shape)
        vs.mul_(torch.where(at % 7 == 0, 2.0 ** -12, 1.0))
        got = run(ctx, cache, table, q, new, starts)
        check(got, *wanted(cache, table, q, new, starts), dtype, weights=weights((4, 2), new, dtype))
        vs.mul_(torch.where(at % 41 == 3, 2.0 ** 9, 1.0))
        ks.mul_(torch.where(at % 41 == 3, 0.0, 1.0))
        got = run(ctx, cache, table, q, new, starts)
        check(got, *wanted(cache, table, q, new, starts), dtype, weights=weights((4, 2), new, dtype))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_not_numbers_in_hidden_places(ctx, dtype):  # noqa: F811
    """Rows of NaN that some queries see and others do not: those behind them in a chunk, those before their windows."""
    def odd(n, start, window):                           # a new token in the middle, and one that falls out of the window there
        return [start + n // 2] if window == 0 else [start + n // 2, max(5, start + n // 2 - window - 2)]
    for heads, new, starts in (((4, 1, 64), [6, 2], [50, 100]), ((4, 1, 128), [100, 70], [50, 0]), ((2, 2, 256), [90], [60])):
        for window, sinks in ((0, 0), (30, 3)):
            cache, table, q = make(12, heads, new, starts, dtype, page=32)
            views = cache.views()
            for b, (n, start) in enumerate(zip(new, starts)):
                for t in odd(n, start, window):
                    where = cache.place(int(table[b, t // 32]), t % 32)
                    for codes, scales in ((views[0], views[2]), (views[1], views[3])):
                        codes[where], scales[where] = 0, math.nan
            got = run(ctx, cache, table, q, new, starts, window, sinks)
            want, size = wanted(cache, table, q, new, starts, window, sinks)
            first = 0
            for n, start in zip(new, starts):            # (0 times NaN in the plain products: a row that sees one is NaN, the others are compared without)
                see = seen(n, start, start + n, window, sinks)
                bad = see[:, odd(n, start, window)].any(1)
                assert bool(torch.isnan(got[first:first + n][bad]).all()) and not torch.isnan(got[first:first + n][~bad]).any()
                assert bool(bad.any()) and bool((~bad).any())
                want[first:first + n][bad], got[first:first + n][bad], size[first:first + n][bad] = 0, 0, 0
                first += n
            check(got, want, size, dtype, weights=weights(heads, new, dtype))


def test_missing_pages_and_limits(ctx):  # noqa: F811
    """Pages that are not there are left out; lengths past max_length are not read, rows past max_new are left alone; positions before 0 see nothing."""
    for new, starts in (([2, 3], [300, 64]), ([150, 70], [140, 100])):
        cache, table, q = make(13, (4, 2, 64), new, starts, BF16, page=32)
        holes = table.clone()
        holes[0, 2], holes[0, 0], holes[1, 1] = -1, 1 << 30, cache.shape[0]
        got = run(ctx, cache, holes, q, new, starts)
        first = 0
        for b, (n, start) in enumerate(zip(new, starts)):
            m = start + n
            k, v = cache.rows(table[b, :(m + 31) // 32].tolist(), m)
            there = torch.tensor([0 <= int(holes[b, t // 32]) < cache.shape[0] for t in range(m)])
            want, size = attend(q[first:first + n].double(), k, v, 0.125, seen(n, start, m, 0, 0) & there)
            check(got[first:first + n], want, size, BF16)
            first += n
        # a table that ends early
        got = run(ctx, cache, table[:, :3].contiguous(), q, new, starts)
        check(got, *wanted(cache, table, q, new, starts, longest=96), BF16)
        got = run(ctx, cache, table, q, new, starts, longest=100)
        check(got, *wanted(cache, table, q, new, starts, longest=100), BF16)
        got = run(ctx, cache, table, q, new, starts, most=1)
        want, size = wanted(cache, table, q, new, starts)
        first = 0
        for n in new:
            check(got[first:first + 1], want[first:first + 1], size[first:first + 1], BF16)
            assert bool((got[first + 1:first + n] == 77).all())
            first += n
        before = [-1, -new[1]]
        got = run(ctx, cache, table, q, new, before, window=40, sinks=2, longest=400)
        want, size = wanted(cache, table, q, new, before, 40, 2)
        check(got, want, size, BF16)
        assert not got[0].any() and not got[new[0]:].any()
        # larger bounds than need be
        got = run(ctx, cache, table, q, new, starts, most=5000, longest=1 << 30)
        check(got, *wanted(cache, table, q, new, starts), BF16)
        # nothing in the cache may be read
        assert not run(ctx, cache, table, q, new, starts, longest=0).any()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [(0, 0), (40, 5)], ids=["all", "window"])
def test_many_sequences(ctx, window, dtype):  # noqa: F811
    """More sequences than share keys out: single tokens, some tokens, pieces of prompts, none."""
    g = gen(17)
    new = [int(n) for n in torch.randint(0, 90, (150,), generator=g)]
    new[::3] = [1] * len(new[::3])
    starts = [int(n) for n in torch.randint(0, 700, (150,), generator=g)]
    for heads in ((2, 1, 64), (6, 2, 32)):
        for most in (new, [min(n, 7) for n in new]):
            cache, table, q = make(18, heads, most, starts, dtype, page=32)
            got = run(ctx, cache, table, q, most, starts, *window)
            check(got, *wanted(cache, table, q, most, starts, *window), dtype, weights=weights(heads, most, dtype))


@pytest.mark.parametrize("heads", [(4, 1, 128), (3, 3, 64), (2, 1, 208)], ids=lambda h: "x".join(map(str, h)))
def test_rows_between_the_forms(ctx, heads):  # noqa: F811
    """As many rows as the kernel of few takes, and one more; a tile's rows and one more."""
    group = heads[0] // heads[1]
    for rows in (16, 32, 64, 128, 256):
        for more in (0, 1):
            n = rows // group + more
            new, starts = [n, 1, n], [300, 900, 0]
            cache, table, q = make(19, heads, new, starts, F16)
            got = run(ctx, cache, table, q, new, starts)
            check(got, *wanted(cache, table, q, new, starts), F16)


def test_replay_with_other_lengths(ctx):  # noqa: F811
    """Captured once, replayed with other lengths, pages and queries: what eager calls with the same bounds give."""
    Hq, H, D, page, batch, most, longest = 8, 2, 64, 32, 4, 40, 3000
    per = longest // page + 1
    cases = [([1, 40, 3, 0], [2000, 100, 0, 50]), ([40, 40, 40, 40], [2960, 0, 1000, 30]), ([2, 1, 0, 1], [5, 2990, 7, 400])]
    g = gen(20)
    caches = [make(21 + i, (Hq, H, D), new, starts, BF16, page=page) for i, (new, starts) in enumerate(cases)]
    pool = max(c.raw.shape[0] for c, _, _ in caches)
    raw = torch.zeros(pool, H, page // 16, 32 * D + 128, dtype=torch.int8, device="cuda")
    c = ng.ngemm_kv_cache_create(ctx, pool, page, H, D, raw, raw.numel())
    n = most * batch
    q, o = (torch.zeros(n, Hq, D, dtype=BF16, device="cuda") for _ in range(2))
    off, start, pages = torch.zeros(batch + 1, dtype=torch.int32, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.full((batch, per), -1).int().cuda()
    size = ng.ngemm_attention_chunk_workspace_bytes(batch, Hq, H, D, n, most, longest, 900, 8)
    ws = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")

    def call():
        ng.ngemm_attention_chunk(ctx, c, ng.NGEMM_BF16, batch, Hq, n, q, Hq * D, D, off, start, most, longest, pages, per, 900, 8, 0.125, o, Hq * D, D, ws, size)

    def fill(i):
        (new, starts), (cache, table, rows) = cases[i], caches[i]
        raw.zero_()
        raw[:cache.raw.shape[0]].copy_(cache.raw)
        q.zero_()
        q[:sum(new)].copy_(rows)
        off.copy_(ints(sums(new)))
        start.copy_(ints(starts))
        pages.fill_(-1)
        pages[:, :table.shape[1]].copy_(table[:, :per])
        o.zero_()
        torch.cuda.synchronize()

    fill(0)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in (0, 1, 2, 0, 2, 1):
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        fill(i)
        call()
        torch.cuda.synchronize()
        assert torch.equal(o, got)
        torch.randn(1000, device="cuda").sum().item()
        new, starts = cases[i]
        cache, table, rows = caches[i]
        check(got.cpu()[:sum(new)], *wanted(cache, table, rows, new, starts, 900, 8), BF16)
        assert not got[sum(new):].any()
    ng.ngemm_kv_cache_free(c)


def test_as_decode(ctx):  # noqa: F811
    """A token of each sequence: what ngemm_attention_decode gives, up to the roundings of both."""
    lengths, heads = [1, 40, 333, 64], (8, 2, 128)
    cache, table, q = make(14, heads, [1] * 4, [n - 1 for n in lengths], F16)
    got = run(ctx, cache, table, q, [1] * 4, [n - 1 for n in lengths])
    from test_gpu_attention import decode
    other = decode(ctx, cache, table, q, lengths, 0.125)
    assert float((got.double() - other.double()).abs().max()) <= 2.0 ** -9 * float(other.double().abs().max())


def test_together(ctx):  # noqa: F811
    """Prompts in pieces, proposed tokens, single ones: rows normalised, rotated and written, then attended to; on a stream, captured and replayed."""
    from turn_ref import table as angles, turned
    Hq, H, D, page, batch, per = 8, 2, 64, 16, 3, 20
    g = gen(15)
    host = angles(per * page, D)
    dev = host.cuda()
    rotation = ng.ngemm_rotation_create(ctx, per * page, D, ng.NGEMM_PAIRS_HALVES, dev, dev.numel() * 4)
    wq, wk = (1 + torch.randn(D, generator=g) / 4 for _ in range(2))
    wqd, wkd = wq.cuda(), wk.cuda()
    cache = Cache(batch * per, page, H, D)
    raw = cache.raw.cuda()
    c = handle(ctx, cache, raw)
    table = torch.randperm(batch * per, generator=g).view(batch, per).int()
    pages = table.cuda()
    starts = [0] * batch
    ks = [torch.zeros(0, H, D) for _ in range(batch)]
    vs = [torch.zeros(0, H, D) for _ in range(batch)]
    for new in ([100, 30, 1], [50, 0, 70], [4, 1, 5], [1, 1, 1], [1, 1, 1]):
        n = sum(new)
        x = torch.randn(n, Hq + 2 * H, D, generator=g).to(BF16)
        xd = x.cuda()
        row = (Hq + 2 * H) * D
        q, k, v = xd[:, :Hq], xd[:, Hq:Hq + H], xd[:, Hq + H:]                  # views, as a projection gives them
        at = torch.cat([torch.arange(a, a + b) for a, b in zip(starts, new)])
        off, start, where = ints(sums(new)), ints(starts), at.int().cuda()
        qr, o = torch.empty(n, Hq, D, dtype=BF16, device="cuda"), torch.empty(n, Hq, D, dtype=BF16, device="cuda")
        longest, window, sinks = max(a + b for a, b in zip(starts, new)), 64, 4
        size = ng.ngemm_attention_chunk_workspace_bytes(batch, Hq, H, D, n, max(new), longest, window, sinks)
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")

        def step():
            ng.ngemm_qk_norm_rotate(ctx, ng.NGEMM_BF16, D, n, Hq, q, row, D, wqd, 0, None, 0, 0, None, 1e-6, rotation, where, qr, Hq * D, D, None, 0, 0)
            ng.ngemm_kv_write_rotated(ctx, c, ng.NGEMM_BF16, batch, n, k, row, D, v, row, D, wkd, 1e-6, rotation, off, start, pages, per)
            ng.ngemm_attention_chunk(ctx, c, ng.NGEMM_BF16, batch, Hq, n, qr, Hq * D, D, off, start, max(new), longest, pages, per, window, sinks, 0.125,
                                     o, Hq * D, D, ws, size)

        step()
        torch.cuda.synchronize()
        eager, bytes_ = o.clone(), raw.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(3):
            o.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, eager) and torch.equal(raw, bytes_)
            torch.randn(1000, device="cuda").sum().item()
        first = 0
        cache.raw = raw.cpu()
        qw, _ = turned(x[:, :Hq], wq, 1e-6, host, at, False)
        for b, m in enumerate(new):
            rows = slice(first, first + m)
            ks[b] = torch.cat([ks[b], x[rows, Hq:Hq + H].float()])
            vs[b] = torch.cat([vs[b], x[rows, Hq + H:].float()])
            first += m
            if m == 0:
                continue
            have = starts[b] + m
            # the cache holds the rotated keys, to a step of their codes
            got = cache.rows(table[b, :(have + page - 1) // page].tolist(), have)
            kw, _ = turned(ks[b].to(BF16), wk, 1e-6, host, torch.arange(have), False)
            for a, w in zip(got, (kw, vs[b].double())):
                assert bool(((a - w).abs() <= (0.5 + 2.0 ** -10) * w.abs().amax(-1, keepdim=True) / 127).all())
            # a query is off by half a step of bf16: the scores by 2^-8 |q| |k| scale at most, the weights by twice that
            moved = 2 * 2.0 ** -8 * float(qw[rows].norm(dim=-1).max() * got[0].norm(dim=-1).max()) * 0.125
            want, size_ = attend(qw[rows], *got, 0.125, seen(m, starts[b], have, window, sinks))
            check(eager.cpu()[rows], want, size_ * (1 + moved / 2.0 ** -8), BF16)
        starts = [a + b for a, b in zip(starts, new)]
    ng.ngemm_kv_cache_free(c)
    ng.ngemm_rotation_free(rotation)


def test_cache_past_32_bits(ctx):  # noqa: F811
    """Blocks behind the first 4 GiB of the cache."""
    page, H, D = 16, 2, 128
    pool = (5 << 30) // (2 * (32 * D + 128))
    raw = torch.zeros(ng.ngemm_kv_cache_bytes(pool, page, H, D), dtype=torch.int8, device="cuda")
    c = ng.ngemm_kv_cache_create(ctx, pool, page, H, D, raw, raw.numel())
    g = gen(16)
    for new, start in (([3], 60), ([70], 30)):
        n, m = new[0], new[0] + start
        table = torch.tensor([pool - 1 - 3 * i for i in range((m + 15) // 16)]).int().unsqueeze(0)
        k, v = (torch.randn(m, H, D, generator=g).to(F16) for _ in range(2))
        ng.ngemm_kv_write_rotated(ctx, c, ng.NGEMM_F16, 1, m, k.cuda(), H * D, D, v.cuda(), H * D, D, None, 0.0, None, ints([0, m]), None, table.cuda(), table.shape[1])
        q = torch.randn(n, 4, D, generator=g).to(F16)
        o = torch.zeros(n, 4, D, dtype=F16, device="cuda")
        size = ng.ngemm_attention_chunk_workspace_bytes(1, 4, H, D, n, n, m, 0, 0)
        ws = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
        ng.ngemm_attention_chunk(ctx, c, ng.NGEMM_F16, 1, 4, n, q.cuda(), 4 * D, D, ints([0, n]), ints([start]), n, m, table.cuda(), table.shape[1], 0, 0, 0.1,
                                 o, 4 * D, D, ws, size)
        torch.cuda.synchronize()
        (kc, ks), (vc, vs) = quantise(k), quantise(v)
        want, sz = attend(q.double(), kc.double() * ks.double().unsqueeze(-1), vc.double() * vs.double().unsqueeze(-1), 0.1, seen(n, start, m, 0, 0))
        # (K's codes may be the next ones near a tie, one in thousands: a step of a code in a score)
        check(o, want, sz * 1.2, F16)
    ng.ngemm_kv_cache_free(c)


@pytest.mark.parametrize("window", [(0, 0), (90, 3)], ids=["all", "window"])
@pytest.mark.parametrize("batch, most, past", [(128, 40, 300), (100, 9, 200), (16, 130, 1100), (70, 2, 900), (3, 400, 1500)])
def test_batches(ctx, batch, most, past, window):  # noqa: F811
    """Every form by itself over batches that fill the device: tiles are numbered over up to 128 sequences, some of which have no tokens."""
    g = gen(batch)
    heads = (16, 8, 32)
    for ragged in (False, True):
        new = [int(n) for n in torch.randint(0, most + 1, (batch,), generator=g)] if ragged else [most] * batch
        starts = [int(n) for n in torch.randint(0, past + 1, (batch,), generator=g)] if ragged else [past] * batch
        if sum(new) == 0:
            continue
        cache, table, q = make(batch + 1, heads, new, starts, BF16, page=64)
        got = run(ctx, cache, table, q, new, starts, *window)
        check(got, *wanted(cache, table, q, new, starts, *window), BF16, weights=weights(heads, new, BF16))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_in_the_queries_place(ctx, dtype):  # noqa: F811
    """O at Q's address: the same bits as elsewhere, with keys shared out and not, for few rows and for many."""
    for heads, new, starts in (((8, 2, 128), [1, 3], [30, 20]), ((8, 2, 128), [2], [9000]), ((8, 2, 128), [16, 9], [700, 40]), ((8, 2, 128), [90, 40, 0, 70], [0, 30, 5, 100]),
                               ((4, 4, 64), [300], [6000]), ((2, 1, 240), [700, 3], [0, 800])):
        cache, table, q = make(23, heads, new, starts, dtype, page=64)
        elsewhere = run(ctx, cache, table, q, new, starts)
        raw = cache.raw.cuda()
        c = handle(ctx, cache, raw)
        rows, (Hq, H, D), longest = q.cuda(), heads, max(a + b for a, b in zip(new, starts))
        size = ng.ngemm_attention_chunk_workspace_bytes(len(new), Hq, H, D, sum(new), max(new), longest, 0, 0)
        ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
        ng.ngemm_attention_chunk(ctx, c, number(dtype), len(new), Hq, sum(new), rows, Hq * D, D, ints(sums(new)), ints(starts), max(new), longest, table.cuda(),
                                 table.shape[1], 0, 0, 0.125, rows, Hq * D, D, ws, size)
        torch.cuda.synchronize()
        assert torch.equal(rows.cpu(), elsewhere)
        ng.ngemm_kv_cache_free(c)


def test_two_streams(ctx):  # noqa: F811
    """Calls on two streams at once, each with a workspace of its own, give what they give one after the other."""
    heads, parts = (8, 2, 128), []
    for new, starts in (([5, 40, 300], [4000, 100, 900]), ([2] * 9, [1500] * 9)):
        cache, table, q = make(29, heads, new, starts, BF16, page=64)
        want = run(ctx, cache, table, q, new, starts)
        raw, longest = cache.raw.cuda(), max(a + b for a, b in zip(new, starts))
        size = ng.ngemm_attention_chunk_workspace_bytes(len(new), 8, 2, 128, sum(new), max(new), longest, 0, 0)
        q = q.cuda()
        parts.append((new, want, raw, handle(ctx, cache, raw), longest, size, q, torch.empty_like(q), table.cuda(), ints(sums(new)), ints(starts),
                      torch.empty(size + 16, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for new, _want, _raw, c, longest, size, q, o, table, offsets, starts, ws, stream in parts:
            ng.ngemm_attention_chunk(ctx, c, ng.NGEMM_BF16, len(new), 8, sum(new), q, 1024, 128, offsets, starts, max(new), longest, table, table.shape[1], 0, 0, 0.125,
                                     o, 1024, 128, ws, size, stream.cuda_stream)
    torch.cuda.synchronize()
    for _new, want, _raw, c, _l, _s, _q, o, *_ in parts:
        assert torch.equal(o.cpu(), want)
        ng.ngemm_kv_cache_free(c)
