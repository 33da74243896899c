"""The 8-bit key-value cache and the attention calls against the plain 64-bit implementation."""
import math

import pytest
import torch

import paper_1910_00178_amd as ng
from attention_ref import Cache, attend, check, quantise

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def number(dtype):
    return {F32: ng.NGEMM_F32, F16: ng.NGEMM_F16, BF16: ng.NGEMM_BF16}[dtype]


@pytest.fixture(scope="module")
def ctx():
    c = ng.ngemm_create(0)
    yield c
    ng.ngemm_destroy(c)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda").contiguous()


def sums(lengths):
    return [sum(lengths[:b]) for b in range(len(lengths) + 1)]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def page_table(g, batch, per, pool, spare=0):
    """Distinct pages of the pool for every sequence, `spare` entries of garbage behind them."""
    t = torch.randperm(pool, generator=g)[:batch * per].view(batch, per).int()
    if spare:
        t = torch.cat([t, torch.tensor([-1, 1 << 30, -(1 << 31), pool])[torch.arange(spare) % 4].int().expand(batch, spare)], 1)
    return t.contiguous()


class Strided:
    """Rows [n][heads][D] on the device: packed, with gaps, heads first, or from an odd address."""

    def __init__(self, x, how, fill=0.0):
        n, H, D = x.shape
        gap = {"packed": 0, "gaps": 8, "odd": 3, "heads_first": 16}[how]
        if how == "heads_first":
            self.token, self.head = D + gap, (D + gap) * n
        else:
            self.token, self.head = (D + gap) * H, D + gap
        self.at = 1 if how == "odd" else 0
        size = self.at + max(0, n - 1) * self.token + max(0, H - 1) * self.head + D if n else 1
        self.buffer = torch.full((size,), fill, dtype=x.dtype, device="cuda")
        self.window = torch.as_strided(self.buffer, (n, H, D), (self.token, self.head, 1), self.at)
        self.window.copy_(x)
        self.fill, self.shape = fill, (n, H, D)

    @property
    def args(self):
        return self.buffer.data_ptr() + self.at * self.buffer.element_size(), self.token, self.head

    def gaps_untouched(self):
        rest = self.buffer.clone()
        torch.as_strided(rest, self.shape, (self.token, self.head, 1), self.at).fill_(self.fill)
        return bool((rest == self.fill).all())


def handle(ctx, cache, raw):
    P, T, H, D = cache.shape
    assert ng.ngemm_kv_cache_bytes(P, T, H, D) == raw.numel()
    return ng.ngemm_kv_cache_create(ctx, P, T, H, D, raw, raw.numel())


# ---- the cache ----

SHAPES = [  # page, heads, D, new tokens, starts
    (16, 1, 16, [1], [0]),
    (16, 2, 64, [1, 1, 1, 1], [0, 15, 16, 33]),
    (64, 3, 128, [17, 0, 40, 1, 100], [5, 3, 0, 63, 31]),
    (48, 2, 80, [16, 32, 15], [16, 0, 1]),
    (32, 1, 256, [50, 3], [0, 14]),
    (16, 5, 96, [33], [7]),
    (16, 2, 240, [20, 1], [3, 9]),
]


@pytest.mark.parametrize("how", ["packed", "gaps", "odd", "heads_first"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:3])))
def test_write_and_read(ctx, shape, dtype, how):
    page, H, D, new, starts = shape
    g = gen(D + len(new))
    per = max((a + n + page - 1) // page for a, n in zip(starts, new))
    pool = len(new) * per + 2
    pages = page_table(g, len(new), per, pool, spare=1)
    want = Cache(pool, page, H, D, fill=0x33)
    raw = want.raw.cuda()
    off = sums(new)
    k = (torch.randn(off[-1], H, D, generator=g) * torch.rand(off[-1], H, 1, generator=g) * 7).to(dtype)
    v = (torch.randn(off[-1], H, D, generator=g) * 3).to(dtype)
    k[0, 0] = 0
    want.write(k, v, off, starts, pages)
    c = handle(ctx, want, raw)
    ks, vs = Strided(k, how), Strided(v, how)
    place = (ints(off), ints(starts), pages.cuda(), pages.shape[1])
    ng.ngemm_kv_write(ctx, c, number(dtype), len(new), off[-1], *ks.args, *vs.args, *place)
    torch.cuda.synchronize()
    if dtype is F32:
        # 127 x is rounded once and the quotient once more: codes are those of 64 bits unless 127 x / amax lies within 2^-16 of a tie
        far = (raw.cpu().int() - want.raw.int()).abs()
        assert int(far[..., :32 * D].max()) <= 1
        assert torch.equal(raw.cpu()[..., 32 * D:], want.raw[..., 32 * D:])
        y = torch.cat([127 * x.double() / x.double().abs().amax(-1, keepdim=True).clamp_min(1e-300) for x in (k, v)])
        ties = int(((y - torch.floor(y) - 0.5).abs() < 2.0 ** -16).sum())
        assert int((far[..., :32 * D] > 0).sum()) <= ties
        want.raw = raw.cpu()
    else:
        assert torch.equal(raw.cpu(), want.raw)          # every byte, those that were not to be written among them
    ko, vo = Strided(torch.full_like(k, 5), how, fill=9.0), Strided(torch.full_like(v, 5), how, fill=9.0)
    ng.ngemm_kv_read(ctx, c, number(dtype), len(new), off[-1], *ko.args, *vo.args, *place)
    torch.cuda.synchronize()
    codes = want.views()
    for out, cd, sc in ((ko, codes[0], codes[2]), (vo, codes[1], codes[3])):
        rows = torch.stack([cd[want.place(int(pages[b, at // page]), at % page)].float() * sc[want.place(int(pages[b, at // page]), at % page)].unsqueeze(-1)
                            for b in range(len(new)) for at in range(starts[b], starts[b] + new[b])]).to(dtype)
        assert torch.equal(out.window.cpu(), rows) and out.gaps_untouched()
    ng.ngemm_kv_cache_free(c)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_read_rounds_floats(ctx, dtype):
    """Every element is the float product of code and scale, rounded to the type: half a million products of any bits."""
    P, page, H, D = 32, 64, 4, 64
    g = gen(4)
    want = Cache(P, page, H, D)
    k, v, ks, vs = want.views()
    k.copy_(torch.randint(-127, 128, k.shape, generator=g))
    v.copy_(torch.randint(-127, 128, v.shape, generator=g))
    ks.copy_(torch.rand(ks.shape, generator=g) + 0.01)
    vs.copy_(torch.rand(vs.shape, generator=g) + 0.01)
    raw = want.raw.cuda()
    c = handle(ctx, want, raw)
    n = P * page
    ko, vo = (torch.empty(n, H, D, dtype=dtype, device="cuda") for _ in range(2))
    ng.ngemm_kv_read(ctx, c, number(dtype), 1, n, ko, H * D, D, vo, H * D, D, ints([0, n]), None, ints([list(range(P))]), P)
    torch.cuda.synchronize()
    for out, codes, scales in ((ko, k, ks), (vo, v, vs)):
        rows = (codes.float() * scales.unsqueeze(-1)).permute(0, 2, 3, 1, 4).reshape(n, H, D).to(dtype)
        assert torch.equal(out.cpu(), rows)
    ng.ngemm_kv_cache_free(c)


SHARED_OUT = {                                             # contexts long enough for several workgroups a tile: some long, some empty or short
    "one long": ([40, 3, 0, 300, 17], [9000, 3, 0, 300, 900]),
    "long last": ([1, 5, 200], [1, 7, 6000]),
    "rows without keys": ([130, 9, 4], [0, 5000, 2]),
    "more rows than keys": ([500, 8], [30, 4000]),
    "many": ([b % 3 for b in range(70)], [(b * 677) % 3000 if b % 5 else 0 for b in range(70)]),
    "most": ([1] * 128, [17 * b for b in range(128)]),
}


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("lengths", SHARED_OUT)
@pytest.mark.parametrize("heads", [(1, 1, 16), (3, 1, 96), (4, 1, 256)], ids=lambda h: "x".join(map(str, h)))
def test_prompt_shares_keys_out(ctx, heads, lengths, causal):
    """Each tile's parts are as many as its share of the keys of all sequences."""
    n, m = SHARED_OUT[lengths]
    assert ng.ngemm_attention_prompt_workspace_bytes(len(n), *heads, sum(n), sum(m)) > 0
    q, k, v = prompt_rows(len(n), heads, n, m, F16, 1.5)
    scale = 1 / math.sqrt(heads[2])
    got = prompt(ctx, q, k, v, n, m, causal, scale)
    check(got, *prompt_wanted(q, k, v, n, m, causal, scale), F16)


MANY_TILES = {                                             # more tiles than the chip has room for at once, of several sequences
    "ragged": ([500, 40, 0, 300, 1, 260, 129], [500, 40, 0, 300, 1, 260, 129]),
    "equal": ([270] * 4, [270] * 4),
    "behind": ([10, 600, 64, 500], [700, 601, 64, 900]),
    "ahead": ([600, 500, 7], [100, 0, 500]),
    "most": ([20 + b for b in range(64)], [20 + b + 3 * (b % 5) for b in range(64)]),
}


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("lengths", MANY_TILES)
@pytest.mark.parametrize("heads", [(64, 16, 32), (32, 16, 144)], ids=lambda h: "x".join(map(str, h)))
def test_prompt_more_tiles_than_places(ctx, heads, lengths, causal):
    n, m = MANY_TILES[lengths]
    assert ng.ngemm_attention_prompt_workspace_bytes(len(n), *heads, sum(n), sum(m)) == 0
    q, k, v = prompt_rows(len(n), heads, n, m, BF16, 1.5)
    scale = 1 / math.sqrt(heads[2])
    got = prompt(ctx, q, k, v, n, m, causal, scale)
    check(got, *prompt_wanted(q, k, v, n, m, causal, scale), BF16)


def test_prompt_infinities_where_keys_are_split(ctx):
    """As below, in a tile of a split context: one part's workgroup goes row by row, the others do not."""
    heads, n, m = (4, 2, 128), [40], [3000]
    q, k, v = prompt_rows(2, heads, n, m, BF16)
    clean = prompt_wanted(q, k, v, n, m, 1, 0.1)
    v[2990, 1, 7] = math.inf                               # seen by queries 30 .. 39
    k[2999] = math.nan                                     # seen by the last query alone
    got = prompt(ctx, q, k, v, n, m, 1, 0.1).double()
    assert bool(torch.isnan(got[39]).all()) and bool((got[30:39, 2:, 7] == math.inf).all())
    want, size = clean
    got[30:39, 2:, 7], want[30:39, 2:, 7] = 0, 0
    check(got[:39], want[:39], size[:39], BF16)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_write_extreme_rows(ctx, dtype):
    """Rows of zeros, of one element, the largest and the smallest numbers, ties, infinities and NaN."""
    D, H = 64, 1
    top, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    rows = torch.zeros(12, H, D, dtype=torch.float64)
    rows[1, 0, 5] = -3
    rows[2, 0] = torch.linspace(-top, top, D).double()
    rows[3, 0] = torch.arange(D).double() * tiny
    rows[4, 0] = torch.arange(D).double() * torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps          # subnormal
    rows[5, 0] = torch.arange(D).double() + 0.5
    rows[5, 0, 0] = 127                                                                                       # ties: x itself is the quotient
    rows[6, 0] = torch.randn(D, generator=gen(1)).double()
    rows[7, 0] = rows[6, 0]
    rows[7, 0, 63] = math.inf
    rows[8, 0, 0] = -math.inf
    rows[9, 0] = rows[6, 0]
    rows[9, 0, 17] = math.nan
    rows[10, 0] = math.nan
    rows[11, 0, 63] = tiny
    x = rows.to(dtype)
    want = Cache(1, 16, H, D)
    raw = want.raw.cuda()
    want.write(x, x, [0, 12], [2], torch.zeros(1, 1).int())
    c = handle(ctx, want, raw)
    d = x.cuda()
    place = (ints([0, 12]), ints([2]), ints([[0]]), 1)
    ng.ngemm_kv_write(ctx, c, number(dtype), 1, 12, d, D, D, d, D, D, *place)
    ko, vo = torch.empty_like(d), torch.empty_like(d)
    ng.ngemm_kv_read(ctx, c, number(dtype), 1, 12, ko, D, D, vo, D, D, *place)
    torch.cuda.synchronize()
    got = Cache(1, 16, H, D)
    got.raw = raw.cpu()
    for a, b in zip(got.views(), want.views()):
        assert torch.equal(a.nan_to_num(123.0) if a.is_floating_point() else a, b.nan_to_num(123.0) if b.is_floating_point() else b)
    codes, scales = quantise(x)
    back = (codes.float() * scales.unsqueeze(-1)).to(dtype)
    assert torch.equal(torch.isnan(ko.cpu()), torch.isnan(back)) and torch.equal(ko.cpu().nan_to_num(0.0), back.nan_to_num(0.0))
    assert torch.equal(torch.isnan(vo.cpu()), torch.isnan(back)) and torch.equal(vo.cpu().nan_to_num(0.0), back.nan_to_num(0.0))
    ng.ngemm_kv_cache_free(c)


def test_places_that_do_not_exist(ctx):
    """Positions before 0, past the table, and pages that are not the cache's: nothing is written there, 0 is read."""
    D, H, page, new = 64, 2, 16, 60
    pages = torch.tensor([[1, -1, 3, 2], [0, 9, 4, 1 << 29]]).int()       # the last page is within the table, not the cache
    starts, off = [-5, 20], [0, 40, 100]
    g = gen(3)
    k, v = (torch.randn(100, H, D, generator=g).to(F16) for _ in range(2))
    want = Cache(5, page, H, D, fill=0x11)
    raw = want.raw.cuda()
    want.write(k, v, off, starts, pages)
    c = handle(ctx, want, raw)
    place = (ints(off), ints(starts), pages.cuda(), 4)
    ng.ngemm_kv_write(ctx, c, ng.NGEMM_F16, 2, 100, k.cuda(), H * D, D, v.cuda(), H * D, D, *place)
    ko, vo = (torch.full((100, H, D), 7, dtype=F16, device="cuda") for _ in range(2))
    ng.ngemm_kv_read(ctx, c, ng.NGEMM_F16, 2, 100, ko, H * D, D, vo, H * D, D, *place)
    torch.cuda.synchronize()
    assert torch.equal(raw.cpu(), want.raw)
    for b in range(2):
        for i in range(off[b], off[b + 1]):
            at = starts[b] + i - off[b]
            there = at >= 0 and at // page < 4 and 0 <= int(pages[b, at // page]) < 5
            assert bool((ko[i] != 0).any()) == there and bool((vo[i] != 0).any()) == there
    ng.ngemm_kv_cache_free(c)


def test_broadcast_rows_and_empty_calls(ctx):
    """Strides of 0: every token and head gets the same row.  Nothing to do: nothing is touched."""
    D, H = 64, 3
    want = Cache(2, 16, H, D)
    raw = want.raw.cuda()
    c = handle(ctx, want, raw)
    row = torch.randn(D, generator=gen(1)).to(BF16)
    pages = torch.tensor([[1, 0]]).int()
    want.write(row.expand(20, H, D), row.expand(20, H, D), [0, 20], None, pages)
    d = row.cuda()
    ng.ngemm_kv_write(ctx, c, ng.NGEMM_BF16, 1, 20, d, 0, 0, d, 0, 0, ints([0, 20]), None, pages.cuda(), 2)
    ng.ngemm_kv_write(ctx, c, ng.NGEMM_BF16, 1, 0, None, 0, 0, None, 0, 0, None, None, None, 0)
    ng.ngemm_kv_write(ctx, c, ng.NGEMM_BF16, 0, 0, None, 0, 0, None, 0, 0, None, None, None, 0)
    ng.ngemm_attention_decode(ctx, c, ng.NGEMM_BF16, 0, H, None, 0, 0, None, 0, None, 0, 1.0, None, 0, 0)
    ng.ngemm_attention_prompt(ctx, ng.NGEMM_BF16, 0, H, H, D, 0, None, 0, 0, 0, None, 0, 0, None, 0, 0, None, None, 1, 1.0, None, 0, 0)
    torch.cuda.synchronize()
    assert torch.equal(raw.cpu(), want.raw)
    ng.ngemm_kv_cache_free(c)


# ---- one token per sequence ----

def filled_cache(g, lengths, page, H, D, spare=2, spread=1.0):
    """A cache that holds random rows at the sequences' positions, and NaN scales wherever nothing was written."""
    per = max(1, max((n + page - 1) // page for n in lengths))
    pool = len(lengths) * per + 2
    pages = page_table(g, len(lengths), per, pool)
    cache = Cache(pool, page, H, D, fill=-1)                # codes -1, scales NaN
    k, v, ks, vs = cache.views()
    for b, n in enumerate(lengths):
        rows = [torch.randn(n, H, D, generator=g) * spread, torch.randn(n, H, D, generator=g) * torch.rand(n, H, 1, generator=g)]
        at = torch.arange(n)
        for x, codes, scales in zip(rows, (k, v), (ks, vs)):
            codes[pages[b][at // page].long(), :, at % page // 16, at % 16], scales[pages[b][at // page].long(), :, at % page // 16, at % 16] = quantise(x)
    for b, n in enumerate(lengths):                         # what lies behind a sequence's pages is never looked up
        pages[b, (n + page - 1) // page:] = torch.tensor([-7, 1 << 30])[torch.arange(per - (n + page - 1) // page) % 2].int()
    table = torch.cat([pages, torch.full((len(lengths), spare), -9).int()], 1).contiguous()
    return cache, table


def decode(ctx, cache, table, q, lengths, scale, how="packed", max_length=None, stream=None, o_how=None):
    P, T, H, D = cache.shape
    raw = cache.raw.cuda()
    c = handle(ctx, cache, raw)
    qs, os_ = Strided(q, how), Strided(torch.full_like(q, 77), o_how or how, fill=55.0)
    most = max(lengths) if max_length is None else max_length
    size = ng.ngemm_attention_decode_workspace_bytes(q.shape[0], q.shape[1], H, D, most)
    ws = torch.full((size + 32,), 0x7f, dtype=torch.uint8, device="cuda")
    out = []
    for _ in range(2):
        ng.ngemm_attention_decode(ctx, c, number(q.dtype), q.shape[0], q.shape[1], *qs.args, ints(lengths), most, table.cuda(), table.shape[1], scale,
                                  *os_.args, ws, size, stream)
        torch.cuda.synchronize()
        out.append(os_.window.cpu().clone())
    assert os_.gaps_untouched() and bool((ws[size:] == 0x7f).all())
    assert torch.equal(out[0].nan_to_num(1e4), out[1].nan_to_num(1e4))
    ng.ngemm_kv_cache_free(c)
    return out[0]


def decode_wanted(cache, table, q, lengths, scale):
    outs, sizes = [], []
    T = cache.shape[1]
    for b, n in enumerate(lengths):
        k, v = cache.rows(table[b, :(n + T - 1) // T].tolist(), n)
        o, s = attend(q[b:b + 1].double(), k, v, scale)
        outs.append(o)
        sizes.append(s)
    return torch.cat(outs), torch.cat(sizes)


HEADS = [(1, 1, 16), (2, 1, 64), (4, 4, 80), (8, 2, 128), (12, 12, 64), (16, 1, 128), (20, 2, 96), (24, 1, 128), (40, 1, 64), (6, 2, 256), (3, 3, 240)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_decode(ctx, heads, dtype):
    Hq, H, D = heads
    g = gen(Hq + D)
    lengths = [1, 0, 15, 16, 17, 31, 63, 64, 65, 129, 300, 700]
    cache, table = filled_cache(g, lengths, 48, H, D)
    q = (torch.randn(len(lengths), Hq, D, generator=g) * 2).to(dtype)
    scale = 1 / math.sqrt(D)
    got = decode(ctx, cache, table, q, lengths, scale, how="gaps" if Hq % 3 == 0 else "packed")
    want, size = decode_wanted(cache, table, q, lengths, scale)
    assert not got[1].any()
    check(got, want, size, dtype, weights=F16)


@pytest.mark.parametrize("length", [1, 16, 100, 1023, 1024, 1025, 4097, 20000, 70001])
@pytest.mark.parametrize("heads", [(8, 2, 128), (12, 12, 64), (32, 2, 64)], ids=lambda h: "x".join(map(str, h)))
def test_decode_long(ctx, heads, length):
    """Few sequences: the work is split over their length."""
    Hq, H, D = heads
    g = gen(length)
    lengths = [length, max(1, length // 3)]
    cache, table = filled_cache(g, lengths, 64, H, D)
    q = torch.randn(2, Hq, D, generator=g).to(BF16)
    got = decode(ctx, cache, table, q, lengths, 0.2)
    want, size = decode_wanted(cache, table, q, lengths, 0.2)
    check(got, want, size, BF16, weights=F16)


@pytest.mark.parametrize("how", ["gaps", "odd", "heads_first"])
def test_decode_strides(ctx, how):
    g = gen(5)
    lengths = [77, 200, 33]
    cache, table = filled_cache(g, lengths, 16, 2, 64)
    q = torch.randn(3, 6, 64, generator=g).to(F16)
    got = decode(ctx, cache, table, q, lengths, 0.125, how=how)
    check(got, *decode_wanted(cache, table, q, lengths, 0.125), F16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.5, 1.0, 30.0])
def test_decode_scores(ctx, dtype, scale):
    """Weights that are all equal, falling the other way, and so far apart that one key takes everything."""
    g = gen(9)
    lengths = [500, 64]
    cache, table = filled_cache(g, lengths, 32, 2, 128)
    q = torch.randn(2, 8, 128, generator=g).to(dtype)
    got = decode(ctx, cache, table, q, lengths, scale)
    want, size = decode_wanted(cache, table, q, lengths, scale)
    # scores up to some thousands: a float's roundoff of the largest sum of |q k| moves an exponent by that much
    k = max(float(cache.rows(table[b, :(n + 31) // 32].tolist(), n)[0].abs().max()) for b, n in enumerate(lengths))
    slack = 128 * float(q.abs().max()) * k * abs(scale) * 2.0 ** -21
    check(got, want, size * (1 + slack / 2.0 ** -11), dtype, weights=F16)


@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_decode_query_sizes(ctx, size):
    """bfloat16 queries far outside of float16's range."""
    g = gen(10)
    lengths = [200, 40]
    cache, table = filled_cache(g, lengths, 32, 2, 64)
    q = torch.randn(2, 4, 64, generator=g).to(BF16)
    big = (q.double() * size).to(BF16)
    got = decode(ctx, cache, table, big, lengths, 0.1 / size)
    check(got, *decode_wanted(cache, table, big, lengths, 0.1 / size), BF16, weights=F16)


def test_decode_value_sizes(ctx):
    """V rows whose scales lie many powers of ten apart, and rows of zeros."""
    g = gen(11)
    lengths = [300, 65]
    cache, table = filled_cache(g, lengths, 32, 2, 64)
    vs = cache.views()[3]
    vs *= torch.exp(torch.randn(vs.shape, generator=g) * 4)
    vs[..., ::5] *= 0
    vs[..., 3] *= 1e30
    q = torch.randn(2, 4, 64, generator=g).to(BF16)
    got = decode(ctx, cache, table, q, lengths, 0.1)
    check(got, *decode_wanted(cache, table, q, lengths, 0.1), BF16, weights=F16)


def test_decode_missing_pages_and_clamped_length(ctx):
    g = gen(12)
    lengths = [200, 200, 200]
    cache, table = filled_cache(g, lengths, 16, 2, 64)
    q = torch.randn(3, 4, 64, generator=g).to(F16)
    kept = [[p for p in range(13) if p not in (0, 5, 12)], [], list(range(10))]
    full = table.clone()
    table[0, [0, 5, 12]] = torch.tensor([-1, 1 << 28, cache.shape[0]]).int()
    table[1] = -1
    # at most max_length tokens are read, and of a table no more than its own width
    got = decode(ctx, cache, table, q, [200, 200, 1 << 30], 0.2, max_length=200)
    want, size = torch.zeros(3, 4, 64, dtype=torch.float64), torch.zeros(3, 4, 64, dtype=torch.float64)
    for b, pages, n in ((0, kept[0], 160), (2, list(range(13)), 200)):
        k, v = cache.rows(full[b, pages].tolist(), n)
        o, s = attend(q[b:b + 1].double(), k, v, 0.2)
        want[b], size[b] = o[0], s[0]
    assert not got[1].any()
    check(got, want, size, F16)
    got = decode(ctx, cache, full, q, [200, -5, 1 << 30], 0.2, max_length=160)
    want, size = decode_wanted(cache, full, q, [160, 0, 160], 0.2)
    check(got, want, size, F16)
    short = full[:, :10].contiguous()
    got = decode(ctx, cache, short, q, [200, 200, 200], 0.2)
    want, size = decode_wanted(cache, full, q, [160, 160, 160], 0.2)
    check(got, want, size, F16)


def test_decode_rows_that_are_not_numbers(ctx):
    """A cached row that is NaN makes the outputs of its own sequence and head NaN; so does a query."""
    g = gen(13)
    lengths = [100, 100, 100]
    cache, table = filled_cache(g, lengths, 16, 2, 64)
    k, v, ks, vs = cache.views()
    ks[int(table[0, 2]), 1, 0, 3] = math.nan
    vs[int(table[1, 3]), 0, 0, 7] = math.nan
    q = torch.randn(3, 4, 64, generator=g).to(F16)
    q[2, 3, 9] = math.nan
    got = decode(ctx, cache, table, q, lengths, 0.2)
    bad = torch.zeros(3, 4, dtype=torch.bool)
    bad[0, 2:], bad[1, :2], bad[2, 3] = True, True, True
    assert torch.equal(torch.isnan(got).all(-1), bad) and torch.equal(torch.isnan(got).any(-1), bad)


def test_cache_past_32_bits(ctx):
    """A cache of more than 4 GiB, pages at both ends."""
    P, page, H, D = 17000, 128, 8, 128                     # 4.6 GB
    size = ng.ngemm_kv_cache_bytes(P, page, H, D)
    assert size > 1 << 32
    raw = torch.full((size,), -1, dtype=torch.int8, device="cuda")
    c = ng.ngemm_kv_cache_create(ctx, P, page, H, D, raw, size)
    g = gen(2)
    n = 300
    pages = torch.tensor([[P - 1, 3, P - 2]]).int().cuda()
    k, v = (torch.randn(n, H, D, generator=g).to(BF16).cuda() for _ in range(2))
    place = (ints([0, n]), None, pages, 3)
    ng.ngemm_kv_write(ctx, c, ng.NGEMM_BF16, 1, n, k, H * D, D, v, H * D, D, *place)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    ng.ngemm_kv_read(ctx, c, ng.NGEMM_BF16, 1, n, ko, H * D, D, vo, H * D, D, *place)
    q = torch.randn(1, 16, D, generator=g).to(BF16).cuda()
    o = torch.empty_like(q)
    wsb = ng.ngemm_attention_decode_workspace_bytes(1, 16, H, D, n)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")
    ng.ngemm_attention_decode(ctx, c, ng.NGEMM_BF16, 1, 16, q, 16 * D, D, ints([n]), n, pages, 3, 0.1, o, 16 * D, D, ws, wsb)
    torch.cuda.synchronize()
    rows = []
    for x, out in ((k, ko), (v, vo)):
        codes, scales = quantise(x.cpu())
        assert torch.equal(out.cpu(), (codes.float() * scales.unsqueeze(-1)).to(BF16))
        rows.append(codes.double() * scales.double().unsqueeze(-1))
    check(o.cpu(), *attend(q.cpu().double(), *rows, 0.1), BF16, weights=F16)
    ng.ngemm_kv_cache_free(c)


# ---- prompts ----

def prompt(ctx, q, k, v, n, m, causal, scale, how="packed", same=False):
    (_, Hq, D), H = q.shape, k.shape[1]
    qs, ks, vs, os_ = Strided(q, how), Strided(k, how), Strided(v, how), Strided(torch.full_like(q, 77), how, fill=55.0)
    size = ng.ngemm_attention_prompt_workspace_bytes(len(n), Hq, H, D, sum(n), sum(m))
    ws = torch.full((size + 32,), 0x7f, dtype=torch.uint8, device="cuda")
    out = []
    for _ in range(2):
        ng.ngemm_attention_prompt(ctx, number(q.dtype), len(n), Hq, H, D, sum(n), *qs.args, sum(m), *ks.args, *vs.args, ints(sums(n)),
                                  None if same else ints(sums(m)), causal, scale, *os_.args, ws, size)
        torch.cuda.synchronize()
        out.append(os_.window.cpu().clone())
    assert os_.gaps_untouched() and bool((ws[size:] == 0x7f).all())
    assert torch.equal(out[0].nan_to_num(1e4), out[1].nan_to_num(1e4))
    return out[0]


def prompt_wanted(q, k, v, n, m, causal, scale):
    outs, sizes, a, c = [], [], 0, 0
    for nb, mb in zip(n, m):
        i, j = torch.arange(nb).unsqueeze(1), torch.arange(mb)
        visible = (j <= i + mb - nb) if causal else torch.ones(nb, mb, dtype=torch.bool)
        o, s = attend(q[a:a + nb].double(), k[c:c + mb].double(), v[c:c + mb].double(), scale, visible)
        outs.append(o)
        sizes.append(s)
        a, c = a + nb, c + mb
    return torch.cat(outs), torch.cat(sizes)


def prompt_rows(seed, heads, n, m, dtype, spread=1.0):
    Hq, H, D = heads
    g = gen(seed)
    return ((torch.randn(sum(n), Hq, D, generator=g) * spread).to(dtype), (torch.randn(sum(m), H, D, generator=g) * spread).to(dtype),
            torch.randn(sum(m), H, D, generator=g).to(dtype))


LENGTHS = {
    "self": ([1, 0, 63, 64, 65, 130, 17], None),
    "behind": ([1, 5, 64, 100, 3, 129], [1, 70, 200, 101, 400, 129]),
    "ahead": ([70, 5, 130, 4], [3, 0, 65, 4]),             # more queries than keys: the first ones see nothing
    "long": ([300, 257], [300, 700]),
    "few": ([2, 1, 16], [1500, 3, 600]),
}


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("heads", [(1, 1, 16), (4, 2, 64), (3, 1, 80), (4, 1, 128), (2, 2, 96), (2, 1, 256), (5, 1, 208)], ids=lambda h: "x".join(map(str, h)))
def test_prompt(ctx, heads, lengths, causal, dtype):
    n, m = LENGTHS[lengths]
    q, k, v = prompt_rows(heads[2] + causal, heads, n, m or n, dtype, 1.5)
    scale = 1 / math.sqrt(heads[2])
    got = prompt(ctx, q, k, v, n, m or n, causal, scale, how="gaps" if heads[2] == 80 else "packed", same=m is None)
    check(got, *prompt_wanted(q, k, v, n, m or n, causal, scale), dtype)


@pytest.mark.parametrize("how", ["gaps", "odd", "heads_first"])
@pytest.mark.parametrize("D", [64, 128, 48])
def test_prompt_strides(ctx, how, D):
    n, m = [40, 150], [100, 150]
    q, k, v = prompt_rows(D, (4, 2, D), n, m, BF16)
    got = prompt(ctx, q, k, v, n, m, 1, 0.1, how=how)
    check(got, *prompt_wanted(q, k, v, n, m, 1, 0.1), BF16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n", [1, 33, 512, 1000])
def test_prompt_behind_a_long_context(ctx, n, dtype):
    """Few rows, a long axis."""
    m = 5000
    q, k, v = prompt_rows(n, (4, 2, 128), [n], [m], dtype)
    got = prompt(ctx, q, k, v, [n], [m], 1, 0.1)
    check(got, *prompt_wanted(q, k, v, [n], [m], 1, 0.1), dtype)


def test_prompt_many_sequences(ctx):
    n = [(7 * b) % 90 for b in range(70)]
    q, k, v = prompt_rows(1, (2, 2, 64), n, n, F16)
    got = prompt(ctx, q, k, v, n, n, 1, 0.2, same=True)
    check(got, *prompt_wanted(q, k, v, n, n, 1, 0.2), F16)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_prompt_scores(ctx, scale):
    n = [200]
    q, k, v = prompt_rows(3, (2, 1, 64), n, n, BF16)
    got = prompt(ctx, q, k, v, n, n, 1, scale)
    want, size = prompt_wanted(q, k, v, n, n, 1, scale)
    slack = 64 * float(q.abs().max()) * float(k.abs().max()) * abs(scale) * 2.0 ** -21
    check(got, want, size * (1 + slack / 2.0 ** -8), BF16)


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("heads", [(2, 1, 64), (2, 2, 128), (1, 1, 256)], ids=lambda h: "x".join(map(str, h)))
def test_prompt_not_numbers_in_masked_places(ctx, heads, value):
    """Keys and values that a query does not see have no effect on it, whatever they hold; a value that it sees has."""
    n, m = [150, 20], [170, 20]
    q, k, v = prompt_rows(8, heads, n, m, BF16)
    clean = prompt_wanted(q, k, v, n, m, 1, 0.1)
    k[169], v[169] = value, value                          # seen by the last query of the first sequence alone
    k[189], v[189] = value, value                          # the same of the second sequence
    v[100, 0, 5] = value                                   # seen by queries 80 .. 149
    got = prompt(ctx, q, k, v, n, m, 1, 0.1)
    rows = [i for i in range(170) if i not in (149, 169)]
    seeing = torch.zeros(170, heads[0], heads[2], dtype=torch.bool)
    seeing[80:150, :heads[0] // heads[1], 5] = True
    fine = ~seeing
    fine[149] = fine[169] = False
    got, want, size = got.double(), clean[0].clone(), clean[1]
    assert bool(torch.isfinite(got[fine]).all())
    bad = got[seeing & (torch.arange(170) != 149)[:, None, None]]
    assert bool((torch.isnan(bad) if math.isnan(value) else bad == value).all())
    want[~fine], got[~fine] = 0, 0
    check(got[rows], want[rows], size[rows], BF16)


# ---- streams, graphs ----

def test_other_stream_and_graph(ctx):
    """All four calls on a stream of their own, captured and replayed with other inputs: the eager results every time."""
    page, Hq, H, D, n = 16, 8, 2, 64, 40
    g = gen(21)
    cache = torch.zeros(ng.ngemm_kv_cache_bytes(8, page, H, D), dtype=torch.int8, device="cuda")
    c = ng.ngemm_kv_cache_create(ctx, 8, page, H, D, cache, cache.numel())
    pages, off, lens = ints([[3, 1, 5], [0, 7, 2]]), ints([0, n, 2 * n - 7]), ints([n, n - 7])
    t = 2 * n - 7
    q, k, v = (torch.empty(t, h, D, dtype=BF16, device="cuda") for h in (Hq, H, H))
    ko, vo, po = torch.empty_like(k), torch.empty_like(v), torch.empty_like(q)
    do = torch.empty(2, Hq, D, dtype=BF16, device="cuda")
    wsb = max(ng.ngemm_attention_decode_workspace_bytes(2, Hq, H, D, n), ng.ngemm_attention_prompt_workspace_bytes(2, Hq, H, D, t, t))
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")

    def calls():
        ng.ngemm_kv_write(ctx, c, ng.NGEMM_BF16, 2, t, k, H * D, D, v, H * D, D, off, None, pages, 3)
        ng.ngemm_kv_read(ctx, c, ng.NGEMM_BF16, 2, t, ko, H * D, D, vo, H * D, D, off, None, pages, 3)
        ng.ngemm_attention_prompt(ctx, ng.NGEMM_BF16, 2, Hq, H, D, t, q, Hq * D, D, t, ko, H * D, D, vo, H * D, D, off, None, 1, 0.2, po, Hq * D, D, ws, wsb)
        ng.ngemm_attention_decode(ctx, c, ng.NGEMM_BF16, 2, Hq, q, Hq * D, D, lens, n, pages, 3, 0.2, do, Hq * D, D, ws, wsb)

    def fill(seed):
        gg = gen(seed)
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gg).to(BF16))
        torch.cuda.synchronize()

    outs = (ko, vo, po, do)
    eager = []
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
        torch.randn(1000, device="cuda").sum().item()      # work of the program's own between replays
    ng.ngemm_kv_cache_free(c)


# ---- refusals ----

def refused(status, fn, *args):
    with pytest.raises(ng.binding.NgemmError) as e:
        fn(*args)
    assert e.value.status == status


def test_refusals(ctx):
    """Arguments that the header does not allow: an error, and nothing is launched."""
    INVALID, SHAPE, SMALL = ng.NGEMM_ERR_INVALID_ARG, ng.NGEMM_ERR_BAD_SHAPE, ng.NGEMM_ERR_BUFFER_TOO_SMALL
    D, H, Hq = 64, 2, 4
    size = ng.ngemm_kv_cache_bytes(4, 16, H, D)
    buf = torch.zeros(size + 16, dtype=torch.uint8, device="cuda")
    create = ng.ngemm_kv_cache_create
    for P, T, h, d in ((0, 16, H, D), (4, 0, H, D), (4, 24, H, D), (4, 16, 0, D), (4, 16, H, 0), (4, 16, H, 72), (4, 16, H, 272), (-1, 16, H, D), (1 << 31, 16, H, D)):
        assert ng.ngemm_kv_cache_bytes(P, T, h, d) == 0
        refused(SHAPE, create, ctx, P, T, h, d, buf, size)
    refused(INVALID, create, ctx, 4, 16, H, D, None, size)
    refused(INVALID, create, ctx, 4, 16, H, D, buf.data_ptr() + 4, size)
    refused(SMALL, create, ctx, 4, 16, H, D, buf, size - 1)
    refused(INVALID, create, None, 4, 16, H, D, buf, size)
    c = create(ctx, 4, 16, H, D, buf, size)

    x = torch.zeros(8, Hq, D, dtype=BF16, device="cuda")
    off, pages = ints([0, 8]), ints([[0]])

    def move(fn, ctx=ctx, c=c, type=ng.NGEMM_BF16, batch=1, tokens=8, k=x, kt=H * D, kh=D, v=x, vt=H * D, vh=D, off=off, pages=pages, stride=1):
        return fn, ctx, c, type, batch, tokens, k, kt, kh, v, vt, vh, off, None, pages, stride

    for fn in (ng.ngemm_kv_write, ng.ngemm_kv_read):
        for status, bad in ((INVALID, {"ctx": None}), (INVALID, {"c": None}), (INVALID, {"type": 3}), (INVALID, {"type": -1}), (SHAPE, {"batch": -1}),
                            (SHAPE, {"batch": 0}), (SHAPE, {"tokens": -1}), (SHAPE, {"tokens": 1 << 31}), (INVALID, {"k": None}), (INVALID, {"v": None}),
                            (INVALID, {"off": None}), (INVALID, {"pages": None}), (SHAPE, {"kt": -1}), (SHAPE, {"vh": -D}), (SHAPE, {"stride": -1}),
                            (INVALID, {"k": x.data_ptr() + 1})):
            refused(status, *move(fn, **bad))
    for bad in ({"kt": D}, {"vt": 0}, {"kh": 0}, {"vh": D - 1}):
        refused(SHAPE, *move(ng.ngemm_kv_read, **bad))         # outputs that overlap

    o = torch.zeros_like(x)
    lens = ints([4] * 8)

    def dec(ctx=ctx, c=c, type=ng.NGEMM_BF16, batch=8, heads=Hq, q=x, qt=Hq * D, lens=lens, most=16, pages=pages.expand(8, 1).contiguous(), stride=1, scale=0.1,
            out=o, ot=Hq * D, oh=D, ws=None, wsb=0):
        return ng.ngemm_attention_decode, ctx, c, type, batch, heads, q, qt, D, lens, most, pages, stride, scale, out, ot, oh, ws, wsb

    for status, bad in ((INVALID, {"ctx": None}), (INVALID, {"c": None}), (INVALID, {"type": ng.NGEMM_F32}), (INVALID, {"type": 9}), (SHAPE, {"batch": -1}),
                        (SHAPE, {"heads": 3}), (SHAPE, {"heads": 0}), (INVALID, {"q": None}), (SHAPE, {"qt": -1}), (INVALID, {"lens": None}), (SHAPE, {"most": -1}),
                        (INVALID, {"pages": None}), (SHAPE, {"stride": -2}), (INVALID, {"scale": math.nan}), (INVALID, {"scale": math.inf}), (INVALID, {"out": None}),
                        (SHAPE, {"ot": 0}), (SHAPE, {"oh": 1})):
        refused(status, *dec(**bad))
    need = ng.ngemm_attention_decode_workspace_bytes(1, Hq, H, D, 100000)
    if need:
        ws = torch.zeros(need + 16, dtype=torch.uint8, device="cuda")
        refused(INVALID, *dec(batch=1, most=100000, wsb=need))
        refused(SMALL, *dec(batch=1, most=100000, ws=ws, wsb=need - 1))
        refused(INVALID, *dec(batch=1, most=100000, ws=ws.data_ptr() + 4, wsb=need))

    def pro(ctx=ctx, type=ng.NGEMM_BF16, batch=1, heads=Hq, kv=H, dim=D, nq=8, q=x, qt=Hq * D, nk=8, k=x, kt=H * D, v=x, off=off, koff=None, scale=0.1, out=o, ot=Hq * D,
            ws=None, wsb=0):
        return (ng.ngemm_attention_prompt, ctx, type, batch, heads, kv, dim, nq, q, qt, D, nk, k, kt, D, v, H * D, D, off, koff, 1, scale, out, ot, D, ws, wsb)

    for status, bad in ((INVALID, {"ctx": None}), (INVALID, {"type": ng.NGEMM_F32}), (SHAPE, {"batch": -1}), (SHAPE, {"batch": 0}), (SHAPE, {"heads": 3}), (SHAPE, {"kv": 0}),
                        (SHAPE, {"dim": 24}), (SHAPE, {"dim": 512}), (SHAPE, {"nq": -1}), (INVALID, {"q": None}), (SHAPE, {"qt": -1}), (SHAPE, {"nk": -1}), (INVALID, {"k": None}),
                        (INVALID, {"v": None}), (SHAPE, {"kt": -1}), (INVALID, {"off": None}), (SHAPE, {"nk": 4}), (INVALID, {"scale": math.nan}), (INVALID, {"out": None}),
                        (SHAPE, {"ot": 0}), (INVALID, {"q": x.data_ptr() + 1})):
        refused(status, *pro(**bad))
    need = ng.ngemm_attention_prompt_workspace_bytes(1, Hq, H, D, 8, 100000)
    if need:
        big = torch.zeros(100000, H, D, dtype=BF16, device="cuda")
        ws = torch.zeros(need + 16, dtype=torch.uint8, device="cuda")
        more = {"nk": 100000, "k": big, "v": big, "koff": ints([0, 100000])}
        refused(INVALID, *pro(wsb=need, **more))
        refused(SMALL, *pro(ws=ws, wsb=need - 1, **more))
        refused(INVALID, *pro(ws=ws.data_ptr() + 4, wsb=need, **more))
    torch.cuda.synchronize()
    assert not buf.any() and not o.any()
    ng.ngemm_kv_cache_free(c)
    refused(INVALID, ng.ngemm_kv_cache_free, ctx)
    ng.ngemm_kv_cache_free(None)
