"""The forms of the cache's and attention's kernels that small batches do not reach: whole sequences by eight wavefronts, several heads a workgroup,
more sequences than a wavefront has lanes."""
import math

import pytest
import torch

import paper_1910_00178_amd as ng
from attention_ref import Cache, attend, check, quantise
from test_gpu_attention import (BF16, F16, F32, Strided, ctx, decode, decode_wanted, filled_cache, gen, handle, ints, number, page_table, prompt,  # noqa: F401
                                prompt_rows, prompt_wanted, sums)
from test_gpu_routes import launches  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- whole sequences ----

WHOLE = [  # query heads, K/V heads, D, sequences: 128 units and more, up to 2048 tokens, heads of up to 192
    (8, 4, 64, 32), (12, 12, 16, 16), (24, 8, 128, 16), (20, 2, 96, 64), (64, 4, 128, 32), (6, 6, 80, 24), (9, 3, 192, 44), (34, 1, 112, 43), (4, 4, 144, 32),
]


def ragged(batch, most):
    """Lengths with empty ones, single tokens, ends inside and on blocks and tiles."""
    special = [most, 0, 1, 15, 16, 17, 63, 64, 65, 511, 512, 513]
    return [special[b] if b < len(special) and special[b] <= most else (b * 7919) % most + 1 for b in range(batch)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("most", [257, 700, 2048])
@pytest.mark.parametrize("heads", WHOLE, ids=lambda h: "x".join(map(str, h)))
def test_decode_whole(ctx, heads, most, dtype):  # noqa: F811
    Hq, H, D, batch = heads
    if most == 2048 and D * H > 512:
        batch = max(1, -(-128 // (H * -(-Hq // H // 16))))
    g = gen(most + D)
    lengths = ragged(batch, most)
    cache, table = filled_cache(g, lengths, 48, H, D)
    q = (torch.randn(batch, Hq, D, generator=g) * 2).to(dtype)
    scale = 1 / math.sqrt(D)
    got = decode(ctx, cache, table, q, lengths, scale)
    assert not got[1].any()
    check(got, *decode_wanted(cache, table, q, lengths, scale), dtype, weights=F16)


def test_decode_forms_that_are_launched(ctx, launches):  # noqa: F811
    """The sizes of these tests reach the forms that they are for."""
    def names(Hq, H, D, batch, most):
        size = ng.ngemm_kv_cache_bytes(1, 16, H, D)
        raw = torch.zeros(size, dtype=torch.uint8, device="cuda")
        c = ng.ngemm_kv_cache_create(ctx, 1, 16, H, D, raw, size)
        x, pages = torch.zeros(batch, Hq, D, dtype=BF16, device="cuda"), torch.zeros(batch, 1, dtype=torch.int32, device="cuda")
        wsb = ng.ngemm_attention_decode_workspace_bytes(batch, Hq, H, D, most)
        ws = torch.empty(max(16, wsb), dtype=torch.uint8, device="cuda")
        seen = launches(lambda st: ng.ngemm_attention_decode(ctx, c, ng.NGEMM_BF16, batch, Hq, x, Hq * D, D, pages, most, pages, 1, 0.1, x, Hq * D, D, ws, wsb, st))
        ng.ngemm_kv_cache_free(c)
        return seen

    for Hq, H, D, batch in WHOLE:
        units = batch * H * -(-Hq // H // 16)
        assert units >= 128 and names(Hq, H, D, batch, 2048) == [(f"attention_decode_kernel<BF16, {D}, 8>", units)]
    for Hq, H, D, batch, most in ((8, 4, 64, 32, 256), (8, 4, 64, 31, 2000), (8, 4, 64, 32, 2049), (4, 4, 208, 32, 2000)):
        seen = names(Hq, H, D, batch, most)
        assert seen[0][0] == f"attention_decode_kernel<BF16, {D}, 4>"
        assert [n for n, _ in seen[1:]] == ([f"attention_decode_join_kernel<BF16, {D}>"] if seen[0][1] > batch * H else [])


@pytest.mark.parametrize("how", ["gaps", "odd", "heads_first"])
def test_decode_whole_strides(ctx, how):  # noqa: F811
    g = gen(6)
    lengths = ragged(22, 600)
    cache, table = filled_cache(g, lengths, 16, 6, 64)
    q = torch.randn(22, 18, 64, generator=g).to(F16)
    got = decode(ctx, cache, table, q, lengths, 0.125, how=how)
    check(got, *decode_wanted(cache, table, q, lengths, 0.125), F16)


@pytest.mark.parametrize("D", [64, 128])
def test_decode_whole_missing_pages_and_clamped_length(ctx, D):  # noqa: F811
    g = gen(14)
    lengths = [300 + 11 * b for b in range(32)]
    cache, table = filled_cache(g, lengths, 16, 4, D)
    q = torch.randn(32, 8, D, generator=g).to(F16)
    full = table.clone()
    missing = {0: [0], 1: [5, 6, 7, 8], 2: [18], 3: list(range(21)), 9: [2, 3], 31: [40]}
    for b, pages in missing.items():
        table[b, pages] = torch.tensor([-1, 1 << 28, cache.shape[0]])[torch.arange(len(pages)) % 3].int()
    given = [n if b % 4 else 1 << 30 for b, n in enumerate(lengths)]
    given[5] = -3
    got = decode(ctx, cache, table, q, given, 0.2, max_length=600)
    want, size = torch.zeros(32, 8, D, dtype=torch.float64), torch.zeros(32, 8, D, dtype=torch.float64)
    for b, n in enumerate(lengths):
        n = 0 if b == 5 else min(n, 600) if b % 4 else min(600, (n + 15) // 16 * 16)         # (a length too long: to the table's end, with what its last page holds)
        pages = [p for p in range((n + 15) // 16) if p not in missing.get(b, ())]
        if not pages or n == 0:
            continue
        k, v = cache.rows(full[b, pages].tolist(), 16 * len(pages))
        last = n - 16 * pages[-1] if pages[-1] == (n + 15) // 16 - 1 else 16
        k, v = k[:16 * (len(pages) - 1) + last], v[:16 * (len(pages) - 1) + last]
        o, s = attend(q[b:b + 1].double(), k, v, 0.2)
        want[b], size[b] = o[0], s[0]
    for b in range(0, 32, 4):                              # (their last pages hold NaN behind the sequence's end where it ends inside one)
        if lengths[b] % 16 and lengths[b] < 600:
            assert bool(torch.isnan(got[b]).all())
            got[b], want[b], size[b] = 0, 0, 0
    assert not got[3].any() and not got[5].any()
    check(got, want, size, F16)


def test_decode_whole_rows_that_are_not_numbers(ctx):  # noqa: F811
    g = gen(15)
    lengths = [300 + b for b in range(32)]
    cache, table = filled_cache(g, lengths, 16, 4, 96)
    k, v, ks, vs = cache.views()
    ks[int(table[0, 2]), 1, 0, 3] = math.nan
    vs[int(table[7, 18]), 0, 0, 7] = math.nan
    q = torch.randn(32, 12, 96, generator=g).to(BF16)
    q[2, 3, 9], q[31, 11, 95] = math.nan, math.inf
    got = decode(ctx, cache, table, q, lengths, 0.2)
    bad = torch.zeros(32, 12, dtype=torch.bool)
    bad[0, 3:6], bad[7, :3], bad[2, 3], bad[31, 11] = True, True, True, True
    assert torch.equal(torch.isnan(got).all(-1), bad) and torch.equal(torch.isnan(got).any(-1), bad)


# ---- many sequences ----

@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("batch", [64, 65, 200, 4097])
def test_write_and_read_many_sequences(ctx, batch, dtype):  # noqa: F811
    """More sequences than a wavefront has lanes, and than its square: empty ones, single tokens, some behind a start inside a block."""
    H, D, page = 2, 32, 16
    g = gen(batch)
    new = [(0, 1, 3, 0, 17)[b % 5] for b in range(batch)]
    starts = [(7 * b) % 23 for b in range(batch)]
    new[-1] = 2
    off, per = sums(new), 3
    pages = page_table(g, batch, per, batch * per + 1)
    raw = torch.zeros(ng.ngemm_kv_cache_bytes(batch * per + 1, page, H, D), dtype=torch.int8, device="cuda")
    cache = Cache(batch * per + 1, page, H, D)
    c = handle(ctx, cache, raw)
    k, v = (torch.randn(off[-1], H, D, generator=g).to(dtype) for _ in range(2))
    place = (ints(off), ints(starts), pages.cuda(), per)
    ng.ngemm_kv_write(ctx, c, number(dtype), batch, off[-1], k.cuda(), H * D, D, v.cuda(), H * D, D, *place)
    ko, vo = (torch.full_like(x, 7).cuda() for x in (k, v))
    ng.ngemm_kv_read(ctx, c, number(dtype), batch, off[-1], ko, H * D, D, vo, H * D, D, *place)
    torch.cuda.synchronize()
    cache.raw = raw.cpu().view(cache.raw.shape)
    seq = torch.repeat_interleave(torch.arange(batch), torch.tensor(new))
    at = torch.arange(off[-1]) - torch.tensor(off)[seq] + torch.tensor(starts)[seq]
    where = (pages[seq, at // page].long(), slice(None), at % page // 16, at % 16)
    written = torch.zeros(cache.raw.shape[:1] + (16,), dtype=torch.bool)
    written[where[0], where[3]] = True
    codes = cache.views()
    for x, out, cd, sc in ((k, ko, codes[0], codes[2]), (v, vo, codes[1], codes[3])):
        want, scales = quantise(x)
        # (floats: 127 x is rounded once and the quotient once more: a code may lie beside that of 64 bits at a tie)
        assert int((cd[where].int() - want.int()).abs().max()) <= (1 if dtype is F32 else 0) and torch.equal(sc[where], scales)
        assert torch.equal(out.cpu(), (cd[where].float() * sc[where].unsqueeze(-1)).to(dtype))
        there = written[:, None, None, :].expand(sc.shape)
        assert not sc[~there].any() and not cd[~there].any()                  # nothing else is written
    ng.ngemm_kv_cache_free(c)


@pytest.mark.parametrize("how", ["packed", "odd"])
@pytest.mark.parametrize("heads", [8, 9])
def test_write_and_read_several_heads_a_workgroup(ctx, heads, how):  # noqa: F811
    """Enough tokens for two heads a workgroup, an odd number of heads among them."""
    D, page, new, starts = 48, 32, [6001, 0, 3100], [13, 0, 2]
    g = gen(heads)
    per = -(-6020 // page)
    pages = page_table(g, 3, per, 3 * per + 1)
    raw = torch.zeros(ng.ngemm_kv_cache_bytes(3 * per + 1, page, heads, D), dtype=torch.int8, device="cuda")
    cache = Cache(3 * per + 1, page, heads, D)
    c = handle(ctx, cache, raw)
    off = sums(new)
    k, v = (torch.randn(off[-1], heads, D, generator=g).to(BF16) for _ in range(2))
    place = (ints(off), ints(starts), pages.cuda(), per)
    ks, vs = Strided(k, how), Strided(v, how)
    ng.ngemm_kv_write(ctx, c, ng.NGEMM_BF16, 3, off[-1], *ks.args, *vs.args, *place)
    ko, vo = Strided(torch.zeros_like(k), how, fill=3.0), Strided(torch.zeros_like(v), how, fill=3.0)
    ng.ngemm_kv_read(ctx, c, ng.NGEMM_BF16, 3, off[-1], *ko.args, *vo.args, *place)
    torch.cuda.synchronize()
    cache.raw = raw.cpu().view(cache.raw.shape)
    seq = torch.repeat_interleave(torch.arange(3), torch.tensor(new))
    at = torch.arange(off[-1]) - torch.tensor(off)[seq] + torch.tensor(starts)[seq]
    where = (pages[seq, at // page].long(), slice(None), at % page // 16, at % 16)
    codes = cache.views()
    for x, out, cd, sc in ((k, ko, codes[0], codes[2]), (v, vo, codes[1], codes[3])):
        want, scales = quantise(x)
        assert torch.equal(cd[where], want) and torch.equal(sc[where], scales)
        assert torch.equal(out.window.cpu(), (want.float() * scales.unsqueeze(-1)).to(BF16)) and out.gaps_untouched()
    ng.ngemm_kv_cache_free(c)


@pytest.mark.parametrize("causal", [0, 1])
def test_prompt_thousands_of_sequences(ctx, causal):  # noqa: F811
    n = [(5 * b) % 13 for b in range(4200)]
    m = [x + b % 4 for b, x in enumerate(n)]
    q, k, v = prompt_rows(3, (2, 1, 32), n, m, F16)
    got = prompt(ctx, q, k, v, n, m, causal, 0.2)
    check(got, *prompt_wanted(q, k, v, n, m, causal, 0.2), F16)
