"""Attention of new tokens where scores, weights and values lie many powers of two apart, and scores of minus infinity."""
import math

import pytest
import torch

from attention_ref import attend, check
from test_gpu_attention import F16, BF16, ctx, gen  # noqa: F401
from test_gpu_attention_chunk import make, run, seen, wanted, weights
from test_gpu_attention_ranges import put

pytestmark = pytest.mark.gpu

FORMS = {                                                  # new tokens, starts, heads: few rows and many, keys whole and shared out
    "few": ([1, 3, 2, 1], [299, 61, 430, 200], (4, 2, 64)),
    "few, shared": ([1, 3, 1, 2], [299, 61, 3000, 1022], (4, 2, 64)),
    "few, eight wavefronts": ([1 + b % 2 for b in range(16)], [400 + 7 * b for b in range(16)], (24, 8, 128)),
    "some": ([9, 16], [300, 64], (4, 2, 128)),
    "some, shared": ([9, 16], [2000, 300], (4, 2, 64)),
    "few, large heads": ([2, 9], [700, 90], (2, 1, 256)),
    "many": ([40, 70], [300, 64], (4, 2, 64)),
    "many, shared": ([40, 130], [3000, 400], (4, 2, 128)),
    "many, large heads": ([150], [700], (2, 1, 256)),
    "wide": ([300, 280], [1500, 1200], (2, 2, 64)),
    "wide, 96": ([200, 140], [1500, 900], (2, 1, 96)),
    "wide, 128": ([200, 140], [1500, 900], (4, 2, 128)),
}


def signs(D, seed=1):
    return torch.where(torch.rand(D, generator=gen(seed)) < 0.5, 1.0, -1.0)


def places(start):
    """Positions before a sequence's new tokens, one of them by turns."""
    return 3, start // 2, start - 1


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("ratio", [20, 60, 80])
@pytest.mark.parametrize("form", FORMS)
def test_large_values_of_no_weight(ctx, form, ratio, dtype):  # noqa: F811
    """A token whose values are 2^ratio times the others' and whose weight is some 2^-200 of theirs is without effect."""
    new, starts, heads = FORMS[form]
    D, scale, u = heads[2], 1 / math.sqrt(heads[2]), signs(heads[2])
    g = gen(ratio)
    cache, table, _ = make(ratio, heads, new, starts, dtype)
    q = (u + 0.25 * torch.randn(sum(new), heads[0], D, generator=g)).to(dtype)
    for b, start in enumerate(starts):
        put(cache, table, b, places(start)[b % 3], (-140 / (scale * D) * u).expand(heads[1], D), torch.randn(heads[1], D, generator=g), 2.0 ** ratio)
    got = run(ctx, cache, table, q, new, starts, scale=scale)
    check(got, *wanted(cache, table, q, new, starts, scale=scale), dtype, weights=weights(heads, new, dtype))


@pytest.mark.parametrize("weight", [-30, -12, 0, 12])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("form", FORMS)
def test_large_values_of_some_weight(ctx, form, dtype, weight):  # noqa: F811
    """Values of 2^10 (f16) or 2^20 times the others' and weights of about 2^weight: sometimes they count, sometimes the others do."""
    new, starts, heads = FORMS[form]
    D, scale, u = heads[2], 1 / math.sqrt(heads[2]), signs(heads[2])
    g = gen(100 + weight)
    cache, table, _ = make(200 + weight, heads, new, starts, dtype)
    q = (u + 0.05 * torch.randn(sum(new), heads[0], D, generator=g)).to(dtype)
    for b, start in enumerate(starts):
        put(cache, table, b, places(start)[(b + 1) % 3], (weight * math.log(2) / (scale * D) * u).expand(heads[1], D), torch.randn(heads[1], D, generator=g),
            2.0 ** (10 if dtype is F16 else 20))
    got = run(ctx, cache, table, q, new, starts, scale=scale)
    check(got, *wanted(cache, table, q, new, starts, scale=scale), dtype, weights=weights(heads, new, dtype))


@pytest.mark.parametrize("rise", [0.04, 0.2, 1.5])
@pytest.mark.parametrize("power", [-110, -60, 0, 60, 87])
@pytest.mark.parametrize("form", FORMS)
def test_sizes_of_all_values(ctx, form, power, rise):  # noqa: F811
    """Values of up to 2^90 or very small ones, while scores rise from token to token or fall: by less than 2^12 in a tile, by about that, and by more;
    with rise 1.5 up to a few hundreds, and level from there on."""
    new, starts, heads = FORMS[form]
    D, u = heads[2], signs(heads[2])
    cache, table, _ = make(300 + power, heads, new, starts, BF16)
    q = u.expand(sum(new), heads[0], D).to(BF16).contiguous()
    kc, _, ks, vs = cache.views()
    kc.copy_((127 * u).to(torch.int8).expand(kc.shape))
    # <q, K> = 127 D ks: ks makes a score log2 of the weight; 400 at most
    for b, (n, start) in enumerate(zip(new, starts)):
        at = torch.arange(start + n)
        bits = (rise * at).clamp_max(400.0) if b % 2 == 0 else (400 - rise * at).clamp_min(0.0)
        where = (table[b, at // cache.shape[1]].long(), slice(None), at % cache.shape[1] // 16, at % 16)
        ks[where] = (bits * math.log(2) / (127 * D)).float().unsqueeze(1).expand(-1, heads[1])
    vs.mul_(2.0 ** power)
    got = run(ctx, cache, table, q, new, starts, scale=1.0)
    want, size = wanted(cache, table, q, new, starts, scale=1.0)
    assert float(want.abs().max()) < 2.0 ** 90
    check(got.double() * 2.0 ** -power, want * 2.0 ** -power, size * 2.0 ** -power, BF16, weights=weights(heads, new, BF16))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [(0, 0), (37, 3)], ids=["all", "window"])
@pytest.mark.parametrize("form", FORMS)
def test_scores_of_minus_infinity(ctx, form, window, dtype):  # noqa: F811
    """K scales of infinity under codes whose products with the queries are below 0.  Rows that see nothing else give 0, in the tiles of rows that do as well."""
    new, starts, heads = FORMS[form]
    H, D, page = heads[1], heads[2], 48
    for which in ("all", "up to the middle", "some"):
        cache, table, q = make(31, heads, new, starts, dtype, page=page)
        q = (torch.rand(q.shape, generator=gen(4)) + 0.1).to(dtype)
        kc, _, ks, _ = cache.views()
        lost = []
        for b, (n, start) in enumerate(zip(new, starts)):
            at = torch.arange(start + n)
            bad = torch.ones(start + n, dtype=torch.bool) if which == "all" else at <= start + (n - 1) // 2 if which == "up to the middle" else at % 5 < 2
            lost.append(bad)
            where = (table[b, at[bad] // page].long(), slice(None), at[bad] % page // 16, at[bad] % 16)
            kc[where] = -1 - torch.randint(0, 126, (int(bad.sum()), H, D), generator=gen(b)).to(torch.int8)
            ks[where] = 1.0
        outs, sizes, first = [], [], 0
        for b, (n, start) in enumerate(zip(new, starts)):
            k, v = cache.rows(table[b, :(start + n + page - 1) // page].tolist(), start + n)
            o, s = attend(q[first:first + n].double(), k, v, 0.125, seen(n, start, start + n, *window) & ~lost[b])
            outs.append(o)
            sizes.append(s)
            first += n
            at = torch.arange(start + n)[lost[b]]
            ks[(table[b, at // page].long(), slice(None), at % page // 16, at % 16)] = math.inf
        want = torch.cat(outs)
        if which == "all":
            assert not want.any()
        got = run(ctx, cache, table, q, new, starts, *window)
        assert not got[(want == 0).flatten(1).all(1)].any()
        check(got, want, torch.cat(sizes), dtype, weights=weights(heads, new, dtype))


@pytest.mark.parametrize("power", [-115, -100, 100, 115])
@pytest.mark.parametrize("form", FORMS)
def test_sizes_of_queries_and_keys(ctx, form, power):  # noqa: F811
    """Keys of any size and bfloat16 queries of the inverse one: scores as ever."""
    new, starts, heads = FORMS[form]
    scale = 1 / math.sqrt(heads[2])
    cache, table, q = make(400 + power, heads, new, starts, BF16)
    cache.views()[2].mul_(2.0 ** power)
    q = (torch.randn(q.shape, generator=gen(power + 500)).double() * 2.0 ** -power).to(BF16)
    got = run(ctx, cache, table, q, new, starts, scale=scale)
    check(got, *wanted(cache, table, q, new, starts, scale=scale), BF16, weights=weights(heads, new, BF16))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("below", [20.5, 25.2, 30.5])
@pytest.mark.parametrize("values", ["small", "half", "none"])
@pytest.mark.parametrize("form", [([3], [20000], (2, 1, 64)), ([2] * 20, [1500 - 3 * b for b in range(20)], (8, 8, 64)), ([100], [20000], (2, 1, 128)),
                                  ([280], [9000], (2, 2, 96))], ids=["few", "eight", "many", "wide"])
def test_many_small_weights(ctx, form, values, below, dtype):  # noqa: F811
    """One token of weight 1, whose values are small or 0 in half of the elements or everywhere, before or behind many of weight 2^-below."""
    new, starts, heads = form
    H, D = heads[1:]
    g, u, scale = gen(17), signs(D), 1 / math.sqrt(D)
    cache, table, _ = make(17, heads, new, starts, dtype, page=16)
    cache.views()[0].zero_()                               # keys: score 0
    q = u.expand(sum(new), heads[0], D).to(dtype).contiguous()
    for b, start in enumerate(starts):
        v = torch.randn(H, D, generator=g)
        v[:, ::2] *= 0 if values == "half" else 1
        put(cache, table, b, places(start)[b % 3], (below * math.log(2) / (scale * D) * u).expand(H, D), v, {"small": 2.0 ** -10, "half": 1.0, "none": 0.0}[values])
    got = run(ctx, cache, table, q, new, starts, scale=scale)
    check(got, *wanted(cache, table, q, new, starts, scale=scale), dtype, weights=weights(heads, new, dtype))
