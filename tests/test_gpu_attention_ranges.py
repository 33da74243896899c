"""Attention where weights and values lie many powers of two apart, and rows too far apart."""
import math

import pytest
import torch

import paper_1910_00178_amd as ng
from attention_ref import check, quantise
from test_gpu_attention import F16, BF16, ctx, decode, decode_wanted, filled_cache, gen, prompt, prompt_rows, prompt_wanted, refused  # noqa: F401

pytestmark = pytest.mark.gpu

FORMS = {                                                  # lengths and heads: sequences in chunks, and whole ones
    "chunks": ([300, 64, 700, 1025], (4, 2, 64)),
    "whole": ([257 + 9 * b for b in range(32)], (8, 4, 64)),
    "whole, wide": ([400 + 7 * b for b in range(16)], (24, 8, 128)),
}


def put(cache, table, b, at, k, v, v_size=1.0):
    """Token `at` of sequence b: rows [head][D] of K and V, and V's scales times v_size."""
    page = cache.shape[1]
    where = cache.place(int(table[b, at // page]), at % page)
    codes = cache.views()
    for x, c, s in ((k, codes[0], codes[2]), (v, codes[1], codes[3])):
        c[where], s[where] = quantise(x)
    codes[3][where] = codes[3][where] * v_size


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("ratio", [16, 20, 24, 28, 60])
@pytest.mark.parametrize("form", FORMS)
def test_decode_large_values_of_no_weight(ctx, form, ratio, dtype):  # noqa: F811
    """A token whose values are 2^ratio times the others' and whose weight is some 2^-200 of theirs is without effect."""
    lengths, (Hq, H, D) = FORMS[form]
    g = gen(ratio)
    cache, table = filled_cache(g, lengths, 16, H, D)
    u = torch.where(torch.rand(D, generator=g) < 0.5, 1.0, -1.0)
    q = (u + 0.25 * torch.randn(len(lengths), Hq, D, generator=g)).to(dtype)
    scale = 1 / math.sqrt(D)
    for b, n in enumerate(lengths):                        # among the first tokens, in the middle, the last one
        at = (3, n // 2, n - 1)[b % 3]
        put(cache, table, b, at, (-140 / (scale * D) * u).expand(H, D), torch.randn(H, D, generator=g), 2.0 ** ratio)
    got = decode(ctx, cache, table, q, lengths, scale)
    check(got, *decode_wanted(cache, table, q, lengths, scale), dtype, weights=F16)


@pytest.mark.parametrize("weight", [-30, -12, 0, 12])
@pytest.mark.parametrize("form", FORMS)
def test_decode_large_values_of_some_weight(ctx, form, weight):  # noqa: F811
    """The same with 2^20 times the values and weights of about 2^weight: sometimes they count, sometimes the others do."""
    lengths, (Hq, H, D) = FORMS[form]
    g = gen(100 + weight)
    cache, table = filled_cache(g, lengths, 32, H, D)
    u = torch.where(torch.rand(D, generator=g) < 0.5, 1.0, -1.0)
    q = (u + 0.05 * torch.randn(len(lengths), Hq, D, generator=g)).to(BF16)
    scale = 1 / math.sqrt(D)
    for b, n in enumerate(lengths):
        put(cache, table, b, (n - 1, 3, n // 2)[b % 3], (weight * math.log(2) / (scale * D) * u).expand(H, D), torch.randn(H, D, generator=g), 2.0 ** 20)
    got = decode(ctx, cache, table, q, lengths, scale)
    check(got, *decode_wanted(cache, table, q, lengths, scale), BF16, weights=F16)


@pytest.mark.parametrize("size", [2.0 ** -110, 2.0 ** -60, 2.0 ** 60, 2.0 ** 110])
@pytest.mark.parametrize("form", FORMS)
def test_decode_sizes_of_all_values(ctx, form, size):  # noqa: F811
    """All values very small or very large, the weights falling from token to token or rising."""
    lengths, (Hq, H, D) = FORMS[form]
    g = gen(3)
    cache, table = filled_cache(g, lengths, 32, H, D)
    u = torch.where(torch.rand(D, generator=g) < 0.5, 1.0, -1.0)
    q = (u + 0.05 * torch.randn(len(lengths), Hq, D, generator=g)).to(BF16)
    scale = 1 / math.sqrt(D)
    for b, n in enumerate(lengths):
        for at in range(0, n, 7):
            put(cache, table, b, at, ((at if b % 2 else n - at) * 100 / n / (scale * D) * u).expand(H, D), torch.randn(H, D, generator=g))
    cache.views()[3].mul_(size)
    got = decode(ctx, cache, table, q, lengths, scale)
    want, bound = decode_wanted(cache, table, q, lengths, scale)
    check(got.double() / size, want / size, bound / size, BF16, weights=F16)


@pytest.mark.parametrize("below", [20.5, 25.2, 30.5])
@pytest.mark.parametrize("values", ["small", "half", "none"])
@pytest.mark.parametrize("form", [([40000], (2, 1, 64)), ([2000 - 3 * b for b in range(32)], (8, 4, 64))], ids=["chunks", "whole"])
def test_decode_many_small_weights(ctx, form, values, below):  # noqa: F811
    """One token of weight 1, whose values are small or 0 in half of the elements or everywhere, before or behind many of weight 2^-below."""
    lengths, (Hq, H, D) = form
    g = gen(17)
    cache, table = filled_cache(g, lengths, 16, H, D)
    cache.views()[0].zero_()                               # keys: score 0
    u = torch.where(torch.rand(D, generator=g) < 0.5, 1.0, -1.0)
    q = u.expand(len(lengths), Hq, D).to(BF16).contiguous()
    scale = 1 / math.sqrt(D)
    for b, n in enumerate(lengths):
        v = torch.randn(H, D, generator=g)
        v[:, ::2] *= 0 if values == "half" else 1
        put(cache, table, b, (0, n - 1, n // 3)[b % 3], (below * math.log(2) / (scale * D) * u).expand(H, D), v, {"small": 2.0 ** -10, "half": 1.0, "none": 0.0}[values])
    got = decode(ctx, cache, table, q, lengths, scale)
    check(got, *decode_wanted(cache, table, q, lengths, scale), BF16, weights=F16)


@pytest.mark.parametrize("below", [20.2, 24.2, 30.2])
@pytest.mark.parametrize("values", ["small", "half", "none"])
@pytest.mark.parametrize("at", ["first", "middle", "last"])
@pytest.mark.parametrize("sizes", [(3, 20000, (2, 1, 64)), (70, 1000, (4, 2, 128)), (5, 9000, (2, 1, 256))], ids=lambda s: f"{s[0]}x{s[1]}x{s[2][2]}")
def test_prompt_many_small_weights(ctx, sizes, at, values, below):  # noqa: F811
    """float16: one key of weight 1, whose values are small or 0 in half of the elements or everywhere, among many of weight 2^-below."""
    n, m, heads = sizes
    q, k, v = prompt_rows(n, heads, [n], [m], F16)
    u = torch.where(torch.rand(heads[2], generator=gen(1)) < 0.5, 1.0, -1.0)
    q[:], k[:] = u.to(F16), 0
    where = {"first": 0, "middle": m // 2, "last": m - 1}[at]
    k[where] = u.to(F16)
    v[where] *= 2.0 ** -10 if values == "small" else 0.0 if values == "none" else 1.0
    v[where, :, ::2] *= 0 if values == "half" else 1
    scale = below * math.log(2) / heads[2]
    got = prompt(ctx, q, k, v, [n], [m], 0, scale)
    want, size = prompt_wanted(q, k, v, [n], [m], 0, scale)
    if below > 25:                                         # weights on a grid: 2^-36 each, in the bound's units of its factor of size
        size = size + 2.0 ** -36 / (2.0 ** -11 + 2.0 ** -13) * v.double().abs().sum(0).repeat_interleave(heads[0] // heads[1], 0)
    check(got, want, size, F16)


def test_prompt_parts_row_by_row_in_float16(ctx):  # noqa: F811
    """One part of a split context goes row by row because of an infinity, the others do not: their sums have the same factor."""
    heads, n, m = (4, 2, 128), [40], [3000]
    q, k, v = prompt_rows(2, heads, n, m, F16)
    want, size = prompt_wanted(q, k, v, n, m, 1, 0.1)
    v[2990, 1, 7] = math.inf                               # seen by queries 30 .. 39
    got = prompt(ctx, q, k, v, n, m, 1, 0.1).double()
    assert bool((got[30:, 2:, 7] == math.inf).all())
    got[30:, 2:, 7], want[30:, 2:, 7] = 0, 0
    check(got, want, size, F16)


def test_rows_too_far_apart(ctx):  # noqa: F811
    """Strides whose products with the rows' number pass 63 bits are refused, whether rows are read or written, before anything is launched."""
    D, H, far = 64, 8, 1 << 40
    size = ng.ngemm_kv_cache_bytes(4, 16, H, D)
    buf = torch.zeros(size, dtype=torch.uint8, device="cuda")
    c = ng.ngemm_kv_cache_create(ctx, 4, 16, H, D, buf, size)
    x = torch.zeros(16, H, D, dtype=BF16, device="cuda")
    pages, off = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([0, 16], dtype=torch.int32, device="cuda")
    for tokens in ((1 << 20) + 1, (1 << 23) + 1):          # 2^60 and some; 2^63: as 64 bits with a sign the heads seemed to lie behind each other
        for head_stride in (0, D, far):
            refused(ng.NGEMM_ERR_BAD_SHAPE, ng.ngemm_kv_read, ctx, c, ng.NGEMM_BF16, 1, tokens, x, far, head_stride, x, H * D, D, off, None, pages, 1)
            refused(ng.NGEMM_ERR_BAD_SHAPE, ng.ngemm_kv_write, ctx, c, ng.NGEMM_BF16, 1, tokens, x, H * D, D, x, far, head_stride, off, None, pages, 1)
            refused(ng.NGEMM_ERR_BAD_SHAPE, ng.ngemm_attention_prompt, ctx, ng.NGEMM_BF16, 1, H, H, D, tokens, x, H * D, D, tokens, x, far, head_stride, x, H * D, D,
                    off, None, 1, 0.1, x, H * D, D)
    torch.cuda.synchronize()
    assert not buf.any() and not x.any()
    ng.ngemm_kv_cache_free(c)


@pytest.mark.parametrize("power", [-115, -100, 100, 115])
@pytest.mark.parametrize("form", FORMS)
def test_decode_sizes_of_queries_and_keys(ctx, form, power):  # noqa: F811
    """Keys of any size and bfloat16 queries of the inverse one: scores as ever."""
    lengths, (Hq, H, D) = FORMS[form]
    g = gen(power + 200)
    cache, table = filled_cache(g, lengths, 32, H, D)
    cache.views()[2].mul_(2.0 ** power)
    q = (torch.randn(len(lengths), Hq, D, generator=g).double() * 2.0 ** -power).to(BF16)
    scale = 1 / math.sqrt(D)
    got = decode(ctx, cache, table, q, lengths, scale)
    check(got, *decode_wanted(cache, table, q, lengths, scale), BF16, weights=F16)
