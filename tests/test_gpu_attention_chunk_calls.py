"""Attention of new tokens, norms and rotations: calls that are unusual but allowed."""
import math
import os
import subprocess
import sys

import pytest
import torch

import paper_1910_00178_amd as ng
from attention_ref import attend, check
from test_gpu_attention import BF16, F16, F32, ctx, gen, handle, ints, sums  # noqa: F401
from test_gpu_attention_chunk import make, run, seen, wanted, weights
from test_gpu_rotation import HALVES, NEIGHBOURS, Rotation, check_turn, check_write

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FIRST_USE = """
import sys
sys.path.insert(0, {root!r})
import torch
import paper_1910_00178_amd as ng
ctx = ng.ngemm_create(0)
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
g = torch.Generator().manual_seed(1)
rows = lambda n, h, d: torch.randn(n, h, d, generator=g).to(torch.bfloat16).cuda()
Hq, H, D, per, page = 8, 2, 256, 40, 32                    # more than 64 KiB of LDS for few rows and for many
n, new, starts = 190, [1, 9, 180], [700, 300, 200]
past = rows(1200, H, D)
angles, w = torch.rand(per * page, D, generator=g).cuda(), torch.rand(D, generator=g).cuda()
rotation = ng.ngemm_rotation_create(ctx, per * page, D, ng.NGEMM_PAIRS_HALVES, angles, angles.numel() * 4)
q, k, v, qo, o = rows(n, Hq, D), rows(n, H, D), rows(n, H, D), rows(n, Hq, D), rows(n, Hq, D)
size = ng.ngemm_kv_cache_bytes(3 * per, page, H, D)
raw = torch.zeros(size, dtype=torch.uint8, device="cuda")
c = ng.ngemm_kv_cache_create(ctx, 3 * per, page, H, D, raw, size)
pages, off, start, at = ints(list(range(3 * per))).view(3, per), ints([0, 1, 10, 190]), ints(starts), ints([a + i for a, b in zip(starts, new) for i in range(b)])
before, ends = ints([0, 700, 1000, 1200]), None
need = ng.ngemm_attention_chunk_workspace_bytes(3, Hq, H, D, n, 180, 701, 0, 0)
assert need > 0
ws = torch.empty(need, dtype=torch.uint8, device="cuda")
def calls():
    ng.ngemm_kv_write_rotated(ctx, c, ng.NGEMM_BF16, 3, 1200, past, H * D, D, past, H * D, D, None, 0.0, None, before, None, pages, per)
    ng.ngemm_qk_norm_rotate(ctx, ng.NGEMM_BF16, D, n, Hq, q, Hq * D, D, w, 0, None, 0, 0, None, 1e-6, rotation, at, qo, Hq * D, D, None, 0, 0)
    ng.ngemm_kv_write_rotated(ctx, c, ng.NGEMM_BF16, 3, n, k, H * D, D, v, H * D, D, w, 1e-6, rotation, off, start, pages, per)
    ng.ngemm_attention_chunk(ctx, c, ng.NGEMM_BF16, 3, Hq, n, qo, Hq * D, D, off, start, 180, 701, pages, per, 0, 0, 0.1, o, Hq * D, D, ws, need)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
found = []
for _ in range(3):
    for x in (qo, o, raw):
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    found.append((qo.clone(), o.clone(), raw.clone()))
for x in (qo, o, raw):
    x.zero_()
calls()
torch.cuda.synchronize()
assert qo.any() and bool(o.flatten(1).any(1).all()) and all(torch.equal(a, b) for f in found for a, b in zip(f, (qo, o, raw)))
print("first use captured")
"""


def test_first_use_in_a_graph():
    """The first calls of a process, captured: they are set up as eager ones are, and give the eager results."""
    done = subprocess.run([sys.executable, "-c", FIRST_USE.format(root=ROOT)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=110)
    assert done.returncode == 0 and "first use captured" in done.stdout, done.stdout[-3000:]


FORMS = [([1, 3, 2], [299, 61, 3000], (4, 2, 64)), ([9, 16], [300, 64], (4, 2, 128)), ([40, 130], [3000, 400], (4, 2, 128)), ([300, 280], [1500, 1200], (2, 2, 96)),
         ([150], [700], (2, 1, 256))]
IDS = ["few", "some", "many", "wide", "large heads"]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_queries_that_are_not_numbers(ctx, form, dtype):  # noqa: F811
    """Queries of NaN and infinity spoil their own rows alone, whatever tile they are in."""
    new, starts, heads = form
    cache, table, q = make(41, heads, new, starts, dtype)
    want, size = wanted(cache, table, q, new, starts)
    bad = torch.zeros(q.shape[:2], dtype=torch.bool)
    bad[::3, 0], bad[1::5, -1] = True, True
    q[::3, 0, 5], q[1::5, -1, 7] = math.nan, math.inf
    got = run(ctx, cache, table, q, new, starts)
    assert bool(torch.isnan(got[bad]).any(-1).all())
    got[bad], want[bad], size[bad] = 0, 0, 0
    check(got, want, size, dtype, weights=weights(heads, new, dtype))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_subnormal_queries(ctx, form, dtype):  # noqa: F811
    """Queries among the type's subnormal numbers, which large keys and a large scale bring back: scores as ever, of the queries as they were rounded."""
    new, starts, heads = form
    down, up = (18, 0) if dtype is F16 else (130, 100)
    cache, table, q = make(45, heads, new, starts, F32)
    q = (q.double() * 2.0 ** -down).to(dtype)
    cache.views()[2].mul_(2.0 ** up)
    scale = 0.125 * 2.0 ** (down - up)
    got = run(ctx, cache, table, q, new, starts, scale=scale)
    check(got, *wanted(cache, table, q, new, starts, scale=scale), dtype, weights=weights(heads, new, dtype))


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_positions_past_the_limit(ctx, form):  # noqa: F811
    """Positions far behind max_length, up to the largest of 32 bits: what lies before it is seen by a row without a window, the first tokens alone with one."""
    new, starts, heads = form
    longest = 190
    cache, table, q = make(42, heads, new, [max(start, longest) for start in starts], BF16)
    far = [(1 << 31) - 1 if b % 2 else 100000 for b in range(len(new))]
    for window, sinks, visible in ((0, 0, 190), (50, 0, 0), (50, 70, 70), (50, 1 << 30, 190)):
        got, first = run(ctx, cache, table, q, new, far, window, sinks, longest=longest), 0
        for b, n in enumerate(new):
            k, v = cache.rows(table[b, :4].tolist(), longest)
            want, size = attend(q[first:first + n].double(), k, v, 0.125, (torch.arange(longest) < visible).expand(n, longest))
            check(got[first:first + n], want, size, BF16, weights=weights(heads, new, BF16))
            first += n


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_shared_pages_and_shared_rows(ctx, dtype):  # noqa: F811
    """Sequences on the same pages (a common prefix), and queries whose heads or tokens are one row (strides of 0)."""
    for new, start, heads in (([2, 2, 2], 700, (4, 2, 64)), ([100, 100], 500, (4, 2, 128))):
        cache, table, q = make(43, heads, new, [start] * len(new), dtype, page=32)
        table[1:] = table[0]
        got = run(ctx, cache, table, q, new, [start] * len(new))
        check(got, *wanted(cache, table, q, new, [start] * len(new)), dtype, weights=weights(heads, new, dtype))
        n, (Hq, H, D), raw = sum(new), heads, cache.raw.cuda()
        c, dev, out = handle(ctx, cache, raw), q.cuda(), torch.zeros(n, Hq, D, dtype=dtype, device="cuda")
        size = ng.ngemm_attention_chunk_workspace_bytes(len(new), Hq, H, D, n, max(new), start + max(new), 0, 0)
        ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
        for strides, rows in (((Hq * D, 0), q[:, :1]), ((0, D), q[:1]), ((0, 0), q[:1, :1])):
            ng.ngemm_attention_chunk(ctx, c, ng.NGEMM_F16 if dtype is F16 else ng.NGEMM_BF16, len(new), Hq, n, dev, *strides, ints(sums(new)), ints([start] * len(new)),
                                     max(new), start + max(new), table.cuda(), table.shape[1], 0, 0, 0.125, out, Hq * D, D, ws, size)
            torch.cuda.synchronize()
            check(out, *wanted(cache, table, rows.expand(n, Hq, D).contiguous(), new, [start] * len(new)), dtype, weights=weights(heads, new, dtype))
        ng.ngemm_kv_cache_free(c)


def test_graphs_that_share_a_workspace(ctx):  # noqa: F811
    """Two captured calls of different sizes with one workspace, replayed in turn with eager work between: the eager bits every time."""
    parts, most = [], 0
    for new, starts, heads in FORMS[:4]:
        cache, table, q = make(44, heads, new, starts, BF16)
        raw, dev, (Hq, H, D), longest = cache.raw.cuda(), q.cuda(), heads, max(a + b for a, b in zip(new, starts))
        size = ng.ngemm_attention_chunk_workspace_bytes(len(new), Hq, H, D, sum(new), max(new), longest, 0, 0)
        most = max(most, size)
        parts.append((new, raw, handle(ctx, cache, raw), dev, torch.zeros_like(dev), ints(sums(new)), ints(starts), table.cuda(), heads, longest, size,
                      run(ctx, cache, table, q, new, starts), torch.cuda.CUDAGraph()))
    ws = torch.empty(most, dtype=torch.uint8, device="cuda")

    def call(new, _raw, c, q, o, off, start, table, heads, longest, size, _want, _graph):
        Hq, H, D = heads
        ng.ngemm_attention_chunk(ctx, c, ng.NGEMM_BF16, len(new), Hq, sum(new), q, Hq * D, D, off, start, max(new), longest, table, table.shape[1], 0, 0, 0.125,
                                 o, Hq * D, D, ws, size)
    torch.cuda.synchronize()
    for p in parts:
        with torch.cuda.graph(p[-1]):
            call(*p)
    for i in (0, 1, 2, 3, 2, 0, 3, 1):
        p = parts[i]
        p[4].zero_()
        ws.fill_(0xff)
        p[-1].replay()
        torch.cuda.synchronize()
        assert torch.equal(p[4].cpu(), p[-2])
        call(*parts[i - 1])
        torch.randn(1000, device="cuda").sum().item()
        assert torch.equal(parts[i - 1][4].cpu(), parts[i - 1][-2])
    for p in parts:
        ng.ngemm_kv_cache_free(p[2])


@pytest.mark.parametrize("pairs", [HALVES, NEIGHBOURS])
@pytest.mark.parametrize("D", range(16, 257, 16))
def test_every_rotated_part(ctx, D, pairs):  # noqa: F811
    """Rows of every size, every multiple of 16 of their elements turned: rows to rows, one head an item and four, and into the cache."""
    for rotated in range(16, D + 1, 16):
        for dtype, n in ((F32, 5), (BF16, 3), (F16, 700 if rotated % 48 == 0 else 4)):
            g = gen(D + rotated)
            q, k = (torch.randn(n, h, D, generator=g).to(dtype) for h in ((30, 7) if n > 99 else (3, 1)))
            rotation = Rotation(ctx, 64, rotated, pairs)
            check_turn(ctx, q, k, 1 + torch.randn(D, generator=g) / 4, 1 + torch.randn(D, generator=g) / 4, 1e-6, rotation, torch.arange(n) % 64)
            rotation.close()
        check_write(ctx, (16, 2, D, rotated, [19, 1], [3, 40]), BF16, pairs, True, "packed")
