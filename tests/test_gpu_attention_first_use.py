"""What a program pays that never uses attention, and the first use of it."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1910_00178_amd", "csrc")

FIRST_USE = """
import sys
sys.path.insert(0, {root!r})
import torch
import paper_1910_00178_amd as ng
ctx = ng.ngemm_create(0)
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
g = torch.Generator().manual_seed(1)
rows = lambda n, h, d: torch.randn(n, h, d, generator=g).to(torch.bfloat16).cuda()
n, Hq, H, D, B, L = 70, 4, 2, 256, 32, 600
q, k, v, o, off = rows(n, Hq, D), rows(n, H, D), rows(n, H, D), torch.zeros(n, Hq, D, dtype=torch.bfloat16, device="cuda"), ints([0, n])
d, hq, hk = 128, 64, 4                                     # whole sequences, all 16 rows of the matrix instructions: more than 64 KiB of LDS
per = (L + 63) // 64
size = ng.ngemm_kv_cache_bytes(B * per, 64, hk, d)
raw = torch.zeros(size, dtype=torch.uint8, device="cuda")
c = ng.ngemm_kv_cache_create(ctx, B * per, 64, hk, d, raw, size)
pages, lens, offs = ints(list(range(B * per))).view(B, per), ints([L] * B), ints([L * b for b in range(B + 1)])
kk, vv, dq, do = rows(B * L, hk, d), rows(B * L, hk, d), rows(B, hq, d), torch.zeros(B, hq, d, dtype=torch.bfloat16, device="cuda")
assert ng.ngemm_attention_prompt_workspace_bytes(1, Hq, H, D, n, n) == 0 and ng.ngemm_attention_decode_workspace_bytes(B, hq, hk, d, L) == 0
def calls():
    ng.ngemm_attention_prompt(ctx, ng.NGEMM_BF16, 1, Hq, H, D, n, q, Hq * D, D, n, k, H * D, D, v, H * D, D, off, None, 1, 0.1, o, Hq * D, D)
    ng.ngemm_kv_write(ctx, c, ng.NGEMM_BF16, B, B * L, kk, hk * d, d, vv, hk * d, d, offs, None, pages, per)
    ng.ngemm_attention_decode(ctx, c, ng.NGEMM_BF16, B, hq, dq, hq * d, d, lens, L, pages, per, 0.1, do, hq * d, d)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
seen = []
for _ in range(3):
    for x in (o, do, raw):
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    seen.append((o.clone(), do.clone()))
for x in (o, do, raw):
    x.zero_()
calls()
torch.cuda.synchronize()
assert o.any() and do.any() and all(torch.equal(a, o) and torch.equal(b, do) for a, b in seen)
print("first use captured")
"""


def test_products_know_nothing_of_attention():
    """A context is made without the attention kernels: their code is loaded, and their LDS asked for, when they are first used."""
    for name in ("ngemm.hip", "ngemm_host.h", "ngemm_kernels.h", "ngemm_mid.h"):
        assert "attention" not in open(os.path.join(CSRC, name)).read(), name


@pytest.mark.gpu
def test_first_use_in_a_graph():
    """The first calls of a process, captured: they are set up as eager ones are, and give the eager results."""
    run = subprocess.run([sys.executable, "-c", FIRST_USE.format(root=ROOT)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=110)
    assert run.returncode == 0 and "first use captured" in run.stdout, run.stdout[-3000:]
