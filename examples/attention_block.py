"""Serving the attention of a transformer block with the library: 8-bit projections, an 8-bit cache in pages, prompts and single tokens.

    python examples/attention_block.py

Sequences arrive as packed prompts (some in two pieces, the second behind what the first left in the cache) and are continued token by
token.  K and V enter the cache with ngemm_kv_write; a prompt reads its whole context back with ngemm_kv_read, so that it sees the
same quantised rows as the tokens after it, and attends to it with ngemm_attention_prompt; a token attends to the pages with
ngemm_attention_decode.  The projections are integer products of u8 activations and packed s8 weights (ngemm_run_u8s8s32).
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1910_00178_amd as ng  # noqa: E402


class Linear:
    """y = x W^T with W as s8 codes times a scale per row and x as u8 codes of one scale and zero-point."""

    def __init__(self, ctx, weight):
        self.ctx, (self.n, self.k) = ctx, weight.shape
        self.scale = weight.abs().amax(1) / 127
        codes = torch.round(weight / self.scale.unsqueeze(1)).to(torch.int8)
        size = ng.ngemm_packed_b_bytes(self.k, self.n)
        self.packed = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.handle = ng.ngemm_pack_b(ctx, self.k, self.n, codes, self.k, self.packed, size)
        torch.cuda.current_stream().synchronize()      # the codes may go once they are packed

    def __call__(self, x):
        step = x.abs().amax().float() / 127
        codes = torch.round(x.float() / step + 128).to(torch.uint8)
        m = codes.shape[0]
        size = ng.ngemm_workspace_bytes(m, self.n, self.k)
        workspace = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        sums = torch.empty(m, self.n, dtype=torch.int32, device="cuda")
        ng.ngemm_run_u8s8s32(self.ctx, m, codes, self.k, 128, self.handle, 0, sums, self.n, workspace, size)
        return (sums * (step * self.scale)).to(x.dtype)


class AttentionBlock:
    def __init__(self, width=768, q_heads=12, kv_heads=4, sequences=8, pages=64, page_tokens=32, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.Hq, self.H, self.D, self.dtype = q_heads, kv_heads, width // q_heads, dtype
        self.type = {torch.bfloat16: ng.NGEMM_BF16, torch.float16: ng.NGEMM_F16}[dtype]
        self.ctx = ng.ngemm_create(torch.cuda.current_device())
        weight = lambda n, k: torch.randn(n, k, device="cuda", generator=g) / math.sqrt(k)  # noqa: E731
        self.qkv, self.out = Linear(self.ctx, weight((q_heads + 2 * kv_heads) * self.D, width)), Linear(self.ctx, weight(width, width))
        size = ng.ngemm_kv_cache_bytes(pages, page_tokens, kv_heads, self.D)
        self.buffer = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.cache = ng.ngemm_kv_cache_create(self.ctx, pages, page_tokens, kv_heads, self.D, self.buffer, size)
        self.page_tokens, self.free = page_tokens, list(range(pages))
        self.table = torch.full((sequences, pages), -1, dtype=torch.int32)           # pages of each sequence, in order
        self.length = [0] * sequences

    def close(self):
        for linear in (self.qkv, self.out):
            ng.ngemm_packed_b_free(linear.handle)
        ng.ngemm_kv_cache_free(self.cache)
        ng.ngemm_destroy(self.ctx)

    def _split(self, x):
        """The projections' output as rows of Q, K and V: views with the token stride of all of them together."""
        y = self.qkv(x).view(x.shape[0], self.Hq + 2 * self.H, self.D)
        return y[:, :self.Hq], y[:, self.Hq:self.Hq + self.H], y[:, self.Hq + self.H:]

    def _grow(self, which, new):
        """Room for `new` more tokens of each of the sequences `which`: their lengths before, and their rows of the page table."""
        before = [self.length[s] for s in which]
        for s, n in zip(which, new):
            have, need = (-(-length // self.page_tokens) for length in (self.length[s], self.length[s] + n))
            for page in range(have, need):
                self.table[s, page] = self.free.pop()
            self.length[s] += n
        return before, self.table[list(which)].cuda()

    def _write(self, k, v, offsets, starts, pages):
        ng.ngemm_kv_write(self.ctx, self.cache, self.type, len(starts), k.shape[0], k, k.stride(0), k.stride(1), v, v.stride(0), v.stride(1),
                          offsets, starts, pages, pages.shape[1])

    def prompt(self, which, x, new):
        """x [sum of new][width]: packed rows of the sequences `which`, behind what they already have."""
        before, pages = self._grow(which, new)
        whole = [b + n for b, n in zip(before, new)]
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        sums = lambda v: ints([sum(v[:i]) for i in range(len(v) + 1)])  # noqa: E731
        q, k, v = self._split(x)
        offsets, context = sums(new), sums(whole)
        self._write(k, v, offsets, ints(before), pages)
        m = sum(whole)
        k, v = (torch.empty(m, self.H, self.D, dtype=self.dtype, device="cuda") for _ in range(2))
        ng.ngemm_kv_read(self.ctx, self.cache, self.type, len(new), m, k, k.stride(0), self.D, v, v.stride(0), self.D, context, None,
                         pages, pages.shape[1])
        o = torch.empty(x.shape[0], self.Hq, self.D, dtype=self.dtype, device="cuda")
        size = ng.ngemm_attention_prompt_workspace_bytes(len(new), self.Hq, self.H, self.D, x.shape[0], m)
        workspace = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        ng.ngemm_attention_prompt(self.ctx, self.type, len(new), self.Hq, self.H, self.D, x.shape[0], q, q.stride(0), q.stride(1), m, k, k.stride(0), self.D,
                                  v, v.stride(0), self.D, offsets, context, True, 1 / math.sqrt(self.D), o, o.stride(0), self.D, workspace, size)
        return self.out(o.view(x.shape[0], -1)), o

    def token(self, which, x):
        """x [len(which)][width]: one more token of each of the sequences `which`."""
        before, pages = self._grow(which, [1] * len(which))
        starts = torch.tensor(before, dtype=torch.int32, device="cuda")
        q, k, v = self._split(x)
        self._write(k, v, torch.arange(len(which) + 1, dtype=torch.int32, device="cuda"), starts, pages)
        o = torch.empty(len(which), self.Hq, self.D, dtype=self.dtype, device="cuda")
        longest = max(before) + 1
        size = ng.ngemm_attention_decode_workspace_bytes(len(which), self.Hq, self.H, self.D, longest)
        workspace = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        ng.ngemm_attention_decode(self.ctx, self.cache, self.type, len(which), self.Hq, q, q.stride(0), q.stride(1), starts + 1, longest, pages,
                                  pages.shape[1], 1 / math.sqrt(self.D), o, o.stride(0), self.D, workspace, size)
        return self.out(o.view(len(which), -1)), o


def attend(q, k, v, scale):
    """One token's attention in 64 bits: q [Hq][D], k and v [n][H][D]."""
    group = q.shape[0] // k.shape[1]
    k, v = k.double().repeat_interleave(group, 1), v.double().repeat_interleave(group, 1)
    p = torch.softmax((q.double().unsqueeze(0) * k).sum(-1) * scale, 0)
    return (p.unsqueeze(-1) * v).sum(0)


def main():
    """Two prompts, one of them in two pieces, three tokens more; what the last tokens attend to is checked against the rows that the cache holds."""
    block = AttentionBlock()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = lambda n: torch.randn(n, 768, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    block.prompt([0, 3], x(70 + 45), [70, 45])
    block.prompt([3], x(20), [20])
    worst = 0.0
    for _ in range(3):
        step = x(2)
        y, o = block.token([0, 3], step)
        assert y.shape == (2, 768) and bool(torch.isfinite(y).all())
        q, _, _ = block._split(step)
        for i, s in enumerate((0, 3)):
            n = block.length[s]
            k, v = (torch.empty(n, block.H, block.D, dtype=torch.float32, device="cuda") for _ in range(2))
            ng.ngemm_kv_read(block.ctx, block.cache, ng.NGEMM_F32, 1, n, k, k.stride(0), block.D, v, v.stride(0), block.D,
                             torch.tensor([0, n], dtype=torch.int32, device="cuda"), None, block.table[s:s + 1].cuda(), block.table.shape[1])
            want = attend(q[i], k, v, 1 / math.sqrt(block.D))
            worst = max(worst, float((o[i].double() - want).norm() / want.norm()))
    print(f"lengths {block.length[0]} and {block.length[3]}; outputs differ from 64 bits by {worst:.2g} of their norm")
    assert block.length[0] == 73 and block.length[3] == 68 and worst < 2.0 ** -8          # a bf16 rounding
    block.close()
    return worst


if __name__ == "__main__":
    main()
