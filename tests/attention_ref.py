"""Plain 64-bit implementation of the cache and of attention (torch on the CPU), and the bounds that outputs are held to."""
import math

import torch

# unit roundoffs
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def quantise(x):
    """Codes (int8) and scales (float32) of rows [..., D], from the definition in 64 bits."""
    y = x.double()
    most = y.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(most) & ~torch.isnan(y).any(-1, keepdim=True)
    codes = torch.where(fine & (most > 0), torch.round(127 * y / torch.where(most > 0, most, 1)), 0)
    codes = torch.where(fine, codes, 0).to(torch.int8)
    return codes, torch.where(fine, most.float() / 127, math.nan)[..., 0].float()


class Cache:
    """A cache buffer on the host in the documented layout."""

    def __init__(self, num_pages, page_tokens, heads, D, fill=0):
        self.shape = (num_pages, page_tokens, heads, D)
        self.raw = torch.full((num_pages, heads, page_tokens // 16, 32 * D + 128), fill, dtype=torch.int8)

    def views(self):
        D = self.shape[3]
        k = self.raw[..., :16 * D].unflatten(-1, (16, D))
        v = self.raw[..., 16 * D:32 * D].unflatten(-1, (D, 16)).transpose(-1, -2)
        s = self.raw[..., 32 * D:].view(torch.float32)
        return k, v, s[..., :16], s[..., 16:]

    def place(self, page, at):
        """index of position `at` of a page: [page, :, block, token]"""
        return page, slice(None), at // 16, at % 16

    def write(self, k, v, offsets, starts, pages):
        views = self.views()
        P, T = self.shape[:2]
        for b in range(len(offsets) - 1):
            for i in range(offsets[b], offsets[b + 1]):
                at = (starts[b] if starts is not None else 0) + i - offsets[b]
                if at < 0 or at // T >= pages.shape[1] or not 0 <= int(pages[b, at // T]) < P:
                    continue
                where = self.place(int(pages[b, at // T]), at % T)
                for x, codes, scales in ((k, views[0], views[2]), (v, views[1], views[3])):
                    codes[where], scales[where] = quantise(x[i])

    def rows(self, page_list, length):
        """K and V of the first `length` positions in 64 bits: [length][head][D]."""
        k, v, ks, vs = (x[list(page_list)] for x in self.views())
        out = []
        for codes, scales in ((k, ks), (v, vs)):
            x = codes.double() * scales.double().unsqueeze(-1)                 # [page][head][block][16][D]
            out.append(x.permute(0, 2, 3, 1, 4).reshape(-1, self.shape[2], self.shape[3])[:length])
        return out


def attend(q, k, v, scale, visible=None):
    """q [n][Hq][D], k and v [m][Hkv][D] in 64 bits, visible [n][m] -> outputs [n][Hq][D] and sum p |v| / sum p, which rounding
    errors of the weights are relative to.  Rows that see nothing give 0; what is not visible is not touched."""
    n, Hq, D = q.shape
    m, Hkv = k.shape[:2]
    out, size = torch.zeros(n, Hq, D, dtype=torch.float64), torch.zeros(n, Hq, D, dtype=torch.float64)
    if visible is None:
        visible = torch.ones(n, m, dtype=torch.bool)
    rows = visible.any(1)
    if not bool(rows.any()):
        return out, size
    for h in range(Hq):
        kh, vh = k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]
        s = (q[:, h] @ kh.t()) * scale if bool(torch.isfinite(kh).all()) else (q[:, h, None, :] * kh[None]).sum(-1) * scale
        p = torch.softmax(s.masked_fill(~visible, -math.inf)[rows], -1)
        if bool(torch.isfinite(vh).all()):
            out[rows, h], size[rows, h] = p @ vh, p @ vh.abs()
        else:
            x = torch.where(visible[rows].unsqueeze(-1), p.unsqueeze(-1) * vh[None], 0.0)
            out[rows, h], size[rows, h] = x.sum(1), x.abs().sum(1)
    return out, size


def check(got, want, size, dtype, weights=None):
    """|got - want| <= u |want| (the output's rounding) + (w + 2^-13) sum p |v| / sum p: w the roundoff of the type that the weights
    enter the second product in; 2^-13 for scores, exponentials and sums in float (scores up to a few hundreds are off by at
    most their sum of |q k| times 2^-22).  The smallest outputs lie on float16's grid of subnormal numbers."""
    w = U[dtype if weights is None else weights]
    got = got.double().cpu()
    bad = torch.isnan(want) | torch.isinf(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    bound = U[dtype] * want.abs() + (w + 2.0 ** -13) * size + 2.0 ** -24
    off = ((got - want).abs() - bound)[~bad]
    assert off.numel() == 0 or float(off.max()) <= 0, f"{float(off.max())} past the bound at {off.argmax().item()} of {off.numel()}"
