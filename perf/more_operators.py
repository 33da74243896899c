"""What a block does between its projections and its attention, and attention of new tokens over the cache's pages, through the
library's public entry points: what is timed when its speed is measured, and the operators' plain forms, which its outputs are compared with.

`listed()` holds the cases, `draw(rng)` more of the same ranges.  Kinds of use:
  rotate   rows of Q and K of new tokens are normalised per head and rotated by their positions, in one pass
  append   K (normalised and rotated on the way) and V of new tokens are quantised into the pages of the cache, and the values that the
           codes stand for are read back
  chunk    new tokens of each sequence, from one to a whole prompt, attend to their sequence in the cache, up to themselves
  window   the same where a token sees the last `window` tokens and the first `sinks` only

The cache is the one of perf/operators.py: pages of `page` tokens, a multiple of 16, for every K/V head; 16 tokens of a head are a block of
32 D + 128 bytes: K codes [16][D], V codes [D][16], K scales [16], V scales [16] (codes int8, scales float32; a token's row is code * scale).
The rotation's table: float32 [positions][rotated], the cosines and behind them the sines of its rotated / 2 pairs.

With `own` false, run() computes in elementary torch operations in 32 bits; with `own` true it makes the calls a user makes.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# (query heads, K/V heads, head size): 768 and 1024 wide blocks, a 4096 wide one with grouped heads, one K/V head for
# all, other group and head sizes
HEADS = ((12, 12, 64), (16, 16, 64), (32, 8, 128), (32, 32, 128), (16, 1, 128), (40, 8, 96), (10, 2, 80), (16, 4, 256), (64, 8, 64))
EPS = 1e-6


def _case(name, use, type, heads, batch, lo, hi, past=0, page=64, norm=True, rotated=0, neighbours=False, window=0, sinks=0, mix=1):
    """lo .. hi: new tokens of a sequence; past: the most tokens that a sequence already has; mix: which lengths of these ranges.
    rotate and append: norm, rotated (elements of a head; 0: all) and neighbours (which elements are a pair).  window, sinks: of window."""
    return {"name": name, "use": use, "type": type, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2],
            "batch": batch, "lo": lo, "hi": hi, "past": past, "page": page, "norm": norm, "rotated": rotated or heads[2],
            "neighbours": neighbours, "window": window, "sinks": sinks, "mix": mix}


def listed():
    return [
        # a step of generation: a token of each of 64 sequences (the smallest call)
        _case("rotate_step_64", "rotate", "bf16", (32, 8, 128), 64, 1, 1, past=4000),
        # packed prompts of ragged lengths
        _case("rotate_prompts_16x2000", "rotate", "bf16", (32, 8, 128), 16, 37, 2000, past=1000),
        # half of each head is rotated, neighbouring elements, without a norm
        _case("rotate_4097_half", "rotate", "f16", (40, 8, 96), 1, 4097, 4097, norm=False, rotated=48, neighbours=True),
        # a step of generation enters the cache
        _case("append_step_64", "append", "bf16", (32, 8, 128), 64, 1, 1, past=4000),
        # prompts of ragged lengths enter the cache, some behind a prefix that ends inside a block
        _case("append_prompts_16x4000", "append", "bf16", (32, 8, 128), 16, 37, 4000, past=1000, page=16),
        # four proposed tokens of each of 32 sequences are checked at once
        _case("chunk_verify_32x4", "chunk", "bf16", (32, 8, 128), 32, 4, 4, past=4000),
        # a step that generates for some sequences and takes in a piece of the prompts of others
        _case("chunk_mixed_16x600", "chunk", "f16", (12, 12, 64), 16, 1, 600, past=3000, page=16),
        # a piece of one long prompt behind what is already in the cache
        _case("chunk_512_behind_16000", "chunk", "bf16", (32, 8, 128), 1, 512, 512, past=16000, page=128, mix=3),
        # a whole prompt straight on the pages: the largest
        _case("chunk_1x8192", "chunk", "bf16", (32, 8, 128), 1, 8192, 8192),
        # a step of generation for 64 sequences, behind texts much longer than the window
        _case("window_step_64x16000", "window", "bf16", (32, 8, 128), 64, 1, 1, past=16000, window=1024, sinks=4),
        # proposed tokens of large heads, a window that few of the texts fill
        _case("window_verify_16x5", "window", "f16", (16, 4, 256), 16, 1, 5, past=9000, window=4096, sinks=16, page=48),
        # prompts of ragged lengths, most of them longer than the window
        _case("window_prompts_4x5000", "window", "bf16", (32, 8, 128), 4, 500, 5000, past=700, window=1000, sinks=4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    use = rng.choice(("rotate", "append", "chunk", "chunk", "window", "window"))
    heads, type = rng.choice(HEADS), rng.choice(("bf16", "f16"))
    row = heads[1] * heads[2]
    more = {"page": rng.choice((16, 32, 48, 64, 128)), "mix": rng.randint(1, 9999)}
    if use in ("rotate", "append"):
        batch = _log(rng, 1, 64)
        hi = rng.choice((1, _log(rng, 2, max(2, 16384 * 1024 // row // batch))))
        more |= {"past": rng.choice((0, _log(rng, 10, 4000))), "norm": rng.random() < 0.7, "neighbours": rng.random() < 0.3,
                 "rotated": rng.choice((0, 0, rng.randint(1, heads[2] // 16) * 16))}
    else:
        batch = _log(rng, 1, 64)
        most = 7500 * 7500 * 32 * 128 // (batch * heads[0] * heads[2])                  # new tokens times context
        hi = rng.choice((1, _log(rng, 1, 16), _log(rng, 2, max(2, min(8192, math.isqrt(most))))))
        hi = max(1, min(hi, math.isqrt(most)))
        more |= {"past": rng.choice((0, _log(rng, 16, max(16, min(32768, (most - hi * hi // 2) // hi // 2, 900000 * 1024 // row // batch)))))}
        if use == "window":
            more |= {"window": _log(rng, 16, 8192), "sinks": rng.choice((0, 1, 4, rng.randint(2, 100)))}
    lo = rng.choice((hi, max(1, hi // 3), max(1, hi // 40)))
    case = _case("", use, type, heads, batch, lo, hi, **more)
    del case["name"]
    return case


def _lengths(case):
    """New tokens and tokens already there, of each sequence."""
    r, n, past = random.Random(case["mix"]), [], []
    for b in range(case["batch"]):
        n.append(case["hi"] if b == 0 else _log(r, case["lo"], case["hi"]))
        past.append(r.randint(case["past"] // 3, case["past"]))
    return n, past


def work(case):
    n, past = _lengths(case)
    tokens, Hq, Hkv, D = sum(n), case["q_heads"], case["kv_heads"], case["head_dim"]
    codes, rows = 2 * D + 8, 4 * D                 # K and V of a token and head: in the cache, and as 16-bit rows
    table = 4 * case["rotated"] * len(set().union(*(range(p, p + l) for l, p in zip(n, past)))) if case["use"] in ("rotate", "append") else 0
    if case["use"] == "rotate":
        return {"bytes": tokens * (Hq + Hkv) * rows + table + 4 * tokens, "flops": 8 * tokens * (Hq + Hkv) * D}
    if case["use"] == "append":
        return {"bytes": tokens * Hkv * (rows + codes + rows) + table, "flops": 12 * tokens * Hkv * D}
    pairs = context = 0
    for l, p in zip(n, past):
        sees = np.arange(p + 1, p + l + 1)         # tokens up to and with each row's
        if case["window"]:
            context += min(p + l, min(case["sinks"], max(0, p + 1 - case["window"])) + l + min(p, case["window"] - 1))
            pairs += int((np.minimum(sees, case["window"]) + np.minimum(case["sinks"], np.maximum(0, sees - case["window"]))).sum())
        else:
            context += p + l
            pairs += int(sees.sum())
    return {"bytes": context * Hkv * codes + tokens * Hq * D * 4, "flops": 4 * pairs * Hq * D}


# ---- the cache's layout ----

def _views(cache, D):
    """cache [page][head][block][32 D + 128] -> K codes [..][16][D], V codes [..][16][D] (a view of [D][16]), K and V scales [..][16]."""
    k = cache[..., :16 * D].unflatten(-1, (16, D))
    v = cache[..., 16 * D:32 * D].unflatten(-1, (D, 16)).transpose(-1, -2)
    s = cache[..., 32 * D:].view(torch.float32)
    return k, v, s[..., :16], s[..., 16:]


def _places(state, seq, at):
    """Page, block in the page and token in the block of the tokens at positions `at` of the sequences `seq`."""
    page = state["case"]["page"]
    return state["pages"][seq, at // page].long(), at % page // 16, at % 16


def _put(x, codes, scales, page, block, token):
    """Rows x [n][head][D] of f32 are quantised and written."""
    most = x.abs().amax(-1, keepdim=True)
    q = torch.where(most > 0, torch.round(x * 127 / most), torch.zeros_like(x))
    codes[page, :, block, token] = q.to(torch.int8)
    scales[page, :, block, token] = (most / 127)[..., 0]


def _get(codes, scales, page, block, token):
    """Rows of f32: [..][head][D] for indexes of any shape."""
    return codes[page, :, block, token].float() * scales[page, :, block, token].unsqueeze(-1)


# ---- inputs ----

_context = None


def _rows(g, n, heads, D, outliers=False):
    """Rows as projections give them: normal, for keys with some channels much larger than the others."""
    x = torch.randn(n, heads, D, device="cuda", generator=g)
    if outliers:
        x *= 1 + 3 * (torch.rand(1, heads, D, device="cuda", generator=g) > 0.95)
    return x


def _table(positions, rotated):
    pair = torch.arange(rotated // 2, device="cuda", dtype=torch.float64)
    angle = torch.arange(positions, device="cuda", dtype=torch.float64).unsqueeze(1) * 10000.0 ** (-2 * pair / rotated)
    return torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()


def prepare(case, seed):
    global _context
    g = torch.Generator(device="cuda").manual_seed(seed)
    type, Hq, Hkv, D, batch, page = TYPES[case["type"]], case["q_heads"], case["kv_heads"], case["head_dim"], case["batch"], case["page"]
    n, past = _lengths(case)
    whole = [a + b for a, b in zip(n, past)]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": case, "type": type, "tokens": sum(n), "max_length": max(whole), "max_new": max(n), "new": ints(n), "starts": ints(past),
         "offsets": ints([sum(n[:b]) for b in range(batch + 1)]), "scale": 1 / math.sqrt(D)}
    if case["use"] in ("rotate", "append"):
        s["table"] = _table(max(whole), case["rotated"])
        weights = lambda: 1 + 0.2 * torch.randn(D, device="cuda", generator=g) if case["norm"] else None  # noqa: E731
        s["q_weight"], s["k_weight"] = weights(), weights()
        s["k"], s["v"] = _rows(g, s["tokens"], Hkv, D, True).to(type), _rows(g, s["tokens"], Hkv, D).to(type)
    if case["use"] != "append":
        s["q"] = _rows(g, s["tokens"], Hq, D).to(type)
    if case["use"] == "rotate":
        s["positions"] = torch.cat([torch.arange(p, p + l, dtype=torch.int32, device="cuda") for l, p in zip(n, past)])
    else:
        per = -(-max(whole) // page)
        pool = batch * per + 3
        s["pages"] = torch.randperm(pool, device="cuda", generator=g)[:batch * per].to(torch.int32).view(batch, per).contiguous()
        s["cache"] = torch.zeros(pool, Hkv, page // 16, 32 * D + 128, dtype=torch.int8, device="cuda")
        if case["use"] != "append":
            kc, vc, ks, vs = _views(s["cache"], D)
            for codes, scales, out in ((kc, ks, True), (vc, vs, False)):
                for p in range(0, pool, 64):          # 64 pages at a time: what the rows take in f32
                    m = min(64, pool - p)
                    x = _rows(g, m * page, Hkv, D, out).view(m, page // 16, 16, Hkv, D).permute(0, 3, 1, 2, 4)
                    most = x.abs().amax(-1)
                    codes[p:p + m], scales[p:p + m] = torch.round(x * 127 / most.unsqueeze(-1)).to(torch.int8), most / 127
    if own:                                           # what a program keeps: the library's handles, outputs, a workspace
        import paper_1910_00178_amd as ng
        s["ng"], s["number"] = ng, {"bf16": ng.NGEMM_BF16, "f16": ng.NGEMM_F16}[case["type"]]
        if _context is None:
            _context = ng.ngemm_create(0)
        s["ctx"] = _context
        if "table" in s:
            pairs = ng.NGEMM_PAIRS_NEIGHBOURS if case["neighbours"] else ng.NGEMM_PAIRS_HALVES
            s["rotation"] = ng.ngemm_rotation_create(s["ctx"], max(whole), case["rotated"], pairs, s["table"], s["table"].numel() * 4)
        if "cache" in s:
            s["handle"] = ng.ngemm_kv_cache_create(s["ctx"], s["cache"].shape[0], page, Hkv, D, s["cache"], s["cache"].numel())
        if case["use"] == "rotate":
            s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        elif case["use"] == "append":
            s["k_out"], s["v_out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        else:
            s["out"] = torch.empty_like(s["q"])
            s["bytes"] = ng.ngemm_attention_chunk_workspace_bytes(batch, Hq, Hkv, D, s["tokens"], s["max_new"], s["max_length"], case["window"],
                                                                  case["sinks"])
            s["workspace"] = torch.empty(max(16, s["bytes"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ----

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["use"]](state)


def _own_rotate(s):
    c = s["case"]
    Hq, Hkv, D = c["q_heads"], c["kv_heads"], c["head_dim"]
    s["ng"].ngemm_qk_norm_rotate(s["ctx"], s["number"], D, s["tokens"], Hq, s["q"], Hq * D, D, s["q_weight"], Hkv, s["k"], Hkv * D, D, s["k_weight"],
                                 EPS, s["rotation"], s["positions"], s["q_out"], Hq * D, D, s["k_out"], Hkv * D, D)
    return s["q_out"], s["k_out"]


def _own_append(s):
    c = s["case"]
    Hkv, D = c["kv_heads"], c["head_dim"]
    s["ng"].ngemm_kv_write_rotated(s["ctx"], s["handle"], s["number"], c["batch"], s["tokens"], s["k"], Hkv * D, D, s["v"], Hkv * D, D,
                                   s["k_weight"], EPS, s["rotation"], s["offsets"], s["starts"], s["pages"], s["pages"].shape[1])
    s["ng"].ngemm_kv_read(s["ctx"], s["handle"], s["number"], c["batch"], s["tokens"], s["k_out"], Hkv * D, D, s["v_out"], Hkv * D, D,
                          s["offsets"], s["starts"], s["pages"], s["pages"].shape[1])
    return s["k_out"], s["v_out"]


def _own_chunk(s):
    c = s["case"]
    Hq, D = c["q_heads"], c["head_dim"]
    s["ng"].ngemm_attention_chunk(s["ctx"], s["handle"], s["number"], c["batch"], Hq, s["tokens"], s["q"], Hq * D, D, s["offsets"], s["starts"],
                                  s["max_new"], s["max_length"], s["pages"], s["pages"].shape[1], c["window"], c["sinks"], s["scale"],
                                  s["out"], Hq * D, D, s["workspace"], s["bytes"])
    return s["out"]


def _new_tokens(s):
    """Sequence and position of every packed new token."""
    i = torch.arange(s["tokens"], device="cuda")
    seq = torch.bucketize(i, s["offsets"][1:], right=True)
    return seq, i - s["offsets"][seq] + s["starts"][seq]


def _turned(x, weight, table, case):
    """Rows x [n][head][D] of f32 normalised, then rotated by the table's rows [n][rotated]."""
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight
    r = case["rotated"]
    cos, sin = table[:, None, :r // 2], table[:, None, r // 2:]
    if case["neighbours"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), x[..., r:]), -1)
    a, b = x[..., :r // 2], x[..., r // 2:r]
    return torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., r:]), -1)


def _plain_rotate(s):
    at = s["table"][s["positions"]]
    return (_turned(s["q"].float(), s["q_weight"], at, s["case"]).to(s["type"]), _turned(s["k"].float(), s["k_weight"], at, s["case"]).to(s["type"]))


def _plain_append(s):
    kc, vc, ks, vs = _views(s["cache"], s["case"]["head_dim"])
    seq, at = _new_tokens(s)
    place = _places(s, seq, at)
    _put(_turned(s["k"].float(), s["k_weight"], s["table"][at], s["case"]), kc, ks, *place)
    _put(s["v"].float(), vc, vs, *place)
    return _get(kc, ks, *place).to(s["type"]), _get(vc, vs, *place).to(s["type"])


def _plain_chunk(s):
    c = s["case"]
    Hkv, D, batch = c["kv_heads"], c["head_dim"], c["batch"]
    i, j = torch.arange(s["max_new"], device="cuda"), torch.arange(s["max_length"], device="cuda")
    real, length = i < s["new"].unsqueeze(1), s["starts"] + s["new"]
    place = _places(s, torch.arange(batch, device="cuda").unsqueeze(1), torch.where(j < length.unsqueeze(1), j, 0))
    kc, vc, ks, vs = _views(s["cache"], D)
    k, v = _get(kc, ks, *place).transpose(1, 2).unsqueeze(2), _get(vc, vs, *place).transpose(1, 2).unsqueeze(2)      # [b][kv head][1][key][D]
    at = (i + s["starts"].unsqueeze(1)).unsqueeze(-1)                                                               # [b][row][1]
    seen = j <= at
    if c["window"]:
        seen &= (j > at - c["window"]) | (j < c["sinks"])
    q = s["q"].float()[torch.where(real, i + s["offsets"][:-1].unsqueeze(1), 0)]
    q = q.view(batch, s["max_new"], Hkv, -1, D).permute(0, 2, 3, 1, 4)                                               # [b][kv head][head][row][D]
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~seen[:, None, None], -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    return o.permute(0, 3, 1, 2, 4).reshape(batch, s["max_new"], c["q_heads"], D)[real].to(s["type"])


_run_own = {"rotate": _own_rotate, "append": _own_append, "chunk": _own_chunk, "window": _own_chunk}
_run_plain = {"rotate": _plain_rotate, "append": _plain_append, "chunk": _plain_chunk, "window": _plain_chunk}


# ---- the definition in 64 bits ----

def _exact_turned(x, weight, positions, case):
    """Pairs as complex numbers, times exp(i angle); the cosines and sines are the table's, which is an input."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    half = case["rotated"] // 2
    first = torch.arange(half, device="cuda") * (2 if case["neighbours"] else 1)
    second = first + (1 if case["neighbours"] else half)
    table = _table(int(positions.max()) + 1, case["rotated"]).double()[positions.long()]
    z = torch.complex(x[..., first], x[..., second]) * torch.complex(table[:, :half], table[:, half:]).unsqueeze(1)
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, D, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    n, past = _lengths(case)
    if case["use"] in ("rotate", "append"):
        positions = torch.cat([torch.arange(p, p + l, device="cuda") for l, p in zip(n, past)])
        k = _exact_turned(s["k"], s["k_weight"], positions, case)
        if case["use"] == "rotate":
            return _exact_turned(s["q"], s["q_weight"], positions, case), k

        def stored(x):
            most = x.abs().amax(-1, keepdim=True).clamp_min(5e-324)
            return torch.round(127 * x / most) * most / 127
        return stored(k), stored(s["v"].double())
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    first, group = 0, Hq // Hkv
    for b, (l, p) in enumerate(zip(n, past)):
        own_pages = s["cache"][s["pages"][b, :-(-(l + p) // page)].long()]            # [page][head][block][bytes]
        scales = own_pages[..., 32 * D:].contiguous().view(torch.float32).double()
        k = own_pages[..., :16 * D].double().reshape(*own_pages.shape[:3], 16, D) * scales[..., :16, None]
        v = own_pages[..., 16 * D:32 * D].double().reshape(*own_pages.shape[:3], D, 16).transpose(-1, -2) * scales[..., 16:, None]
        k, v = (x.permute(1, 0, 2, 3, 4).reshape(Hkv, -1, D)[:, :l + p] for x in (k, v))
        distance = torch.arange(p, p + l, device="cuda").unsqueeze(1) - torch.arange(l + p, device="cuda")
        hidden = distance < 0
        if case["window"]:
            hidden |= (distance >= case["window"]) & (torch.arange(l + p, device="cuda") >= case["sinks"])
        for h in range(Hq):
            x = s["q"][first:first + l, h].double() @ k[h // group].t() * s["scale"]
            out[first:first + l, h] = torch.softmax(x.masked_fill_(hidden, -math.inf), -1) @ v[h // group]
        first += l
    return out
