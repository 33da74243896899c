"""The attention of a block whose projections are integer products, through the library's public entry points: what is timed
when its speed is measured, and the operators' plain forms, which its outputs are compared with.

`listed()` holds the cases, `draw(rng)` more of the same ranges.  Kinds of use:
  store    K and V of new tokens are quantised into the pages of the cache, and the values that the codes stand for are read back
  read     whole sequences come back from the pages as packed rows (a prompt that continues a cached one needs its prefix so)
  decode   one new token per sequence attends to its sequence in the cache
  prompt   packed sequences attend to themselves, or to a prefix and themselves

The cache: pages of `page` tokens, a multiple of 16, for every K/V head; 16 tokens of a head are a block of 32 D + 128 bytes:
K codes [16][D], V codes [D][16], K scales [16], V scales [16] (codes int8, scales float32; a token's row is code * scale).

With `own` false, run() computes in elementary torch operations in 32 bits; with `own` true it makes the calls a user makes.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# (query heads, K/V heads, head size): 768 and 1024 wide blocks, a 4096 wide one with grouped heads, one K/V head for
# all, other group and head sizes
HEADS = ((12, 12, 64), (16, 16, 64), (32, 8, 128), (32, 32, 128), (16, 1, 128), (40, 8, 96), (10, 2, 80), (16, 4, 256), (64, 8, 64))


def _case(name, use, type, heads, batch, lo, hi, page=64, past=0, causal=True, mix=1):
    """lo .. hi: new tokens of a sequence (store, prompt) or its length in the cache (read, decode); past: the most tokens
    that a sequence already has (store, prompt); mix: which lengths of these ranges."""
    return {"name": name, "use": use, "type": type, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2],
            "batch": batch, "lo": lo, "hi": hi, "page": page, "past": past, "causal": causal, "mix": mix}


def listed():
    return [
        # a step of generation: every one of 64 sequences appends its token (the smallest call)
        _case("store_append_64", "store", "bf16", (32, 8, 128), 64, 1, 1, page=64, past=4000),
        # prompts of ragged lengths enter the cache, some behind a prefix that ends inside a block
        _case("store_prompts_16x4000", "store", "bf16", (32, 8, 128), 16, 37, 4000, page=16, past=1000),
        # prefixes of ragged lengths are read back for prompts that continue them
        _case("read_4x1000", "read", "f16", (12, 12, 64), 4, 100, 1000, page=16),
        _case("read_8x8192", "read", "bf16", (32, 8, 128), 8, 2048, 8192, page=64),
        # generating for one sequence: latency
        _case("decode_1x4097", "decode", "bf16", (32, 8, 128), 1, 4097, 4097, page=64),
        # 32 short sequences, a K/V head for each query head
        _case("decode_32x1000", "decode", "f16", (12, 12, 64), 32, 17, 1000, page=16),
        # 64 sequences of very different lengths
        _case("decode_64x8192", "decode", "bf16", (32, 8, 128), 64, 128, 8192, page=64),
        # few long sequences: the cache is a stream
        _case("decode_8x131072", "decode", "bf16", (32, 8, 128), 8, 100000, 131072, page=128),
        # 1024 tokens of a 768 wide block that looks both ways, as 8 sequences
        _case("prompt_8x128_both_ways", "prompt", "f16", (12, 12, 64), 8, 128, 128, causal=False),
        # packed prompts of ragged lengths behind cached prefixes
        _case("prompt_6x2047_continued", "prompt", "bf16", (32, 8, 128), 6, 50, 2047, past=1500),
        # short questions behind a long cached text: few rows, a long axis
        _case("prompt_2x96_behind_16000", "prompt", "f16", (16, 4, 256), 2, 96, 96, past=16000, mix=3),
        # the longest prompt
        _case("prompt_1x8192", "prompt", "bf16", (32, 8, 128), 1, 8192, 8192),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    use = rng.choice(("store", "read", "decode", "decode", "prompt", "prompt"))
    heads, type = rng.choice(HEADS), rng.choice(("bf16", "f16"))
    row = heads[1] * heads[2]
    more = {"page": rng.choice((16, 32, 48, 64, 128)), "mix": rng.randint(1, 9999)}
    if use == "store":
        batch = _log(rng, 1, 64)
        hi = rng.choice((1, _log(rng, 2, max(2, 16384 * 1024 // row // batch))))
        more |= {"past": rng.choice((0, _log(rng, 10, 4000)))}
    elif use == "read":
        batch = _log(rng, 1, 32)
        hi = _log(rng, 16, max(16, 65536 * 1024 // row // batch))
    elif use == "decode":
        batch = _log(rng, 1, 128)
        hi = _log(rng, 16, max(16, min(131072, 900000 * 1024 // row // batch)))
    else:
        batch = _log(rng, 1, 16)
        causal = rng.random() < 0.75
        most = 7500 * 7500 * 32 * 128 // (batch * heads[0] * heads[2]) // (1 if causal else 2)          # new tokens times context
        hi = _log(rng, 1, min(8192, math.isqrt(most)))
        past = rng.choice((0, 0, _log(rng, 16, max(16, min(16384, (most - hi * hi // 2) // hi // 2, 131072 * 1024 // row // batch)))))
        more |= {"past": past, "causal": causal}
    lo = rng.choice((hi, max(1, hi // 3), max(1, hi // 40)))
    case = _case("", use, type, heads, batch, lo, hi, **more)
    del case["name"]
    return case


def _lengths(case):
    """New tokens (or lengths in the cache) and tokens already there, of each sequence."""
    r, n, past = random.Random(case["mix"]), [], []
    for b in range(case["batch"]):
        n.append(case["hi"] if b == 0 else _log(r, case["lo"], case["hi"]))
        past.append(r.randint(0, case["past"]))
    return n, past


def _counts(case):
    n, past = _lengths(case)
    if case["use"] in ("read", "decode"):
        return sum(n), sum(n), 0
    pairs = sum(l * p + (l * (l + 1) // 2 if case["causal"] else l * l) for l, p in zip(n, past))
    return sum(n), sum(n) + sum(past), pairs


def work(case):
    tokens, context, pairs = _counts(case)
    Hq, Hkv, D, use = case["q_heads"], case["kv_heads"], case["head_dim"], case["use"]
    codes, rows = 2 * D + 8, 4 * D                 # K and V of a token and head: in the cache, and as 16-bit rows
    if use == "store":
        return {"bytes": tokens * Hkv * (rows + codes + rows), "flops": 6 * tokens * Hkv * D}
    if use == "read":
        return {"bytes": tokens * Hkv * (codes + rows), "flops": 2 * tokens * Hkv * D}
    if use == "decode":
        return {"bytes": context * Hkv * codes + case["batch"] * Hq * D * 4, "flops": 4 * context * Hq * D}
    return {"bytes": tokens * Hq * D * 4 + context * Hkv * rows, "flops": 4 * pairs * Hq * D}


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


def prepare(case, seed):
    global _context
    g = torch.Generator(device="cuda").manual_seed(seed)
    type, Hq, Hkv, D, batch, page = TYPES[case["type"]], case["q_heads"], case["kv_heads"], case["head_dim"], case["batch"], case["page"]
    n, past = _lengths(case)
    whole = n if case["use"] in ("read", "decode") else [a + b for a, b in zip(n, past)]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    sums = lambda v: ints([sum(v[:b]) for b in range(len(v) + 1)])  # noqa: E731
    s = {"case": case, "type": type, "tokens": sum(n), "lengths": ints(whole), "max_length": max(whole), "max_new": max(n), "new": ints(n),
         "offsets": sums(n), "scale": 1 / math.sqrt(D)}
    if case["use"] in ("store", "read", "decode"):
        per = -(-max(whole) // page)
        pool = batch * per + 3
        s["pages"] = torch.randperm(pool, device="cuda", generator=g)[:batch * per].to(torch.int32).view(batch, per).contiguous()
        s["starts"] = ints(past if case["use"] == "store" else [0] * batch)
        s["cache"] = torch.zeros(pool, Hkv, page // 16, 32 * D + 128, dtype=torch.int8, device="cuda")
        if case["use"] != "store":
            kc, vc, ks, vs = _views(s["cache"], D)
            for codes, scales, out in ((kc, ks, True), (vc, vs, False)):
                for p in range(0, pool, 64):          # 64 pages at a time: what the rows take in f32
                    m = min(64, pool - p)
                    x = _rows(g, m * page, Hkv, D, out).view(m, page // 16, 16, Hkv, D).permute(0, 3, 1, 2, 4)
                    most = x.abs().amax(-1)
                    codes[p:p + m], scales[p:p + m] = torch.round(x * 127 / most.unsqueeze(-1)).to(torch.int8), most / 127
    if case["use"] == "store":
        s["k"], s["v"] = _rows(g, s["tokens"], Hkv, D, True).to(type), _rows(g, s["tokens"], Hkv, D).to(type)
    if case["use"] == "decode":
        s["q"] = _rows(g, batch, Hq, D).to(type)
    if case["use"] == "prompt":
        s["k_offsets"], s["k_tokens"] = sums(whole), sum(whole)
        sizes = ((s["tokens"], Hq, False), (sum(whole), Hkv, True), (sum(whole), Hkv, False))
        s["q"], s["k"], s["v"] = (_rows(g, m, h, D, o).to(type) for m, h, o in sizes)
    if own:                                           # what a program keeps: the library's handles, outputs, a workspace
        import paper_1910_00178_amd as ng
        s["ng"], s["number"] = ng, {"bf16": ng.NGEMM_BF16, "f16": ng.NGEMM_F16}[case["type"]]
        if _context is None:
            _context = ng.ngemm_create(0)
        s["ctx"] = _context
        if "cache" in s:
            s["handle"] = ng.ngemm_kv_cache_create(s["ctx"], s["cache"].shape[0], page, Hkv, D, s["cache"], s["cache"].numel())
        if case["use"] in ("store", "read"):
            s["k_out"], s["v_out"] = (torch.empty(s["tokens"], Hkv, D, dtype=type, device="cuda") for _ in range(2))
        else:
            s["out"] = torch.empty_like(s["q"])
            s["bytes"] = (ng.ngemm_attention_decode_workspace_bytes(batch, Hq, Hkv, D, s["max_length"]) if case["use"] == "decode" else
                          ng.ngemm_attention_prompt_workspace_bytes(batch, Hq, Hkv, D, s["tokens"], s["k_tokens"]))
            s["workspace"] = torch.empty(max(16, s["bytes"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ----

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["use"]](state)


def _own_read(s):
    Hkv, D = s["case"]["kv_heads"], s["case"]["head_dim"]
    s["ng"].ngemm_kv_read(s["ctx"], s["handle"], s["number"], s["case"]["batch"], s["tokens"], s["k_out"], Hkv * D, D, s["v_out"], Hkv * D, D,
                          s["offsets"], s["starts"], s["pages"], s["pages"].shape[1])
    return s["k_out"], s["v_out"]


def _own_store(s):
    Hkv, D = s["case"]["kv_heads"], s["case"]["head_dim"]
    s["ng"].ngemm_kv_write(s["ctx"], s["handle"], s["number"], s["case"]["batch"], s["tokens"], s["k"], Hkv * D, D, s["v"], Hkv * D, D,
                           s["offsets"], s["starts"], s["pages"], s["pages"].shape[1])
    return _own_read(s)


def _own_decode(s):
    Hq, D = s["case"]["q_heads"], s["case"]["head_dim"]
    s["ng"].ngemm_attention_decode(s["ctx"], s["handle"], s["number"], s["case"]["batch"], Hq, s["q"], Hq * D, D, s["lengths"], s["max_length"],
                                   s["pages"], s["pages"].shape[1], s["scale"], s["out"], Hq * D, D, s["workspace"], s["bytes"])
    return s["out"]


def _own_prompt(s):
    c = s["case"]
    Hq, Hkv, D = c["q_heads"], c["kv_heads"], c["head_dim"]
    s["ng"].ngemm_attention_prompt(s["ctx"], s["number"], c["batch"], Hq, Hkv, D, s["tokens"], s["q"], Hq * D, D, s["k_tokens"], s["k"], Hkv * D, D,
                                   s["v"], Hkv * D, D, s["offsets"], s["k_offsets"], c["causal"], s["scale"], s["out"], Hq * D, D,
                                   s["workspace"], s["bytes"])
    return s["out"]


def _new_tokens(s):
    """Sequence and position of every packed new token."""
    i = torch.arange(s["tokens"], device="cuda")
    seq = torch.bucketize(i, s["offsets"][1:], right=True)
    return seq, i - s["offsets"][seq] + s["starts"][seq]


def _plain_read(s):
    kc, vc, ks, vs = _views(s["cache"], s["case"]["head_dim"])
    place = _places(s, *_new_tokens(s))
    return _get(kc, ks, *place).to(s["type"]), _get(vc, vs, *place).to(s["type"])


def _plain_store(s):
    kc, vc, ks, vs = _views(s["cache"], s["case"]["head_dim"])
    place = _places(s, *_new_tokens(s))
    _put(s["k"].float(), kc, ks, *place)
    _put(s["v"].float(), vc, vs, *place)
    return _get(kc, ks, *place).to(s["type"]), _get(vc, vs, *place).to(s["type"])


def _attend(q, k, v, seen, scale):
    """q [b][kv head][rows][D], k and v [b][kv head][keys][D], seen [b][rows or 1][keys]: rows that see nothing give 0."""
    x = torch.matmul(q, k.transpose(-1, -2)) * scale
    seen = seen.unsqueeze(1)
    x = x.masked_fill(~seen, -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True).clamp_min(-1e30))
    return torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp_min(1e-30)


def _plain_decode(s):
    c = s["case"]
    Hkv, D = c["kv_heads"], c["head_dim"]
    at = torch.arange(s["max_length"], device="cuda")
    seen = at < s["lengths"].unsqueeze(1)
    place = _places(s, torch.arange(c["batch"], device="cuda").unsqueeze(1), torch.where(seen, at, 0))
    kc, vc, ks, vs = _views(s["cache"], D)
    k, v = _get(kc, ks, *place).transpose(1, 2), _get(vc, vs, *place).transpose(1, 2)
    q = s["q"].float().view(c["batch"], Hkv, -1, D)
    return _attend(q, k, v, seen.unsqueeze(1), s["scale"]).reshape(s["q"].shape).to(s["type"])


def _plain_prompt(s):
    c = s["case"]
    Hkv, D, batch = c["kv_heads"], c["head_dim"], c["batch"]
    group = c["q_heads"] // Hkv
    i, j = torch.arange(s["max_new"], device="cuda"), torch.arange(s["max_length"], device="cuda")
    real, there = i < s["new"].unsqueeze(1), j < s["lengths"].unsqueeze(1)
    q = s["q"].float()[torch.where(real, i + s["offsets"][:-1].unsqueeze(1), 0)]
    k, v = (s[n].float()[torch.where(there, j + s["k_offsets"][:-1].unsqueeze(1), 0)].transpose(1, 2) for n in "kv")
    seen = there.unsqueeze(1)
    if c["causal"]:
        seen = seen & (j <= i.unsqueeze(1) + (s["lengths"] - s["new"]).view(-1, 1, 1))
    q = q.view(batch, -1, Hkv, group, D).permute(0, 2, 3, 1, 4)
    o = _attend(q, k.unsqueeze(2), v.unsqueeze(2), seen.unsqueeze(1), s["scale"])
    return o.permute(0, 3, 1, 2, 4).reshape(batch, -1, c["q_heads"], D)[real].to(s["type"])


_run_own = {"store": _own_store, "read": _own_read, "decode": _own_decode, "prompt": _own_prompt}
_run_plain = {"store": _plain_store, "read": _plain_read, "decode": _plain_decode, "prompt": _plain_prompt}


# ---- the definition in 64 bits, a sequence at a time ----

def _softmax_rows(q, k, v, scale, diagonal):
    """q [n][D] against k, v [m][D]; row i sees keys up to i + diagonal (None: all)."""
    x = (q @ k.t()) * scale
    if diagonal is not None:
        x.masked_fill_(torch.ones_like(x, dtype=torch.bool).triu(diagonal + 1), -math.inf)
    return torch.softmax(x, -1) @ v


def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, D, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    n, past = _lengths(case)
    group = Hq // Hkv
    first = [sum(n[:b]) for b in range(len(n))]
    if case["use"] == "store":
        def stored(x):
            x = x.double()
            most = x.abs().amax(-1, keepdim=True).clamp_min(5e-324)
            return torch.round(127 * x / most) * most / 127
        return stored(s["k"]), stored(s["v"])

    def cached(b, length):
        """K and V of a sequence: [length][head][D]."""
        own_pages = s["cache"][s["pages"][b, :-(-length // page)].long()]            # [page][head][block][bytes]
        scales = own_pages[..., 32 * D:].contiguous().view(torch.float32).double()
        k = own_pages[..., :16 * D].double().reshape(*own_pages.shape[:3], 16, D) * scales[..., :16, None]
        v = own_pages[..., 16 * D:32 * D].double().reshape(*own_pages.shape[:3], D, 16).transpose(-1, -2) * scales[..., 16:, None]
        return tuple(x.permute(0, 2, 3, 1, 4).reshape(-1, Hkv, D)[:length] for x in (k, v))

    if case["use"] == "read":
        rows = [cached(b, l) for b, l in enumerate(n)]
        return torch.cat([r[0] for r in rows]), torch.cat([r[1] for r in rows])
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    if case["use"] == "decode":
        for b, l in enumerate(n):
            k, v = cached(b, l)
            for h in range(Hkv):
                g = slice(h * group, (h + 1) * group)
                out[b, g] = _softmax_rows(s["q"][b, g].double(), k[:, h], v[:, h], s["scale"], None)
        return out
    begin = 0
    for b, (l, p) in enumerate(zip(n, past)):
        rows = slice(first[b], first[b] + l)
        for h in range(Hq):
            k, v = (s[x][begin:begin + l + p, h // group].double() for x in "kv")
            out[rows, h] = _softmax_rows(s["q"][rows, h].double(), k, v, s["scale"], p if case["causal"] else None)
        begin += l + p
    return out
