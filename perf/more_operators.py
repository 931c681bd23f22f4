"""Rotary positions in all their forms, and a paged cache in 8 bits whose blocks of 16 tokens carry an exponent per head: writing it,
reading it back, and the attention over it.  What is measured, in a plain form and through the package's entry points.

A case of kind
  table   makes the cosines and sines of `positions` positions, angles scaled for long contexts by `scaling`
  rotary  turns the queries and keys of `rows` tokens, or (transposed) takes their gradients back
  append  turns the queries and keys of new tokens and writes keys and values to the cache
  read    reads the tokens of sequences back
  extend  is causal attention of `news` new tokens behind `contexts` cached ones, which stand in the cache like them
  decode  is one token of every sequence: `segs` sequences of each expert, which share their expert's first `prefix` tokens
          and have `private` tokens of their own
Heads are those of a Mistral-7B block (32 query, 8 key / value heads of 128), of a LLaMA-2-13B one (40 of 128 each), or
generic.  Lists of lengths are "3,1,7", or "256:1:4096:5" for 256 of them between 1 and 4096, spread over their logarithm.

The cache holds, for every layer, page, key / value head and block of 16 tokens, e4m3 codes and one exponent e; a value is
code 2^e.  Writing new tokens into a block gives it the least e >= -117 with |x| <= 448 2^e for all finite x of them, or the block's e
where it holds older tokens and that is larger; the older tokens' codes are then rounded to the new e.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BLOCK, LEAST, MOST = 16, -117, 120
BF16, FP32 = "bf16", "fp32"


def _heads(heads=32, kv_heads=8, dim=128):
    return {"heads": heads, "kv_heads": kv_heads, "dim": dim}


def _turns(dims=128, pairs=False):
    return {"turned": dims, "pairs": pairs}


def _table(positions, dims, scaling="", factor=1.0, context=0, low=1.0, high=32.0, magnitude=1.0, base=10000.0):
    return {"kind": "table", "positions": positions, "turned": dims, "scaling": scaling, "factor": factor, "context": context, "low": low, "high": high,
            "magnitude": magnitude, "base": base}


def listed():
    return [
        # angles of a short context, made when a program starts
        _table(2048, 64) | {"name": "table_short"},
        # ... and of a context 16 times as long as the one trained at, slow dimensions stretched and fast ones left
        _table(131072, 128, "bands", 16.0, 8192, 1.0, 32.0, 0.1 * math.log(16.0) + 1.0) | {"name": "table_long_bands"},
        # the tokens of a small decode batch, padding rows among them, neighbours turned, half of the head
        {"name": "rotary_decode_pairs", "kind": "rotary", "rows": 21, "type": BF16, "transposed": False, "padding": 5, **_heads(), **_turns(64, True)},
        # gradients of a long batch's queries and keys, back through the rotation
        {"name": "rotary_gradient_8192", "kind": "rotary", "rows": 8192, "type": BF16, "transposed": True, "padding": 0, **_heads(), **_turns()},
        # the new tokens of a large decode batch
        {"name": "append_decode_256", "kind": "append", "contexts": "256:1:60:7", "news": "256:1:1:0", "page": 16, "layers": 1, **_heads(), **_turns()},
        # prompts behind contexts that end anywhere in a block, neighbours turned, half of the head
        {"name": "append_prompts_pairs", "kind": "append", "contexts": "0,77,1030,5", "news": "1024,1100,977,995", "page": 64, "layers": 2, **_heads(),
         **_turns(64, True)},
        # one short sequence read back
        {"name": "read_one", "kind": "read", "lens": "201", "page": 16, "layers": 2, **_heads()},
        # a batch of contexts read back, for instance into another cache
        {"name": "read_64_contexts", "kind": "read", "lens": "64:64:6000:9", "page": 32, "layers": 1, **_heads()},
        # questions behind a cached system prompt, or the next piece of a long prompt
        {"name": "extend_cached", "kind": "extend", "contexts": "1024,1024,2040,0,1024,77,4096,1024", "news": "64,700,130,333,1,17,512,250",
         "page": 16, "layers": 2, **_heads()},
        # long pieces, no shared heads
        {"name": "extend_long_mha", "kind": "extend", "contexts": "0,5001,0,2048", "news": "3001,1500,1,777", "page": 64, "layers": 1, **_heads(40, 40)},
        # a handful of short sequences
        {"name": "decode_few", "kind": "decode", "segs": "5", "prefix": "0", "private": "1,900,77,0,260", "page": 32, "layers": 2, **_heads(28, 4)},
        # a large batch of 9 experts, most with a system prompt of their own; sequences that have ended keep their rows
        {"name": "decode_256_experts", "kind": "decode", "segs": "90,40,31,9,3,2,1,0,80", "prefix": "2047,700,512,1600,64,4000,300,9,0",
         "private": "0,0,8192,253:16:4096:6", "page": 16, "layers": 1, **_heads()},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _lengths(text):
    """The numbers that a list of lengths stands for."""
    out = []
    for part in str(text).split(","):
        if ":" in part:
            n, lo, hi, seed = (int(v) for v in part.split(":"))
            rng = random.Random(seed)
            out += [_log_int(rng, lo, hi) for _ in range(n)]
        else:
            out.append(int(part))
    return out


def draw(rng):
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (40, 40, 128), (16, 16, 64), (8, 1, 128), (12, 4, 64), (28, 4, 128), (32, 8, 128)])
    kind = rng.choice(["table", "rotary", "append", "append", "read", "extend", "extend", "decode", "decode"])
    if kind == "table":
        context, factor = rng.choice([1000, 2048, 4096, 8192]), rng.choice([1.5, 4.0, 16.0, 40.0])
        return _table(_log_int(rng, 1, 131072), rng.choice([16, 48, 64, 96, 128]), rng.choice(["", "linear", "base", "bands"]), factor, context,
                      *rng.choice([(1.0, 32.0), (1.0, 4.0)]), rng.choice([1.0, 0.1 * math.log(factor) + 1.0]), rng.choice([10000.0, 500000.0]))
    h, turns = _heads(heads, kv_heads, dim), _turns(rng.choice([16, dim // 4, dim // 2, 3 * dim // 4, dim, dim]), rng.random() < 0.5)
    if kind == "rotary":
        rows = _log_int(rng, 1, 8192)
        return {"kind": kind, "rows": rows, "type": rng.choice([BF16, BF16, FP32]), "transposed": rng.random() < 0.5, "padding": rng.randint(0, rows) // 3, **h, **turns}
    paged = {"page": rng.choice([16, 32, 64, 128, 256]), "layers": rng.choice([1, 2])}
    n = _log_int(rng, 1, 128)
    if kind == "append":
        few = rng.random() < 0.5
        return {"kind": kind, "contexts": ",".join(str(rng.choice([0, _log_int(rng, 1, 300)])) for _ in range(n)),
                "news": "%d:1:%d:%d" % (n, 1 if few else max(2, 2000 // n), rng.randrange(1000)), **h, **turns, **paged}
    if kind == "read":
        lens = [_log_int(rng, 1, 1 + int(60000 / n ** 0.8))] + [rng.choice([0, 1, 1, 1, 1]) * _log_int(rng, 1, 1 + int(60000 / n ** 0.8)) for _ in range(n - 1)]
        return {"kind": kind, "lens": ",".join(map(str, lens)), **h, **paged}
    if kind == "extend":
        n = _log_int(rng, 1, 16)
        news = [_log_int(rng, 1, int(1500 / n ** 0.5)) for _ in range(n)]
        contexts = [rng.choice([0, _log_int(rng, 1, int(5000 / n ** 0.5))]) for _ in range(n)]
        return {"kind": kind, "contexts": ",".join(map(str, contexts)), "news": ",".join(map(str, news)), **h, **paged}
    experts = _log_int(rng, 1, 16)
    counts = [0] * experts
    for e in rng.choices(range(experts), [r ** -1.1 for r in range(1, experts + 1)], k=n):
        counts[e] += 1
    prefix = [rng.choice([0, _log_int(rng, 1, 6000)]) for _ in range(experts)]
    return {"kind": kind, "segs": ",".join(map(str, counts)), "prefix": ",".join(map(str, prefix)),
            "private": "%d:1:%d:%d" % (n, _log_int(rng, 8, 2000), rng.randrange(1000)), **h, **paged}


# ---------------------------------------------------------------------------------------------------------- inputs

def _sequences(case):
    """(prefix, length, new tokens) of every sequence, and the number of sequences of every expert."""
    if case["kind"] == "decode":
        segs, prefix, private = _lengths(case["segs"]), _lengths(case["prefix"]), _lengths(case["private"])
        pre = [prefix[e] for e, c in enumerate(segs) for _ in range(c)]
        return pre, [p + v if v else 0 for p, v in zip(pre, private)], [1] * len(pre), segs
    if case["kind"] == "read":
        news = _lengths(case["lens"])
        return [0] * len(news), news, news, [len(news)]
    news = _lengths(case["news"])
    total = [c + n for c, n in zip(_lengths(case["contexts"]), news)]
    return [0] * len(news), total, news, [len(news)]


def _cache(case, g, n_pages):
    """Codes [layers, pages, heads, tokens of a page, head dimension] and exponents [layers, pages, heads, blocks of a page]: keys and values of size
    1, some blocks of them four times as large."""
    shape = (case["layers"], n_pages, case["kv_heads"], case["page"], case["dim"])
    out = []
    for _ in range(2):
        codes = (torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) * 90).clamp_(-448, 448).to(torch.float8_e4m3fn)
        up = torch.randint(0, 8, (*shape[:3], shape[3] // BLOCK), generator=g, device=DEV)
        out += [codes, (120 + (up > 1).int() + 2 * (up > 6).int()).to(torch.uint8).view(torch.float8_e8m0fnu)]
    return {"k_cache": out[0], "k_exponent": out[1], "v_cache": out[2], "v_exponent": out[3]}


def _rows(case, g, tokens, std=1.0):
    q = torch.randn(tokens, case["heads"], case["dim"], generator=g, device=DEV)
    k, v = (torch.randn(tokens, case["kv_heads"], case["dim"], generator=g, device=DEV) for _ in range(2))
    return (q * std).to(torch.bfloat16), k.to(torch.bfloat16), v.to(torch.bfloat16)


def _offsets(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _angles(n, dims):
    angle = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, dims, 2, device=DEV, dtype=torch.float64) / dims)
    return torch.stack([angle.cos(), angle.sin()], 1).float()                          # [positions, 2, dims / 2]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"kind": case["kind"], "case": dict(case)}
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    if case["kind"] == "table":
        # another seed, another base: nothing else goes in
        return {**s, "base": case["base"] * (1 + (int(seed) % 1000) / 4000)}
    host = random.Random(int(seed))
    if case["kind"] == "rotary":
        q, k, _ = _rows(case, g, case["rows"])
        if case["type"] == FP32:
            q, k = q.float() + 1e-3, k.float() - 1e-3
        at = torch.randint(0, 8192, (case["rows"],), generator=g, device=DEV, dtype=torch.int32)
        pad = host.sample(range(case["rows"]), case["padding"])
        at[ints(pad).long()] = -1
        return {**s, "q": q, "k": k, "positions": at, "rotary": _angles(8192, case["turned"])}
    prefix, total, news, segs = _sequences(case)
    page, width = case["page"], -(-max(total + [1]) // case["page"])
    need, bounds = [-(-t // page) for t in total], _offsets(segs)
    shared = [prefix[a] // page if b > a else 0 for a, b in zip(bounds, bounds[1:])]
    n_pages = sum(need) + 3
    ids = iter(host.sample(range(n_pages), n_pages))
    table, first = [], []
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        common = [next(ids) for _ in range(shared[e])] if sum(total[a:b]) else []
        lead = next((i for i in range(a, b) if total[i]), a)
        for i in range(a, b):
            row = common[:need[i]] + [next(ids) for _ in range(max(0, need[i] - len(common)))]
            table.append(row + [0] * (width - len(row)))
            first.append(lead)
    s.update(_cache(case, g, n_pages), table=ints(table), kv_len=ints(total), longest=max(total + [1]))
    # a page that a prefix ends in is every sequence's own, with the same tokens, under exponents of its own where those are other blocks'
    odd = [i for i, p in enumerate(prefix) if p % page and total[i] > p - p % page and first[i] != i]
    if odd:
        at = ints([prefix[i] // page for i in odd]).long()
        rows, lead = ints(odd).long(), ints([first[i] for i in odd]).long()
        mine, lead = s["table"][rows, at].long(), s["table"][lead, at].long()
        keep = torch.arange(page, device=DEV)[None] < ints([prefix[i] % page for i in odd])[:, None]
        for c, x in ((s["k_cache"].view(torch.uint8), s["k_exponent"].view(torch.uint8)), (s["v_cache"].view(torch.uint8), s["v_exponent"].view(torch.uint8))):
            c[:, mine] = torch.where(keep[None, :, None, :, None], c[:, lead], c[:, mine])
            x[:, mine] = torch.where(keep[None, :, None, ::BLOCK], x[:, lead], x[:, mine])
    if case["kind"] == "decode":
        s.update(segs=bounds, prefix=_lengths(case["prefix"]))
    else:
        s.update(offsets=ints(_offsets(news)), new_longest=max(news), tokens=sum(news))
    if case["kind"] == "read":
        return s
    q, k, v = _rows(case, g, sum(news), 1.0 if case["kind"] == "append" else 2.0)
    s["q"] = q
    if case["kind"] == "append":
        # a token in eight is larger than its neighbours, as first tokens of sequences are
        k = k * torch.where(torch.rand(len(k), generator=g, device=DEV) < 0.125, 6.0, 1.0)[:, None, None].to(k.dtype)
        s.update(k=k, v=v, rotary=_angles(width * page, case["turned"]))
    return s


# ------------------------------------------------------------------------------------------------------- plain form

def _plain_table(s):
    c = s["case"]
    n = c["turned"]
    i = torch.arange(0, n, 2, device=DEV, dtype=torch.float64)
    base = s["base"] * c["factor"] ** (n / (n - 2)) if c["scaling"] == "base" else s["base"]
    f = base ** (-i / n)
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "bands":
        keep = ((c["context"] * f / (2 * math.pi) - c["low"]) / (c["high"] - c["low"])).clamp(0, 1)
        f = f * (keep + (1 - keep) / c["factor"])
    angle = torch.arange(c["positions"], device=DEV, dtype=torch.float64)[:, None] * f
    return (torch.stack([angle.cos(), angle.sin()], 1) * c["magnitude"]).float()


def _turned(x, rotary, at, pairs, transposed=False):
    """Rows x [n, heads, d] in fp32: the first 2 rotary.shape[2] dimensions turned by the angles of positions `at`, the others as they are."""
    half = rotary.shape[2]
    c, sn = rotary[at][:, None, 0], rotary[at][:, None, 1]
    if transposed:
        sn = -sn
    x = x.float()
    a, b = (x[..., :2 * half:2], x[..., 1:2 * half:2]) if pairs else (x[..., :half], x[..., half:2 * half])
    y = [a * c - b * sn, b * c + a * sn]
    return torch.cat([torch.stack(y, -1).flatten(-2) if pairs else torch.cat(y, -1), x[..., 2 * half:]], -1)


def _plain_rotary(s):
    c, at = s["case"], s["positions"].long()
    there = (at >= 0)[:, None, None]
    return tuple(torch.where(there, _turned(x, s["rotary"], at.clamp_min(0), c["pairs"], c["transposed"]), 0.0).to(x.dtype) for x in (s["q"], s["k"]))


def _power(e):
    """2^e in fp32, for whole e of -149 to 127 (0 below)."""
    return torch.exp2(e.double()).float()


def _put(codes, exponent, x, page, slot):
    """Writes rows x [n, heads, d] to slots of pages of a layer: what stands before a call's first token in its block is older."""
    pages, heads, size, d = codes.shape
    blocks = size // BLOCK
    where = page * blocks + slot // BLOCK
    finite = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)                          # [n, heads]
    top = torch.zeros(pages * blocks, heads, device=DEV).scatter_reduce_(0, where[:, None].expand(-1, heads), finite, "amax")
    first = torch.full((pages * blocks,), BLOCK, device=DEV).scatter_reduce_(0, where, slot % BLOCK, "amin")
    m, e = torch.frexp(top)                                                                 # top = m 2^e, 0.5 <= m < 1
    e = torch.where(top > 0, e - 9 + (m > 0.875), LEAST).clamp_min(LEAST)                   # 448 = 0.875 2^9
    now = (exponent.view(torch.uint8).int() - 127).transpose(1, 2).reshape(pages * blocks, heads)
    touched = (first < BLOCK)[:, None]
    new = torch.where(touched, torch.where((first > 0)[:, None], torch.maximum(e, now), e), now)
    shape = (pages, blocks, heads)
    # the older tokens of the blocks written to
    follow = _power((now - new).view(shape).transpose(1, 2))[..., None, None]
    c = codes.view(torch.uint8).view(pages, heads, blocks, BLOCK, d)
    older = touched.view(pages, 1, blocks, 1, 1) & (torch.arange(BLOCK, device=DEV)[:, None] < first.view(pages, 1, blocks, 1, 1))
    c.copy_(torch.where(older, (c.view(torch.float8_e4m3fn).float() * follow).to(torch.float8_e4m3fn).view(torch.uint8), c))
    exponent.view(torch.uint8).copy_((new.view(shape).transpose(1, 2) + 127).to(torch.uint8))
    mine = new[where]
    limit = torch.where(mine == MOST, 240.0, 448.0)[..., None]                               # 448 2^120 is no finite number
    code = (x * _power(-mine)[..., None]).clamp(-limit, limit).to(torch.float8_e4m3fn)
    codes.view(torch.uint8)[page, :, slot] = code.view(torch.uint8)


def _plain_append(s):
    token = torch.arange(len(s["q"]), device=DEV)
    seq = torch.searchsorted(s["offsets"][1:].contiguous(), token, right=True)
    at = (s["kv_len"][seq] - s["offsets"][seq + 1] + token).long()
    size = s["k_cache"].shape[3]
    page, slot = s["table"][seq, at // size].long(), at % size
    pairs = s["case"]["pairs"]
    _put(s["k_cache"][-1], s["k_exponent"][-1], _turned(s["k"], s["rotary"], at, pairs), page, slot)
    _put(s["v_cache"][-1], s["v_exponent"][-1], s["v"].float(), page, slot)
    return _turned(s["q"], s["rotary"], at, pairs).to(torch.bfloat16), s["k_cache"], s["k_exponent"], s["v_cache"], s["v_exponent"]


def _read(cache, exponent, table, longest):
    """[n, kv heads, longest, d] of the last layer in fp32: the tokens that the page tables name."""
    size = cache.shape[3]
    pages = table[:, : -(-longest // size)].long()
    x = cache[-1].view(torch.uint8)[pages].view(cache.dtype).float()                        # [n, pages, heads, page, d]
    e = _power(exponent[-1].view(torch.uint8)[pages].int() - 127)                           # [n, pages, heads, blocks]
    n, p, h, t, d = x.shape
    x = (x.view(n, p, h, t // BLOCK, BLOCK, d) * e[..., None, None]).view(n, p, h, t, d)
    return x.permute(0, 2, 1, 3, 4).reshape(n, h, p * t, d)[:, :, :longest]


def _padded(offsets, longest):
    """[n, longest] rows of packed sequences, and which of them are there."""
    at = torch.arange(longest, device=DEV)
    there = at[None] < (offsets[1:] - offsets[:-1])[:, None]
    return torch.where(there, offsets[:-1, None] + at[None], 0).long(), there


def _plain_read(s):
    _, there = _padded(s["offsets"], s["longest"])
    return tuple(_read(s[x + "_cache"], s[x + "_exponent"], s["table"], s["longest"]).transpose(1, 2)[there].to(torch.bfloat16) for x in "kv")


def _softmax_of(q, k, v, visible):
    """q [n, heads, rows, d], k and v [n, kv heads, tokens, d], visible [n, rows, tokens]; rows that see nothing are 0."""
    n, heads, rows, d = q.shape
    m = k.shape[1]
    score = (q.reshape(n, m, heads // m * rows, d) @ k.transpose(2, 3)).view(n, m, heads // m, rows, -1) * d ** -0.5
    score.masked_fill_(~visible[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp_min(-3e38)
    p = score.sub_(top).exp_()
    norm = p.sum(-1, keepdim=True)
    o = p.view(n, m, -1, p.shape[-1]) @ v
    o = o.view(n, m, heads // m, rows, d) / torch.where(norm > 0, norm, torch.ones_like(norm))
    return o.reshape(n, heads, rows, d)


def _plain_attention(s):
    """Queries are the last tokens of their sequences."""
    n = len(s["kv_len"])
    offsets = s.get("offsets", torch.arange(n + 1, dtype=torch.int32, device=DEV))
    rows, there = _padded(offsets, s.get("new_longest", 1))
    at = torch.arange(rows.shape[1], device=DEV)
    last = s["kv_len"][:, None] - (offsets[1:] - offsets[:-1])[:, None] + at[None]
    visible = torch.arange(s["longest"], device=DEV)[None, None] <= last[:, :, None]
    o = _softmax_of(s["q"][rows].transpose(1, 2).float(), _read(s["k_cache"], s["k_exponent"], s["table"], s["longest"]).contiguous(),
                    _read(s["v_cache"], s["v_exponent"], s["table"], s["longest"]).contiguous(), visible)
    out = torch.empty(s["q"].shape, dtype=torch.bfloat16, device=DEV)
    out[rows[there]] = o.transpose(1, 2)[there].to(torch.bfloat16)
    return out


# ----------------------------------------------------------------------------------------------- the package's calls

def _kept(s):
    """What a program keeps beside its cache: descriptors of the cache, the angles and the batch of sequences, the decode workspace."""
    if "mes" not in s:
        import paper_2406_09041_amd as mes

        s["mes"] = mes
        if "k_cache" in s:
            s["cache"] = mes.KvCache.over(s["k_cache"], s["v_cache"], s["k_exponent"], s["v_exponent"])
            s["batch"] = mes.SeqBatch(s["kv_len"], s["table"], s.get("offsets"))
        if "rotary" in s:
            s["angles"] = mes.Angles(s["rotary"], interleaved=s["case"]["pairs"])
        if s["kind"] == "decode":
            s["decode"] = mes.AttnDecode(s["cache"], s["q"].shape[1], max_seqs=len(s["kv_len"]))
    return s["mes"]


def _own(s):
    mes = _kept(s)
    kind, c = s["kind"], s["case"]
    if kind == "table":
        return mes.mes_rotary_table(c["positions"], c["turned"], s["base"], scaling=c["scaling"] or None, factor=c["factor"], context=c["context"],
                                    low=c["low"], high=c["high"], magnitude=c["magnitude"], device=DEV)
    if kind == "rotary":
        return mes.mes_rotary(s["angles"], s["positions"], s["q"], s["k"], transpose=c["transposed"])
    layer = s["k_cache"].shape[0] - 1
    if kind == "append":
        q = mes.mes_kv_append(s["cache"], layer, s["batch"], s["q"], s["k"], s["v"], s["angles"])
        return q, s["k_cache"], s["k_exponent"], s["v_cache"], s["v_exponent"]
    if kind == "read":
        return mes.mes_kv_read(s["cache"], layer, s["batch"], s["tokens"])
    if kind == "extend":
        return mes.mes_attn_extend(s["cache"], layer, s["batch"], s["q"])
    return s["decode"](layer, s["batch"], s["q"], s["segs"], s["prefix"])


def run(state):
    if own:
        return _own(state)
    return {"table": _plain_table, "rotary": _plain_rotary, "append": _plain_append, "read": _plain_read, "extend": _plain_attention,
            "decode": _plain_attention}[state["kind"]](state)


# ------------------------------------------------------------------------------------------------- work and 64 bits

def work(case):
    if case["kind"] == "table":
        return {"bytes": 4 * case["turned"] * case["positions"], "flops": 0}
    d, m, h = case["dim"], case["kv_heads"], case["heads"]
    if case["kind"] == "rotary":
        real = case["rows"] - case["padding"]
        return {"bytes": (case["rows"] + real) * (h + m) * d * (2 if case["type"] == BF16 else 4) + real * 4 * (case["turned"] + 1), "flops": 0}
    prefix, total, news, segs = _sequences(case)
    if case["kind"] == "append":
        places = len({t - i for t, n in zip(total, news) for i in range(1, n + 1)})
        return {"bytes": sum(news) * d * (4 * h + 4 * m + 2 * m) + 4 * case["turned"] * places + 2 * m * sum(-(-n // BLOCK) for n in news), "flops": 0}
    if case["kind"] == "read":
        return {"bytes": sum(news) * 2 * m * d * 3 + 2 * m * sum(-(-n // BLOCK) for n in news), "flops": 0}
    shared = 0
    for a, b in zip(_offsets(segs), _offsets(segs)[1:]):
        shared += max(0, sum(t > 0 for t in total[a:b]) - 1) * prefix[a] if b > a else 0
    return {"bytes": (sum(total) - shared) * 2 * m * (d + 1 / BLOCK) + sum(news) * h * d * 4,
            "flops": sum(4 * d * h * (n * t - n * (n - 1) // 2) for t, n in zip(total, news) if t)}


def _rotation(x, dims, at, pairs, back=False):
    """Rows x [n, heads, d] in 64 bits, as complex numbers times e^(i angle)."""
    i = torch.arange(dims // 2, device=DEV, dtype=torch.float64)
    angle = at.double()[:, None] * 10000.0 ** (-2.0 * i / dims)
    # the table is given, in fp32
    turn = torch.complex(angle.cos().float().double(), angle.sin().float().double())[:, None]
    turn = turn.conj() if back else turn
    x = x.double()
    y = x[..., :dims]
    y = y.reshape(*y.shape[:-1], -1, 2) if pairs else y.reshape(*y.shape[:-1], 2, -1).transpose(-1, -2)
    z = torch.complex(y[..., 0].contiguous(), y[..., 1].contiguous()) * turn
    y = torch.stack([z.real, z.imag], -1 if pairs else -2).reshape(*x.shape[:-1], dims)
    return torch.cat([y, x[..., dims:]], -1)


def _exact_table(case, seed):
    s = prepare(case, seed)
    n, base, f = case["turned"], s["base"], []
    if case["scaling"] == "base":
        base *= case["factor"] ** (n / (n - 2))
    for i in range(n // 2):
        x = math.pow(base, -2 * i / n)
        if case["scaling"] == "linear":
            x /= case["factor"]
        elif case["scaling"] == "bands":
            turns = case["context"] * x / math.tau
            keep = min(max((turns - case["low"]) / (case["high"] - case["low"]), 0.0), 1.0)
            x = keep * x + (1 - keep) * x / case["factor"]
        f.append(x)
    at = torch.outer(torch.arange(case["positions"], dtype=torch.float64, device=DEV), torch.tensor(f, dtype=torch.float64, device=DEV))
    turn = torch.polar(torch.full_like(at, case["magnitude"]), at)
    return torch.stack([turn.real, turn.imag], 1)


def _exact_append(case, s, bounds, total, news):
    at = torch.tensor([t - n + i for t, n in zip(total, news) for i in range(n)], device=DEV)
    k, v = _rotation(s["k"], case["turned"], at, case["pairs"]), s["v"].double()
    out = [_rotation(s["q"], case["turned"], at, case["pairs"])]
    pages, size, m = s["table"].tolist(), case["page"], case["kv_heads"]
    for x, codes, exponent in ((k, s["k_cache"], s["k_exponent"]), (v, s["v_cache"], s["v_exponent"])):
        c, e = codes.double(), exponent.double()
        for i, (t, n) in enumerate(zip(total, news)):
            begin = t - n
            for b in range(begin // BLOCK, -(-t // BLOCK)):
                lo, hi = max(begin, b * BLOCK), min(t, (b + 1) * BLOCK)
                page, block = pages[i][lo // size], lo % size // BLOCK
                rows = x[bounds[i] + lo - begin:bounds[i] + hi - begin].transpose(0, 1)                # [heads, tokens, d]
                least = torch.exp2(torch.ceil(torch.log2(rows.abs().amax((1, 2)) / 448)).clamp_min(LEAST))
                place = block * BLOCK
                if lo % BLOCK:
                    was = e[-1, page, :, block].clone()
                    least = torch.maximum(least, was)
                    c[-1, page, :, place:place + lo % BLOCK] *= (was / least)[:, None, None]
                e[-1, page, :, block] = least
                c[-1, page, :, place + lo % BLOCK:place + lo % BLOCK + hi - lo] = rows / least[:, None, None]
        out += [c, e]
    return tuple(out)


def exact(case, seed):
    if case["kind"] == "table":
        return _exact_table(case, seed)
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        there = (s["positions"] >= 0)[:, None, None]
        return tuple(torch.where(there, _rotation(x, case["turned"], s["positions"], case["pairs"], case["transposed"]), 0.0) for x in (s["q"], s["k"]))
    h, m, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    group = h // m
    _, total, news, _ = _sequences(case)
    bounds = _offsets(news)
    if kind == "append":
        # about a thousand small steps a second
        return _exact_append(case, s, bounds, total, news) if sum(news) // BLOCK + 2 * len(news) < 4000 else None

    def tokens(i, t):
        ids = s["table"][i, : -(-t // page)].long()
        out = []
        for x in "kv":
            c, e = s[x + "_cache"][-1].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double(), s[x + "_exponent"][-1].view(torch.uint8)[ids].double() - 127
            out.append((c * torch.exp2(e).repeat_interleave(BLOCK, -1)[..., None]).transpose(1, 2).reshape(-1, m, d)[:t])
        return out

    if kind == "read":
        got = [tokens(i, t) for i, t in enumerate(total)]
        return tuple(torch.cat([x[j] for x in got]) for j in range(2))
    out = torch.zeros(bounds[-1], h, d, dtype=torch.float64, device=DEV)
    for i, (t, n) in enumerate(zip(total, news)):
        if t == 0:
            continue
        q = s["q"][bounds[i]:bounds[i + 1]].double()
        k, v = tokens(i, t)
        after = torch.arange(t, device=DEV)[None] > (torch.arange(n, device=DEV) + t - n)[:, None]
        for c in range(h):
            e = (q[:, c] @ k[:, c // group].t() / math.sqrt(d)).masked_fill(after, -math.inf)
            out[bounds[i]:bounds[i + 1], c] = torch.softmax(e, -1) @ v[:, c // group]
    return out
