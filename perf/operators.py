"""The attention of a served transformer block, between the projections that the delta linears compute: prompts, prompts
behind a cached context, single tokens over a paged cache whose experts share system prompts, writing to that cache, and
moving its pages.  What is measured, in a plain form and through the package's entry points.

A case of kind
  prompt  is causal attention over packed prompts: `lens` tokens each, keys and values as the projections left them
  extend  is the same where keys and values stand in the cache: `news` new tokens behind `contexts` cached ones
  decode  is one token of every sequence: `segs` sequences of each expert, which share their expert's first `prefix` tokens
          and have `private` tokens of their own
  append  rotates the queries and keys of new tokens and puts keys and values into the cache
  copy    copies pages, all layers of keys and values
Heads are those of a Mistral-7B block (32 query, 8 key / value heads of 128), of a LLaMA-2-13B one (40 of 128 each), or
generic.  Lists of lengths are "3,1,7", or "256:1:4096:5" for 256 of them between 1 and 4096, spread over their logarithm.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BF16, E4M3 = "bf16", "e4m3"

# 64 decoding sequences on 16 experts, Zipf(1.1)
DECODE_64 = "25,8,6,3,3,5,4,1,3,1,0,3,1,1,0,0"


def _heads(heads=32, kv_heads=8, dim=128):
    return {"heads": heads, "kv_heads": kv_heads, "dim": dim}


def _paged(page=16, dtype=BF16, layers=1):
    return {"page": page, "dtype": dtype, "layers": layers}


def listed():
    return [
        # one short question: the smallest prompt, all latency
        {"name": "prompt_one", "kind": "prompt", "lens": "77", "fused": False, **_heads()},
        # the four prompts that share a batch with 256 decoding sequences
        {"name": "prompt_4x1024", "kind": "prompt", "lens": "1024,1024,1024,1024", "fused": False, **_heads()},
        # prompts of every length in one batch, no shared heads, q, k and v views of one buffer; the longest does most of it
        {"name": "prompt_ragged_mha", "kind": "prompt", "lens": "1,517,6001,129,64,1500", "fused": True, **_heads(40, 40)},
        # questions behind a cached system prompt, or the next piece of a long prompt
        {"name": "extend_cached", "kind": "extend", "contexts": "1024,1024,2040,0,1024,77,4096,1024", "news": "64,700,130,333,1,17,512,250",
         **_heads(), **_paged(layers=2)},
        # one sequence being decoded
        {"name": "decode_one", "kind": "decode", "segs": "1", "prefix": "0", "private": "200", **_heads(), **_paged(layers=2)},
        # a decode batch of 16 experts, each with its own system prompt
        {"name": "decode_64_experts", "kind": "decode", "segs": DECODE_64, "prefix": "16:512:1600:3", "private": "64:16:1024:4",
         **_heads(), **_paged()},
        # many users of one expert behind a long shared document, an 8-bit cache
        {"name": "decode_shared_e4m3", "kind": "decode", "segs": "96", "prefix": "8200", "private": "96:1:512:5", **_heads(), **_paged(64, E4M3)},
        # a large decode batch that shares nothing; sequences that have ended keep their rows, with nothing to look at
        {"name": "decode_256_ragged", "kind": "decode", "segs": "256", "prefix": "0", "private": "0,0,0,8192,252:16:4096:6",
         **_heads(), **_paged()},
        # the new tokens of a large decode batch, 8-bit cache
        {"name": "append_decode_256_e4m3", "kind": "append", "contexts": "256:1:60:7", "news": "256:1:1:0", **_heads(), **_paged(16, E4M3)},
        # ... and of four prompts
        {"name": "append_4x1024", "kind": "append", "contexts": "0,0,0,0", "news": "1024,1024,1024,1024", **_heads(), **_paged(layers=2)},
        # sequences forked inside a page: the first write to each copies that page
        {"name": "copy_fork", "kind": "copy", "pairs": 3, "kv_heads": 8, "dim": 128, **_paged(16, BF16, 32)},
        # a cache being compacted
        {"name": "copy_compact", "kind": "copy", "pairs": 400, "kv_heads": 8, "dim": 128, **_paged(16, BF16, 32)},
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
    kind = rng.choice(["prompt", "extend", "decode", "decode", "append", "copy"])
    h, paged = _heads(heads, kv_heads, dim), _paged(rng.choice([16, 32, 64, 128]), rng.choice([BF16, BF16, E4M3]), rng.choice([1, 2]))
    n = _log_int(rng, 1, 16)
    if kind == "prompt":
        lens = [_log_int(rng, 1, max(2, int(6000 / math.sqrt(n)))) for _ in range(n)]
        return {"kind": kind, "lens": ",".join(map(str, lens)), "fused": rng.random() < 0.5, **h}
    if kind == "extend":
        news = [_log_int(rng, 1, 700) for _ in range(n)]
        contexts = [rng.choice([0, _log_int(rng, 1, 4000)]) for _ in range(n)]
        return {"kind": kind, "contexts": ",".join(map(str, contexts)), "news": ",".join(map(str, news)), **h, **paged}
    if kind == "decode":
        n, experts = _log_int(rng, 1, 128), _log_int(rng, 1, 16)
        counts = [0] * experts
        for e in rng.choices(range(experts), [r ** -1.1 for r in range(1, experts + 1)], k=n):
            counts[e] += 1
        prefix = [rng.choice([0, _log_int(rng, 1, 6000)]) for _ in range(experts)]
        return {"kind": kind, "segs": ",".join(map(str, counts)), "prefix": ",".join(map(str, prefix)),
                "private": "%d:1:%d:%d" % (n, _log_int(rng, 8, 2000), rng.randrange(1000)), **h, **paged}
    if kind == "append":
        n = _log_int(rng, 1, 128)
        return {"kind": kind, "contexts": "%d:1:%d:%d" % (n, _log_int(rng, 2, 300), rng.randrange(1000)),
                "news": "%d:1:%d:%d" % (n, rng.choice([1, 40]), rng.randrange(1000)), **h, **paged}
    return {"kind": kind, "pairs": _log_int(rng, 1, 200), "kv_heads": kv_heads, "dim": dim, **{**paged, "layers": rng.choice([2, 13, 24])}}


# ---------------------------------------------------------------------------------------------------------- inputs

def _sequences(case):
    """(prefix, length, new tokens) of every sequence, and the number of sequences of every expert."""
    if case["kind"] == "decode":
        segs, prefix, private = _lengths(case["segs"]), _lengths(case["prefix"]), _lengths(case["private"])
        pre = [prefix[e] for e, c in enumerate(segs) for _ in range(c)]
        return pre, [p + v for p, v in zip(pre, private)], [1] * len(pre), segs
    news = _lengths(case["news"])
    total = [c + n for c, n in zip(_lengths(case["contexts"]), news)]
    return [0] * len(news), total, news, [len(news)]


def _cache(case, g, n_pages):
    """Keys and values [layers, pages, heads, tokens of a page, head dimension], and an 8-bit cache's scales."""
    shape = (case["layers"], n_pages, case["kv_heads"], case["page"], case["dim"])
    if case["dtype"] == BF16:
        k, v = (torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        return {"k_cache": k, "v_cache": v, "k_scale": None, "v_scale": None}
    k, v = ((torch.randn(shape, generator=g, device=DEV) * 40).to(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (0.02 + 0.01 * torch.rand(shape[0], shape[2], generator=g, device=DEV) for _ in range(2))
    return {"k_cache": k, "v_cache": v, "k_scale": ks, "v_scale": vs}


def _rows(case, g, tokens, std=1.0):
    q = torch.randn(tokens, case["heads"], case["dim"], generator=g, device=DEV)
    k, v = (torch.randn(tokens, case["kv_heads"], case["dim"], generator=g, device=DEV) for _ in range(2))
    return (q * std).to(torch.bfloat16), k.to(torch.bfloat16), v.to(torch.bfloat16)


def _offsets(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"kind": case["kind"], "case": dict(case)}
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    if case["kind"] == "prompt":
        lens = _lengths(case["lens"])
        q, k, v = _rows(case, g, sum(lens), 2.0)
        if case["fused"]:
            h, m = case["heads"], case["kv_heads"]
            row = torch.cat([q, k, v], 1).reshape(sum(lens), h + 2 * m, case["dim"])
            q, k, v = row[:, :h], row[:, h:h + m], row[:, h + m:]
        return {**s, "q": q, "k": k, "v": v, "offsets": ints(_offsets(lens)), "longest": max(lens)}
    host = random.Random(int(seed))
    if case["kind"] == "copy":
        n = case["pairs"]
        pages = host.sample(range(2 * n + 7), 2 * n)
        return {**s, **_cache(case, g, 2 * n + 7), "src": pages[:n], "dst": pages[n:]}
    prefix, total, news, segs = _sequences(case)
    page, width = case["page"], -(-max(total + [1]) // case["page"])
    need, bounds = [-(-t // page) for t in total], _offsets(segs)
    shared = [prefix[a] // page if b > a else 0 for a, b in zip(bounds, bounds[1:])]
    n_pages = sum(need) + 3
    ids = iter(host.sample(range(n_pages), n_pages))
    table, first = [], []
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        common = [next(ids) for _ in range(shared[e])] if sum(total[a:b]) else []
        for i in range(a, b):
            row = common[:need[i]] + [next(ids) for _ in range(max(0, need[i] - len(common)))]
            table.append(row + [0] * (width - len(row)))
            first.append(a)
    s.update(_cache(case, g, n_pages), table=ints(table), kv_len=ints(total), longest=max(total))
    # a page that a prefix ends in is every sequence's own, with the same tokens
    odd = [i for i, p in enumerate(prefix) if p % page and total[i] > p - p % page and first[i] != i]
    if odd:
        at = ints([prefix[i] // page for i in odd]).long()
        rows, lead = ints(odd).long(), ints([first[i] for i in odd]).long()
        mine, lead = s["table"][rows, at].long(), s["table"][lead, at].long()
        keep = torch.arange(page, device=DEV)[None] < ints([prefix[i] % page for i in odd])[:, None]
        for c in (s["k_cache"].view(torch.uint8), s["v_cache"].view(torch.uint8)):
            c[:, mine] = torch.where(keep[None, :, None, :, None], c[:, lead], c[:, mine])
    q, k, v = _rows(case, g, sum(news), 1.0 if case["kind"] == "append" else 2.0)
    s.update(q=q, segs=bounds, prefix=_lengths(case["prefix"]) if case["kind"] == "decode" else None)
    if case["kind"] != "decode":
        s.update(offsets=ints(_offsets(news)), new_longest=max(news))
    if case["kind"] == "append":
        angle = torch.arange(width * page, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(0, case["dim"], 2, device=DEV, dtype=torch.float64) / case["dim"])
        s.update(k=k, v=v, rotary=torch.stack([angle.cos(), angle.sin()], 1).float())   # [positions, 2, dim / 2]
    return s


# ------------------------------------------------------------------------------------------------------- plain form

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


def _padded(offsets, longest):
    """[n, longest] rows of packed sequences, and which of them are there."""
    at = torch.arange(longest, device=DEV)
    there = at[None] < (offsets[1:] - offsets[:-1])[:, None]
    return torch.where(there, offsets[:-1, None] + at[None], 0).long(), there


def _read(cache, scale, table, longest):
    """[n, kv heads, longest, d] of the last layer in fp32: the tokens that the page tables name."""
    page = cache.shape[3]
    pages = table[:, : -(-longest // page)].long()
    x = cache[-1].view(torch.uint8)[pages].view(cache.dtype).float()     # [n, pages, heads, page, d]
    n, p, h, t, d = x.shape
    x = x.permute(0, 2, 1, 3, 4).reshape(n, h, p * t, d)[:, :, :longest]
    return x if scale is None else x * scale[-1][None, :, None, None]


def _plain_prompt(s):
    rows, there = _padded(s["offsets"], s["longest"])
    take = lambda t: t[rows].transpose(1, 2).float().contiguous()  # noqa: E731
    at = torch.arange(s["longest"], device=DEV)
    o = _softmax_of(take(s["q"]), take(s["k"]), take(s["v"]), (at[None, :] <= at[:, None])[None].expand(len(rows), -1, -1))
    out = torch.empty(s["q"].shape, dtype=torch.bfloat16, device=DEV)
    out[rows[there]] = o.transpose(1, 2)[there].to(torch.bfloat16)
    return out


def _plain_cached(s):
    """Queries are the last tokens of their sequences."""
    n = len(s["kv_len"])
    offsets = s.get("offsets", torch.arange(n + 1, dtype=torch.int32, device=DEV))
    rows, there = _padded(offsets, s.get("new_longest", 1))
    at = torch.arange(rows.shape[1], device=DEV)
    last = s["kv_len"][:, None] - (offsets[1:] - offsets[:-1])[:, None] + at[None]
    visible = torch.arange(s["longest"], device=DEV)[None, None] <= last[:, :, None]
    o = _softmax_of(s["q"][rows].transpose(1, 2).float(), _read(s["k_cache"], s["k_scale"], s["table"], s["longest"]),
                    _read(s["v_cache"], s["v_scale"], s["table"], s["longest"]), visible)
    out = torch.empty(s["q"].shape, dtype=torch.bfloat16, device=DEV)
    out[rows[there]] = o.transpose(1, 2)[there].to(torch.bfloat16)
    return out


def _rotated(x, rotary, at):
    c, sn = rotary[at][:, None, 0], rotary[at][:, None, 1]
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * c - b * sn, b * c + a * sn], -1)


def _plain_append(s):
    token = torch.arange(len(s["q"]), device=DEV)
    seq = torch.searchsorted(s["offsets"][1:].contiguous(), token, right=True)
    at = (s["kv_len"][seq] - s["offsets"][seq + 1] + token).long()
    page = s["k_cache"].shape[3]
    where = s["table"][seq, at // page].long()
    for x, cache, scale in ((_rotated(s["k"], s["rotary"], at), s["k_cache"], s["k_scale"]), (s["v"].float(), s["v_cache"], s["v_scale"])):
        x = x if scale is None else (x / scale[-1][None, :, None]).clamp(-448, 448)
        item = torch.int16 if scale is None else torch.uint8
        cache[-1].view(item)[where, :, at % page] = x.to(cache.dtype).view(item)
    return _rotated(s["q"], s["rotary"], at).to(torch.bfloat16), s["k_cache"], s["v_cache"]


def _plain_copy(s):
    src, dst = (torch.tensor(s[x], device=DEV) for x in ("src", "dst"))
    for c in (s["k_cache"], s["v_cache"]):
        c.view(torch.uint8)[:, dst] = c.view(torch.uint8)[:, src]
    return s["k_cache"], s["v_cache"]


# ----------------------------------------------------------------------------------------------- the package's calls

def _kept(s):
    """What a program keeps beside its cache: the cache's descriptor, the batch of sequences, the decode workspace."""
    if "cache" not in s:
        import paper_2406_09041_amd as mes

        s["mes"] = mes
        if "k_cache" in s:
            s["cache"] = mes.KvCache.over(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        else:
            s["cache"] = None
        if "table" in s:
            s["batch"] = mes.SeqBatch(s["kv_len"], s["table"], s.get("offsets"))
        if s["kind"] == "decode":
            s["decode"] = mes.AttnDecode(s["cache"], s["q"].shape[1], max_seqs=len(s["kv_len"]))
    return s["mes"]


def _own(s):
    mes = _kept(s)
    kind = s["kind"]
    if kind == "prompt":
        return mes.mes_attn_prompt(s["q"], s["k"], s["v"], s["offsets"])
    layer = s["k_cache"].shape[0] - 1
    if kind == "extend":
        return mes.mes_attn_extend(s["cache"], layer, s["batch"], s["q"])
    if kind == "decode":
        return s["decode"](layer, s["batch"], s["q"], s["segs"], s["prefix"])
    if kind == "append":
        return mes.mes_kv_append(s["cache"], layer, s["batch"], s["q"], s["k"], s["v"], s["rotary"]), s["k_cache"], s["v_cache"]
    mes.mes_kv_copy_pages(s["cache"], s["src"], s["dst"])
    return s["k_cache"], s["v_cache"]


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_prompt, "extend": _plain_cached, "decode": _plain_cached, "append": _plain_append, "copy": _plain_copy}[state["kind"]](state)


# ------------------------------------------------------------------------------------------------- work and 64 bits

def work(case):
    item = 1 if case.get("dtype") == E4M3 else 2
    d, m = case["dim"], case["kv_heads"]
    if case["kind"] == "copy":
        return {"bytes": 2 * case["pairs"] * case["layers"] * 2 * m * case["page"] * d * item, "flops": 0}
    h = case["heads"]
    if case["kind"] == "prompt":
        lens = _lengths(case["lens"])
        return {"bytes": sum(lens) * d * 2 * (2 * h + 2 * m), "flops": sum(4 * d * h * t * (t + 1) // 2 for t in lens)}
    prefix, total, news, segs = _sequences(case)
    if case["kind"] == "append":
        return {"bytes": sum(news) * d * (4 * h + 4 * m + 2 * m * item) + 8 * (d // 2) * len({t - i for t, n in zip(total, news) for i in range(1, n + 1)}),
                "flops": 0}
    shared = 0
    for a, b in zip(_offsets(segs), _offsets(segs)[1:]):
        shared += max(0, b - a - 1) * prefix[a] if b > a else 0
    return {"bytes": (sum(total) - shared) * 2 * m * d * item + sum(news) * h * d * 4,
            "flops": sum(4 * d * h * (n * t - n * (n - 1) // 2) for t, n in zip(total, news) if t)}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "copy":
        k, v = s["k_cache"].float(), s["v_cache"].float()
        for a, b in zip(s["src"], s["dst"]):
            k[:, b], v[:, b] = k[:, a], v[:, a]
        return k, v
    h, m, d = case["heads"], case["kv_heads"], case["dim"]
    group = h // m
    if kind == "prompt":
        bounds = s["offsets"].tolist()
        total = news = [b - a for a, b in zip(bounds, bounds[1:])]
    else:
        _, total, news, _ = _sequences(case)
        bounds, page = _offsets(news), case["page"]
    if kind == "append":
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        at = torch.tensor([t - n + i for t, n in zip(total, news) for i in range(n)], device=DEV, dtype=torch.float64)
        turn = torch.polar(torch.ones(len(at), d // 2, dtype=torch.float64, device=DEV),
                           at[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=torch.float64) / d))[:, None]
        def rotate(x):
            z = torch.complex(x[..., : d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
            return torch.cat([z.real, z.imag], -1)
        out_k, out_v, k = s["k_cache"].double(), s["v_cache"].double(), rotate(k)
        if s["k_scale"] is not None:
            limit = lambda x, y: (x / y[-1].double()[:, None]).clamp(-448, 448)  # noqa: E731
            k, v = limit(k, s["k_scale"]), limit(v, s["v_scale"])
        pages, row = s["table"].tolist(), 0
        where, slot = [], []
        for i, (t, n) in enumerate(zip(total, news)):
            where += [pages[i][p // page] for p in range(t - n, t)]
            slot += [p % page for p in range(t - n, t)]
        where, slot = torch.tensor(where, device=DEV), torch.tensor(slot, device=DEV)
        for c in range(m):
            out_k[-1, where, c, slot], out_v[-1, where, c, slot] = k[:, c], v[:, c]
        return rotate(q), out_k, out_v
    out = torch.zeros(bounds[-1], h, d, dtype=torch.float64, device=DEV)
    for i, (t, n) in enumerate(zip(total, news)):
        if t == 0:
            continue
        q = s["q"][bounds[i]:bounds[i + 1]].double()
        if kind == "prompt":
            k, v = s["k"][bounds[i]:bounds[i + 1]].double(), s["v"][bounds[i]:bounds[i + 1]].double()
        else:
            ids = s["table"][i, : -(-t // page)].long()
            k, v = (c[-1].view(torch.uint8)[ids].view(c.dtype).double().transpose(1, 2).reshape(-1, m, d)[:t] for c in (s["k_cache"], s["v_cache"]))
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][-1].double()[:, None], v * s["v_scale"][-1].double()[:, None]
        after = torch.arange(t, device=DEV)[None] > (torch.arange(n, device=DEV) + t - n)[:, None]
        for c in range(h):
            e = (q[:, c] @ k[:, c // group].t() / math.sqrt(d)).masked_fill(after, -math.inf)
            out[bounds[i]:bounds[i + 1], c] = torch.softmax(e, -1) @ v[:, c // group]
    return out
