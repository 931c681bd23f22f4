"""One token of few sequences against the cache: parts of equal length, the line of work behind them, and lengths that move from one to the other in a
captured graph.  References and tolerances: oracle/attn_oracle.py, for long sequences by sampled heads."""
import random

import pytest
import torch

import paper_2406_09041_amd as mes
from oracle import attn_oracle as O
from test_gpu_attn import DEV, Paged, _check, _ints, _rows
from test_gpu_blocks import Random

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "e4m3", "blocks"]


def _cache(kind, seed, lens, kvh, dim, page, **kw):
    return Random(seed, lens, kvh, dim, page, layers=1, layer=0, **kw) if kind == "blocks" else Paged(seed, lens, kvh, dim, page, kind == "e4m3", layers=1, layer=0, **kw)


def _right(c, lens, out, q, what=""):
    for s, n in enumerate(lens):
        want, tol = O.attend(q[s:s + 1], c.k[s], c.v[s], [n - 1], q.shape[2] ** -0.5)
        _check(out[s:s + 1], want, tol, f"{what} sequence {s} of {n}")


BATCHES = [  # lens, heads, kvh, dim, page
    ([0, 0, 0], 4, 2, 64, 64), ([1], 2, 1, 128, 16), ([513], 8, 1, 128, 32), ([128, 129, 127, 0, 256, 700], 4, 4, 64, 16),
    ([2000, 1], 32, 8, 128, 16), ([0, 9000, 0, 31], 16, 1, 64, 128), ([700] * 9, 12, 4, 64, 32), ([1500, 3, 600], 40, 40, 128, 64),
    ([33] * 63 + [1100], 2, 1, 64, 16), ([600, 0, 1, 40] * 17 + [900], 2, 2, 64, 16), ([520] + [3, 0, 70, 130] * 47, 3, 1, 64, 16),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,heads,kvh,dim,page", BATCHES)
def test_decode_of_few_sequences(lens, heads, kvh, dim, page, kind):
    """Up to 192 sequences and heads; page tables with room to spare, workspaces full of what others left."""
    width = max(-(-max(lens) // page), 0) + -(-600 // page)
    c = _cache(kind, len(lens) + sum(lens), lens, kvh, dim, page, width=width)
    q = _rows(torch.Generator().manual_seed(5), len(lens), heads, dim, 2.0)
    call = mes.AttnDecode(c.cache, heads, len(lens))
    out = []
    for fill in (0, 255):
        call.ws.fill_(fill)
        out.append(call(0, c.batch(), q.to(DEV)))
    assert torch.equal(*out)
    _right(c, lens, out[0], q)


@pytest.mark.parametrize("kind", KINDS)
def test_lengths_grow_in_a_captured_graph(kind):
    """From nothing over parts of every length to the line (more than 512 parts of 8 units) and back: the launches are the same."""
    full, heads, kvh, dim, page = [70000, 60000, 6000, 5000], 8, 4, 64, 256
    g = torch.Generator(device=DEV).manual_seed(5)
    width = -(-max(full) // page)
    shape = (1, len(full) * width, kvh, page, dim)
    if kind == "bf16":
        cache = mes.KvCache.over(*[torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2)])
    else:
        code = [(torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) * 90).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2)]
        scale = [torch.full((1, kvh), 2.0 ** -7, device=DEV) for _ in range(2)] if kind == "e4m3" else \
            [torch.randint(118, 122, (*shape[:3], page // 16), generator=g, device=DEV, dtype=torch.uint8).view(torch.float8_e8m0fnu) for _ in range(2)]
        cache = mes.KvCache.over(*code, *scale)
    table = torch.randperm(len(full) * width, generator=g, device=DEV).to(torch.int32).reshape(len(full), width)
    kv_len = _ints([0] * len(full))
    q = _rows(torch.Generator().manual_seed(6), len(full), heads, dim)
    dq, out = q.to(DEV), torch.empty(len(full), heads, dim, dtype=torch.bfloat16, device=DEV)
    call, batch = mes.AttnDecode(cache, heads, len(full)), mes.SeqBatch(kv_len, table)
    call(0, batch, dq, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0, batch, dq, out=out)
    rng = random.Random(3)
    for lens in ([0, 0, 0, 0], [1, 0, 300, 129], [16384, 1, 2, 3], [16385, 4097, 127, 128], full, [70000, 0, 0, 0], [9000, 8000, 6000, 5000], [5, 6, 7, 8]):
        kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        again = mes.AttnDecode(cache, heads, len(full))(0, batch, dq)
        assert torch.equal(out, again)
        for s, n in enumerate(lens):
            if n == 0:
                assert not out[s].any()
                continue
            k, v = mes.mes_kv_read(cache, 0, mes.SeqBatch(_ints([n]), table[s:s + 1].contiguous(), _ints([0, n])), n)
            h = rng.randrange(kvh)
            pick = slice(2 * h, 2 * h + 2)
            want, tol = O.attend(q[s:s + 1, pick], k[:, h:h + 1], v[:, h:h + 1], [n - 1], dim ** -0.5)
            _check(out[s:s + 1, pick], want, tol, f"sequence {s} of {n}")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,heads,kvh,dim,prefix", [(2, 8, 2, 128, 96), (2, 2, 2, 64, 640), (3, 4, 1, 64, 160), (16, 4, 4, 128, 2048), (4, 8, 2, 64, 1312)])
def test_a_shared_prefix_is_read_through_the_first_sequences_pages(n, heads, kvh, dim, prefix, kind):
    """However few share it: the others need not hold it."""
    lens = [prefix + 10 + 7 * s for s in range(n)]
    share = {s: (0, prefix) for s in range(n)} if kind == "blocks" else [(0, prefix)] * n
    c = _cache(kind, n + prefix, lens, kvh, dim, 32, share=share)
    for s in range(1, n):
        for x in (c.cache.k, c.cache.v):
            pages = torch.tensor(c.table[s][:prefix // 32], device=DEV)
            x.view(torch.uint8)[0, pages] = 0x7f                 # e4m3: NaN; bf16: 3.4e38
    q = _rows(torch.Generator().manual_seed(5), n, heads, dim)
    call = mes.AttnDecode(c.cache, heads, n)
    call.ws.fill_(255)
    _right(c, lens, call(0, c.batch(), q.to(DEV), [0, n], [prefix]), q)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,kvh,dim", [(8, 2, 64), (4, 4, 128), (14, 2, 128)])
def test_passes_of_few_and_of_many_rows(heads, kvh, dim, kind):
    """In one call: experts of two and three sequences, of twenty, of one; sequences shorter than their prefix, as long as it, ended ones."""
    segs, prefix = [3, 20, 2, 1, 2, 2], [3000, 100, 1500, 9, 700, 333]
    bounds, rng, lens, share = [0], random.Random(4), [], {}
    for e, n in enumerate(segs):
        bounds.append(bounds[-1] + n)
        mine = [prefix[e] + rng.choice([0, 1, 31, 400, 1300]) for _ in range(n)]
        if e == 1:
            mine[3], mine[4] = 0, 99
        if e == 4:
            mine[0] = 699                                        # one as long as the prefix: nothing is shared
        first = next((s for s, m in enumerate(mine) if m >= prefix[e]), None)
        share.update({len(lens) + s: (len(lens) + first, prefix[e]) for s, m in enumerate(mine) if m >= prefix[e]})
        lens += mine
    n = len(lens)
    c = _cache(kind, 9, lens, kvh, dim, 16, share=share if kind == "blocks" else [share.get(s, (s, 0)) for s in range(n)])
    q = _rows(torch.Generator().manual_seed(24), n, heads, dim, 2.0)
    call = mes.AttnDecode(c.cache, heads, n)
    out = []
    for fill in (0, 255):
        call.ws.fill_(fill)
        out.append(call(0, c.batch(), q.to(DEV), bounds, prefix))
    assert torch.equal(*out)
    _right(c, lens, out[0], q)
