"""Calls whose keys are shared out and such that are not, on both sides of the rule, by sampled rows; long items over pages of more than 64 tiles; offsets
out of order.  References and tolerances: oracle/attn_oracle.py."""
import pytest
import torch

import paper_2406_09041_amd as mes
from oracle import attn_oracle as O
from test_gpu_attn import DEV, Paged, _check, _ints, _rows
from test_gpu_blocks import Random, _offsets

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "e4m3", "blocks"]


def _cache(kind, seed, lens, kvh, dim, page):
    return Random(seed, lens, kvh, dim, page, layers=1, layer=0) if kind == "blocks" else Paged(seed, lens, kvh, dim, page, kind == "e4m3", layers=1, layer=0)


def _sampled(out, q, c, off, lens, news, rows_of, heads):
    for s, n in enumerate(news):
        rows = sorted(rows_of(n))
        pick = [off[s] + r for r in rows]
        want, tol = O.attend(q[pick], c.k[s], c.v[s], [lens[s] - n + r for r in rows], q.shape[2] ** -0.5)
        _check(out[pick], want, tol, f"sequence {s}")


@pytest.mark.parametrize("kind", KINDS)
def test_more_items_than_places_are_cut(kind):
    """528 items of 512 places, the longest with company: 32 heads over 8."""
    contexts, news = [1024, 1024, 2040, 0, 1024, 77, 4096, 1024], [64, 700, 130, 333, 1, 17, 512, 250]
    lens, off, heads, kvh, dim = [a + b for a, b in zip(contexts, news)], _offsets(news), 32, 8, 64
    c = _cache(kind, 4, lens, kvh, dim, 16)
    q = _rows(torch.Generator().manual_seed(2), off[-1], heads, dim, 2.0)
    out = mes.mes_attn_extend(c.cache, c.layer, c.batch(off), q.to(DEV))
    assert torch.isfinite(out).all()
    _sampled(out, q, c, off, lens, news, lambda n: {0, n // 3, n - 1}, heads)


@pytest.mark.parametrize("kind", KINDS)
def test_long_items_that_are_not_cut(kind):
    """More than 64 sequences are never cut: pages and exponents of 64 tiles are looked up again while tiles are on their way."""
    lens, news, heads, kvh, dim = [9000] + [20] * 65 + [4200], [70] + [3] * 65 + [40], 4, 1, 64
    c, off = _cache(kind, 6, lens, kvh, dim, 16), _offsets(news)
    q = _rows(torch.Generator().manual_seed(3), off[-1], heads, dim, 2.0)
    out = mes.mes_attn_extend(c.cache, c.layer, c.batch(off), q.to(DEV))
    _sampled(out, q, c, off, lens, news, lambda n: {0, n // 2, n - 1}, heads)


@pytest.mark.parametrize("lens,heads,kvh,dim", [([5800], 8, 1, 128), ([4000], 16, 2, 128), ([2000, 500, 700, 300], 16, 2, 64), ([7000, 300], 4, 4, 64), ([3000], 12, 4, 64)])
def test_packed_prompts_on_both_sides_of_the_rule(lens, heads, kvh, dim):
    g, off = torch.Generator().manual_seed(sum(lens)), _offsets(lens)
    q, k, v = _rows(g, off[-1], heads, dim, 2.0), _rows(g, off[-1], kvh, dim), _rows(g, off[-1], kvh, dim)
    out = mes.mes_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), _ints(off))
    assert torch.isfinite(out).all()
    for a, b in zip(off, off[1:]):
        rows = sorted({0, (b - a) // 3, (b - a) // 2 + 1, b - a - 1})
        want, tol = O.attend(q[[a + r for r in rows]], k[a:b], v[a:b], rows, dim ** -0.5)
        _check(out[[a + r for r in rows]], want, tol, f"rows {a}..{b}")


@pytest.mark.parametrize("kind", ["packed", "bf16", "blocks"])
def test_offsets_out_of_order(kind):
    """They name more rows than the call has, in parts that the workspace has no room for: the call ends, and the next one is right."""
    heads, kvh, dim, T = 8, 1, 64, 6000
    g = torch.Generator().manual_seed(8)
    bad, good = [0, T] + [5000, 5300] * 31 + [5000], [0, T] + [T] * 63
    q, k, v = _rows(g, T, heads, dim, 2.0), _rows(g, T, kvh, dim), _rows(g, T, kvh, dim)
    dq, dk, dv = (x.to(DEV) for x in (q, k, v))
    out = torch.zeros_like(dq)
    if kind == "packed":
        call = lambda off: mes.mes_attn_prompt(dq, dk, dv, _ints(off), out)  # noqa: E731
    else:
        cache = mes.KvCache(1, T // 16, 16, kvh, dim, mes.KV_BF16 if kind == "bf16" else mes.KV_E4M3_BLOCKS)
        table = torch.arange(T // 16, dtype=torch.int32).repeat(64, 1)
        batch = lambda off: mes.SeqBatch(_ints([T] + [300] * 63), table.to(DEV), _ints(off))  # noqa: E731
        mes.mes_kv_append(cache, 0, mes.SeqBatch(_ints([T]), table[:1].to(DEV), _ints([0, T])), None, dk, dv)
        k, v = (x.cpu() for x in mes.mes_kv_read(cache, 0, mes.SeqBatch(_ints([T]), table[:1].to(DEV), _ints([0, T])), T))
        call = lambda off: mes.mes_attn_extend(cache, 0, batch(off), dq, out)  # noqa: E731
    call(bad)
    assert torch.isfinite(out).all()
    call(good)
    rows = [0, 1, 3000, 5100, T - 1]
    want, tol = O.attend(q[rows], k, v, rows, dim ** -0.5)
    _check(out[rows], want, tol)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("many", [0, 70])
def test_fewer_rows_than_the_offsets_name(kind, many):
    """The rows that are there are the first of their sequence's, with and without more than 64 sequences beside it: those of the whole call."""
    lens, news = [5] * many + [40, 900], [2] * many + [33, 300]
    heads, kvh, dim, T = 4, 2, 64, 2 * many + 33 + 130
    c, off = _cache(kind, 3, lens, kvh, dim, 16), _offsets(news)
    q = _rows(torch.Generator().manual_seed(3), off[-1], heads, dim, 2.0).to(DEV)
    whole = mes.mes_attn_extend(c.cache, c.layer, c.batch(off), q)
    some = mes.mes_attn_extend(c.cache, c.layer, c.batch(off), q[:T])
    for s in range(len(lens)):
        rows = [r for r in (0, 1, news[s] // 3, news[s] - 1) if off[s] + r < T]
        pick = [off[s] + r for r in rows]
        want, tol = O.attend(q[pick].cpu(), c.k[s], c.v[s], [lens[s] - news[s] + r for r in rows], dim ** -0.5)
        _check(whole[pick], want, tol, f"all rows, sequence {s}")
        _check(some[pick], want, tol, f"some rows, sequence {s}")
