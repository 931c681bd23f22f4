"""The cache in blocks (e4m3 codes, an exponent for each block of 16 tokens and head): writing it and reading it back bit by bit, the
attention over it against row-by-row fp64 references.  References: oracle/blocks_oracle.py, oracle/attn_oracle.py."""
import random

import numpy as np
import pytest
import torch

import paper_2406_09041_amd as mes
from oracle import attn_oracle as O
from oracle import blocks_oracle as BO
from test_gpu_attn import DEV, INF, NAN, _check, _ints, _rows

pytestmark = pytest.mark.gpu


def _offsets(counts):
    off = [0]
    for n in counts:
        off.append(off[-1] + n)
    return off


def _exponents(x):
    return x.view(torch.uint8).cpu().int() - 127


def _same(cache, layer, want, which, what=""):
    """All of a layer's codes and exponents."""
    got = getattr(cache, which)[layer].cpu().double().numpy()
    e = _exponents(getattr(cache, which + "_scale")[layer]).numpy()
    assert np.array_equal(e, want.e), f"{what} {which}: exponents differ at {np.argwhere(e != want.e)[:3].tolist()}"
    assert np.array_equal(got, want.code, equal_nan=True), f"{what} {which}: codes differ at {np.argwhere((got != want.code) & ~(np.isnan(got) & np.isnan(want.code)))[:3].tolist()}"


class Written:
    """A cache that is written call by call, on both sides."""

    def __init__(self, seqs, heads, kvh, dim, page, n_pages=None, layers=2, layer=1, dims=None, interleaved=False, width=8, seed=1):
        self.rng, self.g = random.Random(seed), torch.Generator().manual_seed(seed)
        self.heads, self.kvh, self.dim, self.page, self.layer, self.width = heads, kvh, dim, page, layer, width
        n_pages = n_pages or seqs * width + 3
        ids = self.rng.sample(range(n_pages), n_pages)
        self.pages = [[ids.pop() for _ in range(width)] for _ in range(seqs)]
        self.cache = mes.KvCache(layers, n_pages, page, kvh, dim, mes.KV_E4M3_BLOCKS)
        self.k, self.v = BO.Blocks(n_pages, kvh, page, dim), BO.Blocks(n_pages, kvh, page, dim)
        self.length = [0] * seqs
        self.table = mes.mes_rotary_table(width * page, dims or dim)
        self.angles, self.interleaved = mes.Angles(self.table, interleaved=interleaved), interleaved

    def batch(self, news):
        return mes.SeqBatch(_ints(self.length), _ints(self.pages), _ints(_offsets(news)))

    def append(self, news, k=None, v=None, behind=0):
        off = _offsets(news)
        T = off[-1] + behind
        q = _rows(self.g, T, self.heads, self.dim)
        size = torch.exp2(torch.randint(-6, 7, (T, 1, 1), generator=self.g).float())
        k = (_rows(self.g, T, self.kvh, self.dim) * size).to(torch.bfloat16) if k is None else k
        v = (_rows(self.g, T, self.kvh, self.dim) / size).to(torch.bfloat16) if v is None else v
        begin = list(self.length)
        self.length = [a + n for a, n in zip(self.length, news)]
        at = [begin[s] + i for s, n in enumerate(news) for i in range(n)]
        turned = [BO.turn(x[:off[-1]], self.table.cpu(), at, self.interleaved) for x in (q, k)]
        for s, n in enumerate(news):
            if n:
                self.k.put(self.pages[s], begin[s], turned[1][off[s]:off[s + 1]].numpy())
                self.v.put(self.pages[s], begin[s], v[off[s]:off[s + 1]].float().numpy())
        out = mes.mes_kv_append(self.cache, self.layer, self.batch(news), q.to(DEV), k.to(DEV), v.to(DEV), self.angles)
        assert torch.equal(out[:off[-1]].cpu(), turned[0].to(torch.bfloat16)) and not out[off[-1]:].any()
        self.check()
        return q

    def check(self, what=""):
        _same(self.cache, self.layer, self.k, "k", what)
        _same(self.cache, self.layer, self.v, "v", what)
        other = 1 - self.layer
        assert not self.cache.k.view(torch.uint8)[other].any() and torch.all(self.cache.v_scale.view(torch.uint8)[other] == 10)


APPENDS = [  # calls, one after the other: new tokens of each sequence
    ([[1], [1], [14], [1], [1], [40]], 4, 2, 64, 16, None, False), ([[5, 0, 33], [1, 1, 1], [20, 16, 0], [1, 1, 1]], 4, 1, 128, 32, 64, True),
    ([[17, 3], [31, 100], [2, 1]], 5, 5, 128, 64, 128, False), ([[100], [27], [3]], 8, 8, 64, 128, 16, True), ([[1] * 9] * 3, 4, 4, 128, 16, 96, False),
    ([[16], [16], [8], [8], [7], [9]], 2, 1, 64, 256, 48, False),
]


@pytest.mark.parametrize("calls,heads,kvh,dim,page,dims,interleaved", APPENDS)
def test_append(calls, heads, kvh, dim, page, dims, interleaved):
    """Every code and exponent of the layer after every call, sizes of tokens over 12 powers of two."""
    w = Written(len(calls[0]), heads, kvh, dim, page, dims=dims, interleaved=interleaved, seed=len(calls) + dim)
    for news in calls:
        w.append(news, behind=2)


def test_append_of_values_out_of_the_ordinary():
    """Infinities become the largest code, NaN stays and neither counts for the exponent; the type's largest and smallest values, zeros."""
    dim, kvh = 64, 2
    w = Written(1, 2, kvh, dim, 16, seed=9, dims=16)
    w.table.zero_()
    w.table[:, 0] = 1.0                                          # nothing is turned
    big, tiny = 3.3895313892515355e38, 9.2e-41
    v = torch.zeros(64, kvh, dim)
    v[0, 0, :4] = torch.tensor([INF, -INF, 1.0, NAN])
    v[3, 0, 5] = -300.0
    v[16:18, 0, :3] = torch.tensor([big, -big, 2.0])             # the largest exponent: codes up to 240
    v[18, 0, 0] = INF
    v[16, 1, :3] = torch.tensor([tiny, -tiny, 1e-36])            # the least
    v[32, 0, :] = NAN
    v[33, 1, :2] = torch.tensor([INF, NAN])
    v[48, 0, 0], v[49, 0, 0], v[50, 0, 0] = 448.0, 448.0, -0.0
    v[51, 1, 0], v[52, 1, 1] = 450.0, 1e-3
    v = v.to(torch.bfloat16)
    w.append([64], k=v.clone(), v=v)
    got = mes.mes_kv_read(w.cache, 1, w.batch([64]), 64)[1].cpu().float()
    assert got[0, 0, :3].tolist() == [448.0, -448.0, 1.0] and got[0, 0, 3].isnan() and torch.isfinite(got[16:32]).all()
    # larger tokens behind them, one by one: the older codes follow, NaN as NaN
    w = Written(1, 2, kvh, dim, 16, seed=10, dims=16)
    for i, size in enumerate([1e-30, 1e-5, 1.0, NAN, 0.0, INF, 1e4, 3e38, 1.0, 2.0]):
        x = torch.full((1, kvh, dim), size)
        x[0, 0, 0], x[0, 1, 1] = 0.3, -0.0
        w.append([1], k=x.to(torch.bfloat16), v=(x * 0.7).to(torch.bfloat16))


def test_append_where_there_is_no_place():
    """Fewer tokens than rows, past the table's room, pages outside the cache, rows behind the last sequence: nothing else is touched."""
    kvh, dim, page = 2, 64, 16
    cache = mes.KvCache(1, 6, page, kvh, dim, mes.KV_E4M3_BLOCKS)
    pages = [[0, 1], [2, -1], [6, 3], [4, 5]]
    kv_len, news = [5, 20, 30, 40], [9, 10, 20, 12]              # rows before position 0; a page that is not there; as well; past the room of 32
    off, g = _offsets(news), torch.Generator().manual_seed(2)
    T = off[-1] + 3
    q, k, v = (_rows(g, T, h, dim) for h in (4, kvh, kvh))
    angles = mes.Angles(mes.mes_rotary_table(32, dim))
    want = [BO.Blocks(6, kvh, page, dim) for _ in range(2)]
    at = [n - m + i for n, m in zip(kv_len, news) for i in range(m)] + [None] * 3
    places = [p if p is not None and 0 <= p < 32 else None for p in at]
    turned = [BO.turn(x, angles.table.cpu(), places, False) for x in (q, k)]
    for s in range(4):
        rows = [i for i in range(off[s], off[s + 1]) if places[i] is not None]
        want[0].put(pages[s], places[rows[0]], turned[1][rows].numpy())
        want[1].put(pages[s], places[rows[0]], v[rows].float().numpy())
    batch = mes.SeqBatch(_ints(kv_len), _ints(pages), _ints(off))
    out = mes.mes_kv_append(cache, 0, batch, q.to(DEV), k.to(DEV), v.to(DEV), angles)
    assert torch.equal(out.cpu(), turned[0].to(torch.bfloat16))
    given = torch.full_like(out, 7.0)
    mes.mes_kv_append(cache, 0, batch, q.to(DEV), k.to(DEV), v.to(DEV), angles, given)
    there = torch.tensor([p is not None for p in places])
    assert torch.equal(given.cpu()[there], out.cpu()[there]) and torch.all(given.cpu()[~there] == 7.0)
    _same(cache, 0, want[0], "k")
    _same(cache, 0, want[1], "v")


def test_append_without_queries_or_angles_and_with_fused_rows():
    kvh, dim = 2, 128
    w = Written(2, 4, kvh, dim, 16, seed=3)
    g = torch.Generator().manual_seed(3)
    row = _rows(g, 21, 8, dim).to(DEV)
    off = [0, 20, 21]
    w.length = [20, 1]
    batch = mes.SeqBatch(_ints(w.length), _ints(w.pages), _ints(off))
    k, v = row[:, 4:6], row[:, 6:]
    mes.mes_kv_append(w.cache, 1, batch, None, k, v)
    for s in range(2):
        w.k.put(w.pages[s], 0, k[off[s]:off[s + 1]].float().cpu().numpy())
        w.v.put(w.pages[s], 0, v[off[s]:off[s + 1]].float().cpu().numpy())
    w.check()
    # in place, and one row per sequence without offsets
    q = row[:, :4]
    w.length = [21, 2]
    want = BO.turn(q[:2].cpu(), w.table.cpu(), [20, 1], False)
    turned = BO.turn(k[:2].cpu(), w.table.cpu(), [20, 1], False)
    mes.mes_kv_append(w.cache, 1, mes.SeqBatch(_ints(w.length), _ints(w.pages)), q[:2], k[:2], v[:2], w.table, q[:2])
    assert torch.equal(q[:2].cpu(), want.to(torch.bfloat16))
    for s in range(2):
        w.k.put(w.pages[s], w.length[s] - 1, turned[s:s + 1].numpy())
        w.v.put(w.pages[s], w.length[s] - 1, v[s:s + 1].float().cpu().numpy())
    w.check()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("interleaved,dims", [(True, 64), (False, 32), (True, 16)])
def test_append_to_the_other_caches_in_other_forms(dtype, interleaved, dims):
    g = torch.Generator().manual_seed(6)
    heads, kvh, dim, n = 4, 2, 64, 37
    scale = [0.01 + 0.02 * torch.rand(2, kvh, generator=g) for _ in range(2)] if dtype == "e4m3" else [None, None]
    cache = mes.KvCache(2, 5, 16, kvh, dim, mes.KV_E4M3 if dtype == "e4m3" else mes.KV_BF16, *[None if x is None else x.to(DEV) for x in scale])
    angles = mes.Angles(mes.mes_rotary_table(48, dims), interleaved=interleaved)
    q, k, v = (_rows(g, n, h, dim) for h in (heads, kvh, kvh))
    batch = mes.SeqBatch(_ints([n + 3]), _ints([[3, 0, 4]]), _ints([0, n]))
    out = mes.mes_kv_append(cache, 1, batch, q.to(DEV), k.to(DEV), v.to(DEV), angles)
    turned = [BO.turn(x, angles.table.cpu(), range(3, n + 3), interleaved) for x in (q, k)]
    assert torch.equal(out.cpu(), turned[0].to(torch.bfloat16))
    kk, vv = mes.mes_kv_read(cache, 1, batch, n)
    for x, got, s in ((turned[1], kk, scale[0]), (v.float(), vv, scale[1])):
        if s is None:
            want = x.to(torch.bfloat16)
        else:
            by = s[1][None, :, None]
            want = ((x / by).clamp(-448, 448).to(torch.float8_e4m3fn).float() * by).to(torch.bfloat16)
        assert torch.equal(got.cpu(), want)


# ------------------------------------------------------------------------------------------------------- reading back

class Random:
    """A cache of blocks with random codes and exponents, on both sides; pages in random order, unused ones full of NaN, tokens behind a
    sequence's end as well."""

    def __init__(self, seed, lens, kvh, dim, page, layers=2, layer=1, spare=2, width=None, share=None, least=118, most=124):
        g, rng = torch.Generator().manual_seed(seed), random.Random(seed)
        self.lens, self.page, self.layer = lens, page, layer
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + spare
        ids = rng.sample(range(self.n_pages), self.n_pages)
        self.width = width or max(need + [1])
        table = [[ids.pop() for _ in range(n)] for n in need]
        self.table = [row + [0] * (self.width - len(row)) for row in table]
        shape = (layers, self.n_pages, kvh, page, dim)
        code = [torch.full(shape, 0x7f, dtype=torch.uint8) for _ in range(2)]
        e = [torch.full((*shape[:3], page // 16), 255, dtype=torch.uint8) for _ in range(2)]
        self.values = [[], []]
        for s, n in enumerate(lens):
            first, common = (share or {}).get(s, (s, 0))
            for x in range(2):
                c = (torch.randn(n, kvh, dim, generator=g) * 90).clamp(-448, 448).to(torch.float8_e4m3fn)
                p = torch.randint(least, most, (-(-n // 16), kvh), generator=g, dtype=torch.uint8)
                if first != s:
                    c.view(torch.uint8)[:common] = self.codes[first][x].view(torch.uint8)[:common]
                    p[:-(-common // 16)] = self.powers[first][x][:-(-common // 16)]
                if x == 0:
                    self.__dict__.setdefault("codes", []).append([])
                    self.__dict__.setdefault("powers", []).append([])
                self.codes[s].append(c)
                self.powers[s].append(p)
                for j in range(n):
                    code[x][layer, table[s][j // page], :, j % page] = c[j].view(torch.uint8)
                    e[x][layer, table[s][j // page], :, j % page // 16] = p[j // 16]
                by = torch.exp2(p.double() - 127).repeat_interleave(16, 0)[:n]
                self.values[x].append(c.double() * by[:, :, None])
        self.k, self.v = self.values
        self.cache = mes.KvCache.over(*[c.to(DEV).view(torch.float8_e4m3fn) for c in code], *[p.to(DEV).view(torch.float8_e8m0fnu) for p in e])

    def batch(self, offsets=None, kv_len=None, table=None):
        return mes.SeqBatch(_ints(self.lens if kv_len is None else kv_len), _ints(self.table if table is None else table).reshape(len(self.lens), self.width),
                            None if offsets is None else _ints(offsets))


@pytest.mark.parametrize("lens,news,kvh,dim,page", [([1], [1], 2, 64, 16), ([40, 0, 300, 17], [40, 0, 130, 17], 2, 128, 32), ([129] * 3, [1, 128, 64], 5, 64, 256)])
def test_read(lens, news, kvh, dim, page):
    c = Random(sum(lens), lens, kvh, dim, page)
    off = _offsets(news)
    k, v = mes.mes_kv_read(c.cache, 1, c.batch(off), off[-1] + 2)
    assert not k[off[-1]:].any() and not v[off[-1]:].any()
    for s, n in enumerate(news):
        for got, want in ((k, c.k), (v, c.v)):
            assert torch.equal(got[off[s]:off[s + 1]].double().cpu(), want[s][lens[s] - n:])
    # into rows of one buffer, one of the two alone, rows behind as they are
    wide = torch.full((off[-1] + 2, 2 * kvh + 1, dim), 7.0, dtype=torch.bfloat16, device=DEV)
    mes.mes_kv_read(c.cache, 1, c.batch(off), off[-1] + 2, wide[:, :kvh], wide[:, kvh:2 * kvh])
    assert torch.equal(wide[:off[-1], :kvh], k[:off[-1]]) and torch.equal(wide[:off[-1], kvh:2 * kvh], v[:off[-1]])
    assert torch.all(wide[:, -1] == 7.0) and torch.all(wide[off[-1]:] == 7.0)
    alone = torch.empty_like(k)
    assert mes.mes_kv_read(c.cache, 1, c.batch(off), off[-1], None, alone[:off[-1]])[0] is None
    assert torch.equal(alone[:off[-1]], v[:off[-1]])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "blocks"])
def test_read_where_there_is_nothing(dtype):
    from test_gpu_attn import Paged
    lens, dim, kvh = [100, 64, 50, 96], 64, 2
    c = Random(3, lens, kvh, dim, 16) if dtype == "blocks" else Paged(3, lens, kvh, dim, 16, dtype == "e4m3")
    off, kv_len = [0, 130, 140, 150, 200], [100, -5, 50, 150]
    table = [list(r) for r in c.table]
    table[2][1], table[2][3] = c.n_pages, -1
    table = [r[:6] for r in table]                               # room for 96 tokens
    c.width = 6
    k, v = mes.mes_kv_read(c.cache, c.layer, c.batch(off, kv_len, table), 200)
    for got, want in ((k.cpu(), c.k), (v.cpu(), c.v)):
        assert not got[:30].any() and torch.equal(got[30:126], want[0][:96].to(torch.bfloat16)) and not got[126:140].any()
        for i in range(10):
            there = (40 + i) // 16 not in (1, 3)
            assert torch.equal(got[140 + i], want[2][40 + i].to(torch.bfloat16) if there else torch.zeros(kvh, dim, dtype=torch.bfloat16))
        assert not got[150:200].any()


def test_exponents_outside_those_that_are_written():
    """Bytes below 10 and above 247 count as these."""
    c = Random(5, [80], 1, 64, 16)
    for x in (c.cache.k_scale, c.cache.v_scale):
        b = x.view(torch.uint8)
        for i, value in enumerate([0, 9, 10, 247, 248]):
            b[1, c.table[0][i]] = value
    c.cache.k.view(torch.uint8)[1] &= 0xb7                       # codes below 240
    k, _ = mes.mes_kv_read(c.cache, 1, c.batch([0, 80]), 80)
    code = c.cache.k[1, c.table[0]].cpu().double().transpose(1, 2).reshape(80, 1, 64)
    by = torch.exp2(torch.tensor([-117.0, -117, -117, 120, 120], dtype=torch.float64)).repeat_interleave(16)[:, None, None]
    assert torch.equal(k.double().cpu(), code * by)


# ---------------------------------------------------------------------------------------------------------- attention

EXTENDS = [
    ([1], [1], 4, 2, 64, 16), ([40], [40], 2, 1, 128, 16), ([300], [1], 4, 2, 128, 32), ([300, 64, 17], [130, 64, 1], 4, 2, 64, 16),
    ([129, 0, 200], [1, 0, 200], 2, 2, 128, 64), ([77, 500], [70, 129], 8, 1, 64, 256), ([20] * 66, [3] * 66, 2, 1, 64, 16), ([4400], [70], 4, 1, 64, 16),
]


@pytest.mark.parametrize("lens,news,heads,kvh,dim,page", EXTENDS)
def test_extend(lens, news, heads, kvh, dim, page):
    c = Random(len(lens) * 7 + lens[0], lens, kvh, dim, page)
    g, off = torch.Generator().manual_seed(9), _offsets(news)
    q = _rows(g, off[-1] + 2, heads, dim, 2.0)
    out = torch.full((off[-1] + 2, heads, dim), 7.0, dtype=torch.bfloat16, device=DEV)
    mes.mes_attn_extend(c.cache, c.layer, c.batch(off), q.to(DEV), out)
    torch.cuda.synchronize()
    assert torch.all(out[off[-1]:] == 7.0)
    for s in range(len(lens)):
        if news[s]:
            rows = sorted(set(range(0, news[s], 5)) | {news[s] - 1})
            pick = [off[s] + r for r in rows]
            want, tol = O.attend(q[pick], c.k[s], c.v[s], [lens[s] - news[s] + r for r in rows], dim ** -0.5)
            _check(out[pick], want, tol, f"sequence {s}")


def test_extend_with_lengths_and_pages_that_do_not_fit():
    lens, dim, heads, kvh = [100, 64, 50, 96], 64, 4, 2
    c = Random(3, lens, kvh, dim, 16)
    g = torch.Generator().manual_seed(2)
    off, kv_len = [0, 130, 140, 150, 200], [100, -5, 50, 150]
    table = [list(r) for r in c.table]
    table[2][1], table[2][3] = c.n_pages, -1
    table = [r[:6] for r in table]
    c.width = 6
    q = _rows(g, 200, heads, dim, 2.0)
    out = mes.mes_attn_extend(c.cache, c.layer, c.batch(off, kv_len, table), q.to(DEV)).cpu()
    assert not out[:30].any() and not out[130:140].any()
    want, tol = O.attend(q[30:130], c.k[0][:96], c.v[0][:96], range(100), dim ** -0.5)
    _check(out[30:130], want, tol, "longer than the table")
    there = [j for j in range(50) if j // 16 not in (1, 3)]
    for i in range(10):
        seen = [x for x, j in enumerate(there) if j <= 40 + i]
        want, tol = O.attend(q[140 + i:141 + i], c.k[2][there], c.v[2][there], [len(seen) - 1], dim ** -0.5)
        _check(out[140 + i:141 + i], want, tol, "pages missing")
    want, tol = O.attend(q[150:200], c.k[3], c.v[3], [min(100 + i, 95) for i in range(50)], dim ** -0.5)
    _check(out[150:200], want, tol, "positions past the table")


DECODES = [  # lens, heads, kvh, dim, page, (segments, prefixes)
    ([1], 4, 2, 64, 16, None), ([0], 2, 2, 128, 16, None), ([200], 32, 8, 128, 16, None), ([127, 33, 0, 400, 512], 8, 2, 128, 32, None),
    ([127, 128, 0, 1000, 1, 31, 32, 33], 4, 2, 64, 64, None), ([2100, 5, 300], 16, 1, 128, 16, None), ([8300, 17], 4, 4, 64, 128, None),
    ([90, 300], 34, 2, 128, 16, None), ([700] * 3, 64, 1, 64, 256, None), ([150, 33, 400, 290], 4, 2, 64, 16, None), ([500, 129], 12, 4, 64, 32, None),
    ([400, 200, 300, 250, 10], 40, 2, 128, 32, ([0, 5], [190])),                # own parts and the prefix in the larger body
    ([300, 170, 151, 150, 149, 3, 0], 8, 2, 128, 16, ([0, 7], [150])), ([100] * 20 + [60, 9], 8, 2, 64, 32, ([0, 20, 22], [64, 5])),
    ([350, 400, 330, 90, 80, 70, 1], 32, 8, 128, 64, ([0, 3, 3, 6, 7], [321, 9, 17, 1])), ([1300, 1290], 4, 1, 128, 16, ([0, 2], [1281])),
]


@pytest.mark.parametrize("lens,heads,kvh,dim,page,shared", DECODES)
def test_decode(lens, heads, kvh, dim, page, shared):
    n, share = len(lens), {}
    if shared:
        for e, common in enumerate(shared[1]):
            mine = [s for s in range(shared[0][e], shared[0][e + 1]) if lens[s] >= common]
            share.update({s: (mine[0], common) for s in mine})
    c = Random(n + lens[0], lens, kvh, dim, page, share=share)
    q = _rows(torch.Generator().manual_seed(24), n, heads, dim, 2.0)
    out = mes.AttnDecode(c.cache, heads, n)(c.layer, c.batch(), q.to(DEV), *(shared or (None, None)))
    again = mes.AttnDecode(c.cache, heads, n)(c.layer, c.batch(), q.to(DEV), *(shared or (None, None)))
    assert torch.equal(out, again)
    for s, m in enumerate(lens):
        want, tol = O.attend(q[s:s + 1], c.k[s], c.v[s], [m - 1], dim ** -0.5)
        _check(out[s:s + 1], want, tol, f"sequence {s}")


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "blocks"])
def test_a_large_batch_by_sampled_rows(kind):
    """Lengths over two powers of ten, experts of many and few sequences, with and without prefixes, ended sequences: rows whose pieces are cut over
    many wavefronts, that are one wavefront's, that end with their prefix."""
    from test_gpu_attn import Paged
    rng = random.Random(5)
    segs, prefix = [60, 31, 9, 3, 2, 1, 0, 54], [700, 333, 512, 1600, 64, 900, 9, 0]
    bounds, lens, share = _offsets(segs), [], {}
    for e, n in enumerate(segs):
        for i in range(n):
            own = rng.choice([0, 1, 31, 32, rng.randint(1, 60), rng.randint(1, 400), rng.randint(1, 2500)])
            lens.append(rng.choice([0, prefix[e] // 2] + [prefix[e] + own] * 8))
        mine = [s for s in range(bounds[e], bounds[e + 1]) if lens[s] >= prefix[e]]
        share.update({s: (mine[0], prefix[e]) for s in mine if prefix[e]})
    heads, kvh, dim, n = 8, 2, 128, len(lens)
    lens[130] = 9000
    if kind == "blocks":
        c = Random(3, lens, kvh, dim, 16, layers=1, layer=0, share=share)
    else:
        c = Paged(3, lens, kvh, dim, 16, kind == "e4m3", layers=1, layer=0, share=[share.get(s, (s, 0)) for s in range(n)])
    q = _rows(torch.Generator().manual_seed(24), n, heads, dim, 2.0)
    call = mes.AttnDecode(c.cache, heads, n)
    call.ws.fill_(255)
    out = call(0, c.batch(), q.to(DEV), bounds, prefix)
    alone = call(0, c.batch(), q.to(DEV))                        # nothing shared
    for s in sorted({0, 1, 59, 60, 75, 95, 100, 101, 103, 105, 106, 130, n - 1} | set(rng.sample(range(n), 30))):
        want, tol = O.attend(q[s:s + 1], c.k[s], c.v[s], [lens[s] - 1], dim ** -0.5)
        _check(out[s:s + 1], want, tol, f"sequence {s} of {lens[s]}")
        _check(alone[s:s + 1], want, tol, f"sequence {s} of {lens[s]}, nothing shared")
    assert torch.isfinite(out).all() and torch.isfinite(alone).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "blocks"])
@pytest.mark.parametrize("heads,kvh,dim", [(4, 2, 64), (12, 3, 128), (16, 1, 64), (2, 2, 128)])
def test_short_sequences_without_a_join(kind, heads, kvh, dim):
    """Up to 512 tokens: one workgroup per sequence and key / value head, one to four steps of each of its wavefronts."""
    from test_gpu_attn import Paged
    lens = [512, 150, 33, 400, 290, 0, 1, 129, 257]
    c = Random(6, lens, kvh, dim, 32) if kind == "blocks" else Paged(6, lens, kvh, dim, 32, kind == "e4m3")
    q = _rows(torch.Generator().manual_seed(7), len(lens), heads, dim, 2.0)
    out = mes.AttnDecode(c.cache, heads, len(lens))(c.layer, c.batch(), q.to(DEV))
    for s, n in enumerate(lens):
        want, tol = O.attend(q[s:s + 1], c.k[s], c.v[s], [n - 1], dim ** -0.5)
        _check(out[s:s + 1], want, tol, f"{n} tokens")


@pytest.mark.parametrize("kind", ["bf16", "blocks"])
def test_long_pieces_of_wavefronts(kind):
    """So many long sequences that a wavefront takes more than the 32 steps whose pages it looks up together; exponents of blocks far apart."""
    n, tokens, heads, kvh, dim, page = 64, 10000, 8, 4, 64, 128
    width = -(-tokens // page)
    g = torch.Generator(device=DEV).manual_seed(5)
    shape = (1, n * width, kvh, page, dim)
    if kind == "blocks":
        code = [(torch.randn(shape, generator=g, device=DEV) * 90).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2)]
        e = [torch.randint(117, 123, (*shape[:3], page // 16), generator=g, device=DEV, dtype=torch.uint8).view(torch.float8_e8m0fnu) for _ in range(2)]
        cache = mes.KvCache.over(*code, *e)
    else:
        cache = mes.KvCache.over(*[torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2)])
    table = torch.randperm(n * width, generator=g, device=DEV).to(torch.int32).reshape(n, width)
    kv_len = _ints([tokens - 37 * (s % 5) for s in range(n)])
    q = _rows(torch.Generator().manual_seed(6), n, heads, dim)
    out = mes.AttnDecode(cache, heads, n)(0, mes.SeqBatch(kv_len, table), q.to(DEV))
    assert torch.isfinite(out).all()
    for s in (0, 1, 17, 33, 63):
        m = int(kv_len[s])
        k, v = mes.mes_kv_read(cache, 0, mes.SeqBatch(kv_len[s:s + 1], table[s:s + 1], _ints([0, m])), m)
        want, tol = O.attend(q[s:s + 1], k.cpu(), v.cpu(), [m - 1], dim ** -0.5)
        _check(out[s:s + 1], want, tol, f"sequence {s}")


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "blocks"])
def test_rows_behind_contexts_of_many_lengths_by_sampled_rows(kind):
    """More items than compute units, the longest several times the mean: the call is cut, and its parts added up."""
    from test_gpu_attn import Paged
    contexts, news = [1024, 1024, 2040, 0, 1024, 77, 4096, 1024], [64, 700, 130, 333, 1, 17, 512, 250]
    lens, off, heads, kvh, dim = [a + b for a, b in zip(contexts, news)], _offsets(news), 16, 4, 64
    c = Random(4, lens, kvh, dim, 16) if kind == "blocks" else Paged(4, lens, kvh, dim, 16, kind == "e4m3")
    q = _rows(torch.Generator().manual_seed(2), off[-1], heads, dim, 2.0)
    out = mes.mes_attn_extend(c.cache, c.layer, c.batch(off), q.to(DEV))
    assert torch.isfinite(out).all()
    for s, n in enumerate(news):
        rows = sorted({0, n // 3, n // 2, n - 1})
        pick = [off[s] + r for r in rows]
        want, tol = O.attend(q[pick], c.k[s], c.v[s], [contexts[s] + r for r in rows], dim ** -0.5)
        _check(out[pick], want, tol, f"sequence {s}")


def test_decode_with_pages_that_are_not_there():
    lens, dim, heads, kvh = [600, 200], 128, 8, 2
    c = Random(8, lens, kvh, dim, 16)
    table = [list(r) for r in c.table]
    table[0][3], table[0][20], table[1][0] = -1, c.n_pages, 10 ** 9
    q = _rows(torch.Generator().manual_seed(4), 2, heads, dim, 2.0)
    out = mes.AttnDecode(c.cache, heads, 2)(c.layer, c.batch(table=table), q.to(DEV))
    for s, gone in enumerate([(3, 20), (0,)]):
        there = [j for j in range(lens[s]) if j // 16 not in gone]
        want, tol = O.attend(q[s:s + 1], c.k[s][there], c.v[s][there], [len(there) - 1], dim ** -0.5)
        _check(out[s:s + 1], want, tol, f"sequence {s}")


@pytest.mark.parametrize("least,most", [(10, 12), (100, 128), (10, 60)])
def test_attention_over_exponents_far_apart(least, most):
    """Keys of all sizes from 2^-117 codes up: a block's exponent is its own."""
    lens, heads, kvh, dim = [333], 4, 2, 128
    c = Random(11, lens, kvh, dim, 16, least=least, most=most)
    q = _rows(torch.Generator().manual_seed(4), 70, heads, dim, 0.05)
    out = mes.mes_attn_extend(c.cache, c.layer, c.batch([0, 70]), q.to(DEV))
    one = mes.AttnDecode(c.cache, heads, 1)(c.layer, c.batch(), q[69:].to(DEV))
    want, tol = O.attend(q, c.k[0], c.v[0], range(263, 333), dim ** -0.5)
    tol = tol + 2.0 ** -126                                      # outputs below the least normal value
    _check(out, want, tol)
    _check(one, want[69:], tol[69:])


@pytest.mark.parametrize("bad", ["code", "exponent"])
def test_rows_are_not_touched_by_what_they_do_not_see(bad):
    """NaN codes, or a largest exponent, in tokens behind a row's own: within its tile, its block and in later ones."""
    lens, heads, kvh, dim = [200, 90], 4, 2, 64
    c = Random(12, lens, kvh, dim, 16)
    q = _rows(torch.Generator().manual_seed(4), 60 + 30, heads, dim, 2.0)
    at = 165
    for x, e in ((c.cache.k, c.cache.k_scale), (c.cache.v, c.cache.v_scale)):
        if bad == "code":
            x.view(torch.uint8)[1, c.table[0][at // 16], 0, at % 16, 3] = 0x7f
        else:
            e.view(torch.uint8)[1, c.table[0][-1], 0] = 255          # the block of tokens 192 on
            at = 192
    out = mes.mes_attn_extend(c.cache, c.layer, c.batch([0, 60, 90]), q.to(DEV)).cpu()
    want, tol = O.attend(q[:60], c.k[0], c.v[0], range(140, 200), dim ** -0.5)
    _check(out[:at - 140], want[:at - 140], tol[:at - 140], "rows before it")
    _check(out[:60, 2:], want[:, 2:], tol[:, 2:], "heads beside it")
    want, tol = O.attend(q[60:], c.k[1], c.v[1], range(60, 90), dim ** -0.5)
    _check(out[60:], want, tol, "the other sequence")
    kv_len = [at, 90]
    one = mes.AttnDecode(c.cache, heads, 2)(c.layer, c.batch(kv_len=kv_len), q[:2].to(DEV)).cpu()
    for s in range(2):
        want, tol = O.attend(q[s:s + 1], c.k[s], c.v[s], [kv_len[s] - 1], dim ** -0.5)
        _check(one[s:s + 1], want, tol, f"decode {s}")


# --------------------------------------------------------------------------------------------------------- together

def test_a_run_of_them_with_forks_and_copies():
    """Prompts, decode steps, a fork, copies on the first write, compaction and reading back, as a serving loop makes them; the reference
    keeps what the cache holds by the definition."""
    heads, kvh, dim, page, layers = 8, 2, 64, 32, 2
    pool = mes.PagePool(24, page, 4, 6)
    cache = mes.KvCache(layers, 24, page, kvh, dim, mes.KV_E4M3_BLOCKS)
    want = [[BO.Blocks(24, kvh, page, dim) for _ in range(2)] for _ in range(layers)]
    angles = mes.Angles(mes.mes_rotary_table(6 * page, 32, scaling="bands", factor=2.0, context=64), interleaved=True)
    g = torch.Generator().manual_seed(8)
    decode = mes.AttnDecode(cache, heads, 4)

    def copy(src, dst):
        mes.mes_kv_copy_pages(cache, src, dst)
        for pair in want:
            for x in pair:
                for a, b in zip(src, dst):
                    x.code[b], x.e[b] = x.code[a], x.e[a]

    def step(seqs, news, prefix=None):
        copy(*pool.grow(seqs, news))
        table, length = pool.table(seqs)
        off = _offsets(news)
        batch = mes.SeqBatch(length.to(DEV), table.to(DEV), _ints(off))
        for layer in range(layers):
            q, k, v = (_rows(g, off[-1], h, dim) for h in (heads, kvh, kvh))
            at = [int(n) - m + i for n, m in zip(length, news) for i in range(m)]
            turned = [BO.turn(x, angles.table.cpu(), at, True) for x in (q, k)]
            for s, m in enumerate(news):
                for x, rows in zip(want[layer], (turned[1].numpy(), v.float().numpy())):
                    x.put(table[s].tolist(), int(length[s]) - m, rows[off[s]:off[s + 1]])
            qr = mes.mes_kv_append(cache, layer, batch, q.to(DEV), k.to(DEV), v.to(DEV), angles)
            if max(news) == 1:
                out = decode(layer, batch, qr, *([0, len(seqs)], [prefix]) if prefix else (None, None))
            else:
                out = mes.mes_attn_extend(cache, layer, batch, qr)
            for s, m in enumerate(news):
                vals = [x.values(table[s].tolist(), int(length[s])) for x in want[layer]]
                ref, tol = O.attend(qr[off[s]:off[s + 1]].cpu(), *vals, range(int(length[s]) - m, int(length[s])), dim ** -0.5)
                _check(out[off[s]:off[s + 1]], ref, tol, f"layer {layer}, sequence {seqs[s]}")
        for layer in range(layers):
            _same(cache, layer, want[layer][0], "k")
            _same(cache, layer, want[layer][1], "v")

    step([0, 3], [45, 7])
    pool.fork(0, 1)
    pool.fork(0, 2, 40)                                           # inside a block: its exponent is that of tokens that it has no more
    step([0, 1, 2], [1, 1, 1], prefix=40)
    step([0, 1, 2], [1, 1, 1], prefix=40)
    step([1, 3], [30, 60])
    pool.free(0)
    src, dst = pool.compact()
    copy(src, dst)
    step([1, 2, 3], [1, 1, 1])
    table, length = pool.table([1, 2, 3])
    n = [int(x) for x in length]
    k, v = mes.mes_kv_read(cache, 1, mes.SeqBatch(length.to(DEV), table.to(DEV), _ints(_offsets(n))), sum(n))
    for s, (a, b) in enumerate(zip(_offsets(n), _offsets(n)[1:])):
        for got, x in ((k, want[1][0]), (v, want[1][1])):
            assert torch.equal(got[a:b].double().cpu(), x.values(table[s].tolist(), n[s]))


@pytest.mark.parametrize("page,kvh", [(16, 2), (256, 3), (64, 5)])
def test_copies_take_the_exponents_along(page, kvh):
    dim, layers, n = 128, 3, 9
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randint(0, 256, (layers, n, kvh, page, dim), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2))
    ke, ve = (torch.randint(0, 256, (layers, n, kvh, page // 16), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2))
    want = [x.clone() for x in (k, v, ke, ve)]
    cache = mes.KvCache.over(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ke.view(torch.float8_e8m0fnu), ve.view(torch.float8_e8m0fnu))
    mes.mes_kv_copy_pages(cache, [0, 0, 7], [8, 3, 1])
    for x, y in zip((k, v, ke, ve), want):
        y[:, [8, 3, 1]] = y[:, [0, 0, 7]]
        assert torch.equal(x, y)


def test_a_captured_step_replayed_while_sequences_grow():
    """Writing, both attentions and reading in one graph, on a stream of its own, replayed with other lengths and rows; eager work between."""
    heads, kvh, dim, page, n = 8, 2, 128, 16, 5
    g = torch.Generator().manual_seed(2)
    caches = [mes.KvCache(1, 64, page, kvh, dim, mes.KV_E4M3_BLOCKS) for _ in range(2)]
    table = _ints([[i * 12 + j for j in range(12)] for i in range(n)])
    start = [30, 0, 100, 15, 47]
    angles = mes.Angles(mes.mes_rotary_table(192, dim))
    first = _rows(g, sum(start), 2 * kvh, dim).to(DEV)
    for c in caches:
        mes.mes_kv_append(c, 0, mes.SeqBatch(_ints(start), table, _ints(_offsets(start))), None, first[:, :kvh], first[:, kvh:], angles)
    kv_len = _ints(start)
    batch = mes.SeqBatch(kv_len, table, _ints(list(range(n + 1))))
    rows = torch.zeros(n, heads + 2 * kvh, dim, dtype=torch.bfloat16, device=DEV)
    decode = [mes.AttnDecode(c, heads, n) for c in caches]

    def step(c, d):
        kv_len.add_(1)
        q = mes.mes_kv_append(c, 0, batch, rows[:, :heads], rows[:, heads:heads + kvh], rows[:, heads + kvh:], angles)
        return [q, d(0, batch, q), mes.mes_attn_extend(c, 0, batch, q), *mes.mes_kv_read(c, 0, batch, n)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(caches[0], decode[0])
    kv_len.copy_(_ints(start))
    for i in range(4):
        rows.copy_(_rows(g, n, heads + 2 * kvh, dim) * 2 ** i)
        before = kv_len.clone()
        graph.replay()
        torch.cuda.synchronize()
        kv_len.copy_(before)
        want = step(caches[1], decode[1])
        for a, b in zip(got, want):
            assert torch.equal(a, b), i
        for a, b in ((caches[0].k, caches[1].k), (caches[0].v, caches[1].v), (caches[0].k_scale, caches[1].k_scale)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_offsets_past_32_bits():
    """Pages more than 2^32 bytes into a layer of keys: writing, reading and both attentions."""
    kvh, dim, page, heads = 8, 128, 256, 16
    n_pages = 17000                                               # 262144 bytes each
    cache = mes.KvCache(1, n_pages, page, kvh, dim, mes.KV_E4M3_BLOCKS)
    small = mes.KvCache(1, 2, page, kvh, dim, mes.KV_E4M3_BLOCKS)
    g = torch.Generator().manual_seed(3)
    q, k, v = (_rows(g, 300, h, dim).to(DEV) for h in (heads, kvh, kvh))
    angles = mes.Angles(mes.mes_rotary_table(512, dim))
    out = []
    for c, pages in ((cache, [n_pages - 1, n_pages - 9]), (small, [0, 1])):
        batch = mes.SeqBatch(_ints([300]), _ints([pages]), _ints([0, 300]))
        turned = mes.mes_kv_append(c, 0, batch, q, k, v, angles)
        one = mes.SeqBatch(_ints([300]), _ints([pages]))
        out.append([turned, mes.mes_attn_extend(c, 0, batch, turned), mes.AttnDecode(c, heads, 1)(0, one, turned[299:]), *mes.mes_kv_read(c, 0, batch, 300),
                    c.k_scale.view(torch.uint8)[0, pages], c.k.view(torch.uint8)[0, pages]])
    for a, b in zip(*out):
        assert torch.equal(a, b)
