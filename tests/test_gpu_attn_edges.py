"""Attention calls where values, scales or places are out of the ordinary: scales of the caller's own, an 8-bit cache's scales of any sign,
values that are not finite behind rows that do not see them and in front of rows that do, rows without a place, the type's largest
values.  References and tolerances: oracle/attn_oracle.py."""
import pytest
import torch

import paper_2406_09041_amd as mes
from oracle import attn_oracle as O
from test_gpu_attn import DEV, INF, NAN, Paged, _check, _ints, _rows

pytestmark = pytest.mark.gpu


def _offsets(counts):
    off = [0]
    for n in counts:
        off.append(off[-1] + n)
    return off


# ------------------------------------------------------------------------------------------------- a scale of the caller's

@pytest.mark.parametrize("scale", [0.004, 0.31, 3.0])
def test_scales_of_the_callers_own(scale):
    g = torch.Generator().manual_seed(12)
    heads, kvh, dim, lens = 4, 2, 64, [150, 33]
    q, k, v = _rows(g, 183, heads, dim), _rows(g, 183, kvh, dim), _rows(g, 183, kvh, dim)
    out = mes.mes_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), _ints([0, 150, 183]), scale=scale)
    for a, b in ((0, 150), (150, 183)):
        want, tol = O.attend(q[a:b], k[a:b], v[a:b], range(b - a), scale)
        _check(out[a:b], want, tol, f"prompt {a}..{b}")
    for e4m3 in (False, True):
        c = Paged(13, lens, kvh, dim, 16, e4m3)
        out = mes.mes_attn_extend(c.cache, c.layer, c.batch([0, 20, 22]), q[:22].to(DEV), scale=scale)
        each = mes.AttnDecode(c.cache, heads, 2)(c.layer, c.batch(), q[20:22].to(DEV), scale=scale)
        for s, (a, b) in enumerate(((0, 20), (20, 22))):
            want, tol = O.attend(q[a:b], c.k[s], c.v[s], range(lens[s] - (b - a), lens[s]), scale)
            _check(out[a:b], want, tol, f"extend, sequence {s}")
            want, tol = O.attend(q[20 + s:21 + s], c.k[s], c.v[s], [lens[s] - 1], scale)
            _check(each[s:s + 1], want, tol, f"decode, sequence {s}")


# ----------------------------------------------------------------------------------- an 8-bit cache's scales: any finite number

def _rescaled(c, k_scale, v_scale):
    """The same codes under other scales, one per key / value head."""
    for x, old, new, there in ((c.k, c.scales[0], k_scale, c.cache.k_scale), (c.v, c.scales[1], v_scale, c.cache.v_scale)):
        new = torch.tensor(new, dtype=torch.float32)
        for s, n in enumerate(c.lens):
            code = (x[s] / old[c.layer][:, None].double()).float().to(torch.float8_e4m3fn).double()
            x[s] = code * new[:, None].double()
        there[c.layer] = new.to(DEV)


# scales of keys and of values (two heads), and of the scores: 0, negative, and a product that is 0 in fp32
SCALES = [([0.0, -0.013], [0.02, -0.01], 0.125), ([-0.02, 0.015], [0.0, 0.02], 0.125), ([1e-30, -1e-30], [0.01, 0.02], 1e-20)]


@pytest.mark.parametrize("k_scale,v_scale,scale", SCALES)
@pytest.mark.parametrize("lens,news,heads,dim,page", [([300, 64, 17], [130, 64, 1], 4, 64, 16), ([129, 0, 77], [1, 0, 70], 2, 128, 64),
                                                      ([3000], [70], 8, 128, 16)])
def test_extend_with_scales_of_any_sign(lens, news, heads, dim, page, k_scale, v_scale, scale):
    c = Paged(21, lens, 2, dim, page, True)
    _rescaled(c, k_scale, v_scale)
    off = _offsets(news)
    q = _rows(torch.Generator().manual_seed(22), off[-1], heads, dim, 2.0)
    out = mes.mes_attn_extend(c.cache, c.layer, c.batch(off), q.to(DEV), scale=scale)
    for s in range(len(lens)):
        if news[s]:
            rows = sorted(set(range(0, news[s], 7)) | {news[s] - 1})
            pick = [off[s] + r for r in rows]
            want, tol = O.attend(q[pick], c.k[s], c.v[s], [lens[s] - news[s] + r for r in rows], scale)
            _check(out[pick], want, tol, f"sequence {s}")


@pytest.mark.parametrize("k_scale,v_scale,scale", SCALES)
@pytest.mark.parametrize("lens,heads,dim,prefix", [
    ([127, 33, 0, 400], 8, 128, None),                     # one workgroup per sequence
    ([127, 128, 0, 1000], 4, 64, None),                    # pieces
    ([90, 300], 34, 128, None),                            # more than 16 rows
    ([300] * 8 + [170, 3], 8, 128, 150)])                  # a shared prefix
def test_decode_with_scales_of_any_sign(lens, heads, dim, prefix, k_scale, v_scale, scale):
    n = len(lens)
    c = Paged(23, lens, 2, dim, 16, True, share=[(0 if m >= prefix else s, prefix) for s, m in enumerate(lens)] if prefix else None)
    _rescaled(c, k_scale, v_scale)
    q = _rows(torch.Generator().manual_seed(24), n, heads, dim, 2.0)
    out = mes.AttnDecode(c.cache, heads, n)(c.layer, c.batch(), q.to(DEV), [0, n] if prefix else None, [prefix] if prefix else None, scale=scale)
    for s, m in enumerate(lens):
        want, tol = O.attend(q[s:s + 1], c.k[s], c.v[s], [m - 1], scale)
        _check(out[s:s + 1], want, tol, f"sequence {s}")


def test_append_under_a_scale_of_zero():
    """What is 0 stays 0 (0 / 0 has no code), the rest is clamped: a head whose scale is 0 holds zeros, and rows that see it are finite."""
    heads, kvh, dim, n = 4, 2, 64, 40
    scale = [torch.tensor([[0.0, 0.02]], device=DEV) for _ in range(2)]
    cache = mes.KvCache(1, 4, 16, kvh, dim, mes.KV_E4M3, *scale)
    g = torch.Generator().manual_seed(25)
    q, k, v = (_rows(g, n, h, dim) for h in (heads, kvh, kvh))
    k[:, 0, ::2], v[:, 0, 1::2], k[3, 1, :], k[:, 0, 4] = 0.0, 0.0, 0.0, -0.0
    batch = mes.SeqBatch(_ints([n]), _ints([[2, 0, 1, 3]]), _ints([0, n]))
    mes.mes_kv_append(cache, 0, batch, None, k.to(DEV), v.to(DEV), None)
    kept = []
    for x, got in ((k, cache.k), (v, cache.v)):
        code = torch.where(x.float() == 0, torch.zeros(()), x.float() / scale[0].cpu()[0][None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn).float()
        got = got[0, [2, 0, 1]].cpu().float().transpose(1, 2).reshape(48, kvh, dim)[:n]
        assert torch.equal(got, code)
        kept.append(code.double() * scale[0].cpu()[0][None, :, None].double())
    out = mes.mes_attn_extend(cache, 0, batch, q.to(DEV))
    want, tol = O.attend(q, kept[0], kept[1], range(n), dim ** -0.5)
    _check(out, want, tol)


# --------------------------------------------------------------------------------------------- what is not finite, and not seen

def _spoil(c, which, s, j, head, d, bad):
    """Element d of token j of sequence s, in the cache only."""
    x = c.cache.k if which == "k" else c.cache.v
    if x.dtype == torch.float8_e4m3fn:
        x, bad = x.view(torch.uint8), 0x7f                                 # the type's NaN: it has no infinities
    x[c.layer, c.table[s][j // c.page], head, j % c.page, d] = bad


def _check_around(out, q, k, v, positions, scale, d, what):
    """Rows that see a value that is not finite in dimension d of v (a number in the reference): that dimension alone has it."""
    out = out.cpu()
    assert not torch.isfinite(out[:, :, d]).any(), what
    keep = [x for x in range(out.shape[2]) if x != d]
    want, tol = O.attend(q, k, v, positions, scale)
    _check(out[:, :, keep], want[:, :, keep], tol[:, :, keep], what)


@pytest.mark.parametrize("e4m3,bad", [(False, NAN), (False, INF), (False, -INF), (True, NAN)])
@pytest.mark.parametrize("heads,kvh,dim,page", [(2, 2, 128, 16), (4, 2, 64, 32), (4, 1, 128, 64), (8, 2, 64, 16)])
def test_extend_rows_are_not_touched_by_what_they_do_not_see(heads, kvh, dim, page, e4m3, bad):
    """A value that is not finite in a new token: earlier rows of the same tile, other heads and other sequences as without it; a page
    is missing before it."""
    lens, news, at = [260, 150], [130, 140], 200
    c = Paged(31, lens, kvh, dim, page, e4m3)
    table = [list(r) for r in c.table]
    table[0][64 // page] = -1
    gone = range(64 // page * page, 64 // page * page + page)
    off = _offsets(news)
    q = _rows(torch.Generator().manual_seed(32), off[-1], heads, dim)
    there = [j for j in range(lens[0]) if j not in gone]
    k0, v0 = c.k[0][there], c.v[0][there]
    group, scale, skip = heads // kvh, dim ** -0.5, lens[0] - len(there)
    for which in ("k", "v"):
        c = Paged(31, lens, kvh, dim, page, e4m3)
        _spoil(c, which, 0, at, 0, 5, bad)
        out = mes.mes_attn_extend(c.cache, c.layer, c.batch(off, None, table), q.to(DEV))
        first = at - (lens[0] - news[0])                                   # the first row that sees it
        want, tol = O.attend(q[:first], k0, v0, [130 + i - skip for i in range(first)], scale)
        _check(out[:first], want, tol, f"rows before it, {which}")
        want, tol = O.attend(q[130:], c.k[1], c.v[1], range(10, 150), scale)
        _check(out[130:], want, tol, f"the other sequence, {which}")
        rows = list(range(first, 130, 9))
        after = [130 + i - skip for i in rows]
        if kvh > 1:
            want, tol = O.attend(q[rows, group:], k0[:, 1:], v0[:, 1:], after, scale)
            _check(out[rows, group:], want, tol, f"other heads, {which}")
        if which == "v":
            _check_around(out[rows, :group], q[rows, :group], k0[:, :1], v0[:, :1], after, scale, 5, "rows that see it")
        elif bad != bad:
            assert torch.isnan(out[first:130, :group]).all()


@pytest.mark.parametrize("e4m3,bad", [(False, NAN), (False, INF), (True, NAN)])
@pytest.mark.parametrize("heads,dim", [(1, 128), (2, 64), (4, 128), (12, 64)])
def test_extend_with_keys_shared_out_and_a_value_that_is_not_finite(heads, dim, e4m3, bad):
    lens, news, at = [3000], [100], 2950
    c = Paged(33, lens, 1, dim, 16, e4m3)
    _spoil(c, "v", 0, at, 0, 5, bad)
    q = _rows(torch.Generator().manual_seed(34), 100, heads, dim)
    out = mes.mes_attn_extend(c.cache, c.layer, c.batch([0, 100]), q.to(DEV))
    rows = [0, 1, 31, 32, 48, 49]
    want, tol = O.attend(q[rows], c.k[0], c.v[0], [2900 + r for r in rows], dim ** -0.5)
    _check(out[rows], want, tol, "rows before it")
    rows = [50, 51, 63, 64, 99]
    _check_around(out[rows], q[rows], c.k[0], c.v[0], [2900 + r for r in rows], dim ** -0.5, 5, "rows that see it")


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("heads,kvh,dim,T", [(2, 1, 128, 1700), (1, 1, 64, 2500), (4, 1, 128, 1100)])
def test_prompt_with_keys_shared_out_and_a_value_that_is_not_finite(heads, kvh, dim, T, bad):
    g = torch.Generator().manual_seed(35)
    at = T - 200
    q, k, v = _rows(g, T, heads, dim), _rows(g, T, kvh, dim), _rows(g, T, kvh, dim)
    spoilt = v.clone()
    spoilt[at, 0, 5] = bad
    out = mes.mes_attn_prompt(q.to(DEV), k.to(DEV), spoilt.to(DEV), _ints([0, T]))
    rows = [0, 63, 64, 700, at - 130, at - 1]
    want, tol = O.attend(q[rows], k, v, rows, dim ** -0.5)
    _check(out[rows], want, tol, "rows before it")
    rows = [at, at + 1, at + 60, T - 1]
    _check_around(out[rows], q[rows], k, v, rows, dim ** -0.5, 5, "rows that see it")


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads,kvh,dim", [(4, 2, 128), (34, 2, 64), (17, 1, 128), (64, 1, 64)])
def test_decode_does_not_see_its_own_copy_of_a_shared_prefix(heads, kvh, dim, e4m3):
    """The prefix is read through the first sequence's pages: what the others hold in its place does not touch them (the last tokens of the
    prefix lie in the tile that their own part begins in)."""
    lens, prefix = [200, 210, 160, 170], 100
    c = Paged(36, lens, kvh, dim, 16, e4m3, share=[(0, prefix)] * 4)
    for s, which, j in ((1, "v", 64), (2, "v", 99), (3, "k", 97)):
        _spoil(c, which, s, j, 0, 7, NAN)
    q = _rows(torch.Generator().manual_seed(37), 4, heads, dim)
    out = mes.AttnDecode(c.cache, heads, 4)(c.layer, c.batch(), q.to(DEV), [0, 4], [prefix])
    for s, n in enumerate(lens):
        want, tol = O.attend(q[s:s + 1], c.k[s], c.v[s], [n - 1], dim ** -0.5)
        _check(out[s:s + 1], want, tol, f"sequence {s}")


@pytest.mark.parametrize("lens,heads,kvh,prefix,at", [([2000], 4, 2, None, 1990), ([2000, 1900], 34, 2, None, 1890), ([3000] * 3, 8, 8, None, 2999),
                                                      ([200, 210, 160], 34, 2, 100, 80), ([200, 210, 160], 34, 2, 100, 150), ([1200, 1300], 8, 2, 1000, 990)])
def test_decode_rows_that_see_an_infinite_value_are_infinite(lens, heads, kvh, prefix, at):
    """sum w_j v_j with one v_j = inf and weights above 0 is inf, not NaN, however the tokens are cut into pieces."""
    dim, n = 128, len(lens)
    c = Paged(38, lens, kvh, dim, 16, share=[(0, prefix)] * n if prefix else None)
    for s in range(n):
        _spoil(c, "v", s, at, 0, 7, INF)
    q = _rows(torch.Generator().manual_seed(39), n, heads, dim, 0.5)
    out = mes.AttnDecode(c.cache, heads, n)(c.layer, c.batch(), q.to(DEV), [0, n] if prefix else None, [prefix] if prefix else None).cpu()
    group = heads // kvh
    assert (out[:, :group, 7] == INF).all()
    out[:, :group, 7] = 0.0
    for s, m in enumerate(lens):
        want, tol = O.attend(q[s:s + 1], c.k[s], c.v[s], [m - 1], dim ** -0.5)
        want[:, :group, 7] = 0.0
        _check(out[s:s + 1], want, tol, f"sequence {s}")


# ------------------------------------------------------------------------------------------------------ rows without a place

def test_turned_queries_of_rows_without_a_position():
    """A q_out that the call allocates holds zeros for rows that have no position or no sequence, whatever was in its memory; the other
    rows are turned, also those whose page is outside the cache."""
    heads, kvh, dim, page, T = 4, 2, 64, 16, 30
    g = torch.Generator().manual_seed(40)
    cache = mes.KvCache(1, 6, page, kvh, dim)
    rotary = mes.rotary_table(2 * page, dim)
    q, k, v = (_rows(g, T, h, dim).to(DEV) for h in (heads, kvh, kvh))
    #  rows 0..9 of a sequence of 6 tokens (4 have no position), 10..19 of one longer than the table, 20..25 on no page; 26..29: no sequence
    batch = mes.SeqBatch(_ints([6, 37, 6]), _ints([[0, 1], [2, 3], [-1, 6]]), _ints([0, 10, 20, 26]))
    for _ in range(3):
        stale = torch.full((T, heads, dim), NAN, dtype=torch.bfloat16, device=DEV)
        del stale                                                      # its memory is the next tensor's
        out = mes.mes_kv_append(cache, 0, batch, q, k, v, rotary).cpu()
        pos = {**{4 + i: i for i in range(6)}, **{10 + i: 27 + i for i in range(5)}, **{20 + i: i for i in range(6)}}
        rows = sorted(pos)
        want = O.rotate(q.cpu()[rows], rotary.cpu(), torch.tensor([pos[r] for r in rows])).to(torch.bfloat16)
        assert torch.equal(out[rows].view(torch.int16), want.view(torch.int16))
        assert not out[[r for r in range(T) if r not in pos]].view(torch.int16).any()
        none = mes.SeqBatch(_ints([]), torch.zeros(0, 2, dtype=torch.int32, device=DEV), _ints([0]))
        assert not mes.mes_kv_append(cache, 0, none, q, k, v, rotary).view(torch.int16).any()            # no sequences at all


# ----------------------------------------------------------------------------------------------------------- the largest values

@pytest.mark.parametrize("dim", [64, 128])
def test_rows_that_see_the_largest_value_are_finite(dim):
    """The type's largest number as a value, at a token whose score is above that of the tokens before it, but not by much: a sum of weights
    that are at most 1 holds it."""
    big, n, at, heads, kvh = 3.3895313892515355e38, 200, 150, 4, 2
    g = torch.Generator().manual_seed(50)
    k, v, q = torch.zeros(n, kvh, dim), _rows(g, n, kvh, dim), torch.zeros(n, heads, dim)
    q[:, :, 0], k[at, :, 0] = 4.0, 1.0                                   # scores 0, and 4 for this token: 2^5.8 times their weight
    q, k, scale = q.to(torch.bfloat16), k.to(torch.bfloat16), 1.0
    v[at, 0, 5], v[at, 1, 6] = big, -big
    want, tol = O.attend(q, k, v, range(n), scale)
    assert bool(torch.isfinite(want).all()) and float(want.abs().max()) > 5e37
    out = mes.mes_attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), _ints([0, n]), scale=scale)
    _check(out, want, tol, "prompt")
    cache = mes.KvCache(1, 13, 16, kvh, dim)
    batch = mes.SeqBatch(_ints([n]), _ints([list(range(13))]), _ints([0, n]))
    mes.mes_kv_append(cache, 0, batch, None, k.to(DEV), v.to(DEV), None)
    _check(mes.mes_attn_extend(cache, 0, batch, q.to(DEV), scale=scale), want, tol, "extend")
    one = mes.SeqBatch(_ints([n]), _ints([list(range(13))]))
    _check(mes.AttnDecode(cache, heads, 1)(0, one, q[-1:].to(DEV), scale=scale), want[-1:], tol[-1:], "decode")
    two = mes.SeqBatch(_ints([n, n]), _ints([list(range(13))] * 2))
    order = torch.tensor([0, 1] * 10 + [2, 3] * 10)
    wide = q[-1:][:, order].to(DEV)                                       # 20 heads per key / value head: rows share tiles
    out = mes.AttnDecode(cache, 40, 2)(0, two, torch.cat([wide, wide]), [0, 2], [n - 10], scale=scale)
    for row in out:
        _check(row[None], want[-1:][:, order], tol[-1:][:, order], "decode, shared")
