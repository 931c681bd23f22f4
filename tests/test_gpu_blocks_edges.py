"""The cache in blocks where its sequences differ, calls with fewer rows than their offsets name.  References: oracle/attn_oracle.py over what
mes_kv_read gives of a sequence's own pages."""
import pytest
import torch

import paper_2406_09041_amd as mes
from oracle import attn_oracle as O
from test_gpu_attn import DEV, _check, _ints, _rows

pytestmark = pytest.mark.gpu


def _own(cache, layer, table, kv_len):
    """Keys and values of every sequence as its own pages hold them."""
    out = []
    for pages, n in zip(table, kv_len):
        k, v = mes.mes_kv_read(cache, layer, mes.SeqBatch(_ints([n]), _ints([pages]), _ints([0, n])), n)
        out.append((k.cpu(), v.cpu()))
    return out


@pytest.mark.parametrize("larger", [1e3, 1e4, 3e5])
@pytest.mark.parametrize("at_once", [False, True])
@pytest.mark.parametrize("heads,kvh,dim,page,prefix", [(4, 2, 64, 16, 9), (8, 2, 128, 16, 41), (4, 4, 64, 64, 41), (34, 2, 64, 16, 25), (8, 1, 128, 32, 48), (4, 2, 64, 16, 15)])
def test_a_shared_prefix_is_what_every_sequence_holds(heads, kvh, dim, page, prefix, at_once, larger):
    """The first sequence goes on with a much larger token in the block that the prefix ends in, which rounds its copy of the prefix there
    again: the others' rows are of their own copies.  The last sequence is one token shorter than the prefix and holds other tokens."""
    g, news = torch.Generator().manual_seed(prefix + heads), [3, 1, 20, 2, -1]
    n = len(news)
    width = -(-(prefix + max(news)) // page)
    cache = mes.KvCache(2, n * width, page, kvh, dim, mes.KV_E4M3_BLOCKS)
    table = torch.randperm(n * width, generator=g).reshape(n, width).tolist()
    common = [_rows(g, prefix, kvh, dim) for _ in range(2)]
    rows = []
    for s, m in enumerate(news[:-1]):
        k, v = (_rows(g, m, kvh, dim) for _ in range(2))
        if s == 0:
            k[0], v[0] = k[0] * larger, v[0] * larger
        rows.append([torch.cat([a, b]) for a, b in zip(common, (k, v))])
    rows.append([_rows(g, prefix - 1, kvh, dim) for _ in range(2)])
    for s, m in enumerate(news):
        for a, b in [(0, prefix + m)] if at_once else [(0, min(prefix, prefix + m))] + [(prefix + i, prefix + i + 1) for i in range(m)]:
            k, v = (x[a:b].contiguous().to(DEV) for x in rows[s])
            mes.mes_kv_append(cache, 1, mes.SeqBatch(_ints([b]), _ints([table[s]]), _ints([0, b - a])), None, k, v)
    kv_len = [prefix + m for m in news]
    held = _own(cache, 1, table, kv_len)
    q = _rows(g, n, heads, dim, 2.0)
    call, batch = mes.AttnDecode(cache, heads, n), mes.SeqBatch(_ints(kv_len), _ints(table))
    shared, alone = call(1, batch, q.to(DEV), [0, n], [prefix]), call(1, batch, q.to(DEV))
    for s in range(n):
        want, tol = O.attend(q[s:s + 1], *held[s], [kv_len[s] - 1], dim ** -0.5)
        _check(alone[s:s + 1], want, tol, f"sequence {s}, nothing shared")
        _check(shared[s:s + 1], want, tol, f"sequence {s}")


CUT = [  # rows, offsets, lengths: the offsets reach past the call's rows
    (5, [0, 20], [20]), (5, [0, 20], [33]), (1, [0, 16], [40]), (10, [0, 3, 40], [19, 45]), (33, [0, 0, 30, 49], [4, 35, 19]), (7, [0, 9, 12], [9, 90]), (12, [0, 30], [9]),
]


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "blocks"])
@pytest.mark.parametrize("kvh,dim", [(8, 128), (2, 64)])
@pytest.mark.parametrize("T,offsets,kv_len", CUT)
def test_append_of_fewer_rows_than_the_offsets_name(T, offsets, kv_len, kvh, dim, kind):
    """The rows that are there get their places, all heads of them; what lies behind them in memory goes nowhere."""
    page, heads, n = 32, 2 * kvh, len(kv_len)
    g = torch.Generator().manual_seed(T + kvh)
    scale = [torch.full((1, kvh), x, device=DEV) for x in (0.25, 0.0625)]
    kinds = {"bf16": mes.KV_BF16, "e4m3": mes.KV_E4M3, "blocks": mes.KV_E4M3_BLOCKS}
    make = lambda: mes.KvCache(1, 4 * n, page, kvh, dim, kinds[kind], *(scale if kind == "e4m3" else (None, None)))  # noqa: E731
    table = torch.randperm(4 * n, generator=g).reshape(n, 4)
    angles = mes.Angles(mes.mes_rotary_table(4 * page, dim))
    wide = [torch.cat([_rows(g, T, h, dim), 1e4 * _rows(g, 40, h, dim)]).to(DEV) for h in (heads, kvh, kvh)]
    q, k, v = (x[:T] for x in wide)
    got, want = make(), make()
    for c in (got, want):                                        # older tokens, in the blocks that follow too
        old = [_rows(g, 4 * page, kvh, dim) for _ in range(2)] if c is got else old
        for s in range(n):
            mes.mes_kv_append(c, 0, mes.SeqBatch(_ints([4 * page]), _ints(table[s:s + 1].tolist()), _ints([0, 4 * page])), None, *(x.to(DEV) for x in old))
    out = mes.mes_kv_append(got, 0, mes.SeqBatch(_ints(kv_len), _ints(table.tolist()), _ints(offsets)), q, k, v, angles)
    # one call for each sequence, of the rows that are there
    turned = torch.zeros_like(out)
    for s in range(n):
        a, b = offsets[s], min(offsets[s + 1], T)
        if b > a:
            batch = mes.SeqBatch(_ints([kv_len[s] - (offsets[s + 1] - b)]), _ints(table[s:s + 1].tolist()), _ints([0, b - a]))
            turned[a:b] = mes.mes_kv_append(want, 0, batch, q[a:b], k[a:b], v[a:b], angles)
    assert torch.equal(out, turned)
    parts = ["k", "v"] + ["k_scale", "v_scale"] * (kind == "blocks")
    for x in parts:
        a, b = (getattr(c, x).view(torch.uint8) for c in (got, want))
        assert torch.equal(a, b), x


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "blocks"])
@pytest.mark.parametrize("offsets", [[0, 8, 3, 12], [0, 20, -5, 12], [4, 2, 1, 0], [0, -1, 40, 5]])
def test_append_with_offsets_out_of_order(offsets, kind):
    """Which row is whose is anyone's guess: the call ends, and pages that are none of the sequences' are left as they are."""
    page, kvh, dim, T = 16, 2, 64, 12
    g = torch.Generator().manual_seed(3)
    scale = [torch.ones(1, kvh, device=DEV) for _ in range(2)] if kind == "e4m3" else [None, None]
    cache = mes.KvCache(1, 20, page, kvh, dim, {"bf16": mes.KV_BF16, "e4m3": mes.KV_E4M3, "blocks": mes.KV_E4M3_BLOCKS}[kind], *scale)
    table = [[1, 3], [5, 7], [9, 11]]
    q, k, v = (_rows(g, T, h, dim).to(DEV) for h in (4, kvh, kvh))
    batch = mes.SeqBatch(_ints([30, 17, 12]), _ints(table), _ints(offsets))
    out = mes.mes_kv_append(cache, 0, batch, q, k, v, mes.Angles(mes.mes_rotary_table(2 * page, dim)))
    assert torch.isfinite(out).all()
    rest = torch.tensor([p for p in range(20) if p not in sum(table, [])], device=DEV)
    assert not cache.k.view(torch.uint8)[0, rest].any() and not cache.v.view(torch.uint8)[0, rest].any()
    for x in mes.mes_kv_read(cache, 0, batch, T):
        assert torch.isfinite(x).all()
