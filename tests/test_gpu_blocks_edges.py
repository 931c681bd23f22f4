"""The cache in blocks where its sequences differ: prefixes that end inside a block.  References: oracle/attn_oracle.py over what
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
