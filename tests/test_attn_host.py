"""Attention and its paged cache, host side (no GPU): every refusal of the entry points, before any HIP call, and the page
bookkeeping against its plain definition, operation by operation."""
import ctypes
import random

import pytest

import paper_2406_09041_amd as mes
import paper_2406_09041_amd.binding as B
from oracle.attn_oracle import Pages

lib = B.lib
FAKE, ODD = 0x10000, 0x10004


def _kv(**kw):
    d = dict(n_layers=2, n_pages=8, page_tokens=16, n_kv_heads=2, head_dim=64, dtype=0, k=FAKE, v=FAKE, k_scale=None, v_scale=None)
    d.update(kw)
    return B.mes_kv(*[d[n] for n, _ in B.mes_kv._fields_])


def _seqs(**kw):
    d = dict(n_seqs=3, table_pages=4, q_offsets=FAKE, kv_len=FAKE, page_table=FAKE)
    d.update(kw)
    return B.mes_seqs(*[d[n] for n, _ in B.mes_seqs._fields_])


def _append(kv=None, layer=0, seqs=None, q=FAKE, k=FAKE, v=FAKE, T=5, heads=4, ld_q=256, ld_k=128, ld_v=128, rotary=FAKE, n_pos=64, q_out=FAKE, ld_o=256):
    kv, seqs = kv or _kv(), seqs or _seqs()
    return lib.mes_kv_append(ctypes.byref(kv), layer, ctypes.byref(seqs), q, k, v, T, heads, ld_q, ld_k, ld_v, rotary, n_pos, q_out, ld_o, None)


def _prompt(q=FAKE, k=FAKE, v=FAKE, T=5, n=1, off=FAKE, heads=4, kvh=2, dim=64, ld_q=256, ld_k=128, ld_v=128, scale=0.125, out=FAKE, ld_o=256, ws=None, wsb=0):
    return lib.mes_attn_prompt(q, k, v, T, n, off, heads, kvh, dim, ld_q, ld_k, ld_v, scale, out, ld_o, ws, wsb, None)


def _extend(kv=None, layer=0, seqs=None, q=FAKE, T=5, heads=4, ld_q=256, scale=0.125, out=FAKE, ld_o=256, ws=None, wsb=0):
    kv, seqs = kv or _kv(), seqs or _seqs()
    return lib.mes_attn_extend(ctypes.byref(kv), layer, ctypes.byref(seqs), q, T, heads, ld_q, scale, out, ld_o, ws, wsb, None)


def _decode(kv=None, layer=0, seqs=None, q=FAKE, heads=4, ld_q=256, seg=(0, 1, 3), pre=(5, 0), E=None, scale=0.125, out=FAKE, ld_o=256, ws=FAKE, wsb=1 << 30):
    kv, seqs = kv or _kv(), seqs or _seqs()
    segc = None if seg is None else (ctypes.c_int32 * len(seg))(*seg)
    prec = None if pre is None else (ctypes.c_int32 * len(pre))(*pre)
    return lib.mes_attn_decode(ctypes.byref(kv), layer, ctypes.byref(seqs), q, heads, ld_q, len(pre or ()) if E is None else E, segc, prec, scale, out,
                               ld_o, ws, wsb, None)


@pytest.mark.parametrize("call", [_append, _extend, _decode])
def test_cache_descriptor_errors(call):
    assert call(kv=_kv(dtype=2)) == 3
    assert call(kv=_kv(n_layers=0)) == 2 and call(kv=_kv(n_pages=0)) == 2
    for page in (0, 8, 24, 512, -16):
        assert call(kv=_kv(page_tokens=page)) == 2
    for dim in (0, 32, 96, 256):
        assert call(kv=_kv(head_dim=dim)) == 2
    assert call(kv=_kv(n_kv_heads=0)) == 2
    assert call(kv=_kv(k=None)) == 1 and call(kv=_kv(v=None)) == 1
    assert call(kv=_kv(k=ODD)) == 6 and call(kv=_kv(v=ODD)) == 6
    assert call(kv=_kv(dtype=1)) == 1 and call(kv=_kv(dtype=1, k_scale=FAKE)) == 1        # e4m3 needs both scales
    assert call(layer=-1) == 2 and call(layer=2) == 2
    assert b"layer" in lib.mes_last_error()


@pytest.mark.parametrize("call", [_append, _extend, _decode])
def test_batch_errors(call):
    assert call(seqs=_seqs(n_seqs=-1)) == 2 and call(seqs=_seqs(n_seqs=2049)) == 2
    assert call(seqs=_seqs(table_pages=0)) == 2 and call(seqs=_seqs(table_pages=1 << 30)) == 2
    assert call(seqs=_seqs(kv_len=None)) == 1 and call(seqs=_seqs(page_table=None)) == 1
    assert call(seqs=_seqs(n_seqs=0, kv_len=None, page_table=None)) == 0                  # no sequences: nothing to do


def test_append_errors():
    assert _append(T=-1) == 2
    assert _append(T=0, k=None, v=None, q=None, q_out=None) == 0
    assert _append(seqs=_seqs(q_offsets=None)) == 5                                       # 5 rows, one for each of 3 sequences
    assert _append(k=None) == 1 and _append(v=None) == 1
    assert _append(q=None) == 1 and _append(q_out=None) == 1                              # both or neither
    assert _append(rotary=None) == 1                                                      # queries only pass through to be turned
    assert _append(k=ODD) == 6 and _append(q=ODD) == 6 and _append(q_out=ODD) == 6 and _append(rotary=ODD) == 6
    assert _append(ld_k=127) == 2 and _append(ld_k=132) == 2 and _append(ld_v=120) == 2 and _append(ld_q=248) == 2 and _append(ld_o=255) == 2
    assert _append(n_pos=63) == 2 and b"rotary" in lib.mes_last_error()                   # the table has room for 64 tokens
    assert _append(heads=0) == 2
    assert _append(ld_o=512) == 2                                                         # in place, but rows elsewhere


def test_prompt_and_extend_errors():
    for call in (_prompt, _extend):
        assert call(T=-1) == 2 and call(T=0, q=None, out=None) == 0
        assert call(q=None) == 1 and call(out=None) == 1
        assert call(q=ODD) == 6 and call(out=ODD) == 6
        assert call(ld_q=255) == 2 and call(ld_q=260) == 2 and call(ld_o=128) == 2
        assert call(heads=3) == 2 and call(heads=0) == 2 and call(heads=130) == 2         # a multiple of 2, up to 64 times
        for scale in (0.0, -1.0, float("nan"), float("inf")):
            assert call(scale=scale) == 2
        n = 1 if call is _prompt else 3
        need = lib.mes_attn_prompt_workspace_bytes(5, n, 4, 2, 64)
        assert need > 0 and call(ws=FAKE, wsb=need - 1) == 7 and call(ws=ODD, wsb=need) == 6       # NULL is fine: no item is cut
    for bad in ((-1, 1, 4, 2, 64), (5, -1, 4, 2, 64), (5, 2049, 4, 2, 64), (5, 1, 5, 2, 64), (5, 1, 4, 2, 32)):
        assert lib.mes_attn_prompt_workspace_bytes(*bad) == 0
    assert lib.mes_attn_prompt_workspace_bytes(1 << 20, 64, 32, 8, 128) == (1024 + 512) * 128 * (8 + 128 * 4)
    assert _prompt(k=None) == 1 and _prompt(v=ODD) == 6 and _prompt(ld_k=64) == 2 and _prompt(ld_v=129) == 2
    assert _prompt(off=None) == 1 and _prompt(n=-1) == 2 and _prompt(n=2049) == 2 and _prompt(n=0) == 0
    assert _prompt(dim=80) == 2 and _prompt(kvh=0) == 2
    assert _extend(seqs=_seqs(q_offsets=None)) == 1


def test_decode_errors():
    assert _decode(q=None) == 1 and _decode(out=ODD) == 6 and _decode(ld_q=100) == 2 and _decode(heads=5) == 2
    for scale in (0.0, float("nan")):
        assert _decode(scale=scale) == 2
    assert _decode(seg=None) == 1 and _decode(pre=None, E=2) == 1                          # both or neither
    assert _decode(seg=(1, 1, 3)) == 5 and _decode(seg=(0, 2, 1)) == 5 and _decode(seg=(0, 1, 4)) == 5
    assert _decode(pre=(5, -1)) == 5
    assert _decode(E=0) == 2 and _decode(E=65) == 2
    need = lib.mes_attn_decode_workspace_bytes(3, 4, 2, 64)
    assert need > 0 and _decode(wsb=need - 1) == 7 and _decode(ws=None) == 7 and _decode(ws=ODD) == 6
    assert b"workspace" in lib.mes_last_error()
    assert _decode(seqs=_seqs(n_seqs=2048, table_pages=1 << 22), seg=None, pre=None) == 2  # more units than 32 bits number
    for bad in ((0, 4, 2, 64), (2049, 4, 2, 64), (3, 5, 2, 64), (3, 4, 0, 64), (3, 4, 2, 96), (3, 130, 2, 64)):
        assert lib.mes_attn_decode_workspace_bytes(*bad) == 0
    assert lib.mes_attn_decode_workspace_bytes(256, 32, 8, 128) < 96 << 20


def test_copy_errors():
    def call(src, dst, kv=None, n=None):
        kv = kv or _kv()
        arr = lambda v: None if v is None else (ctypes.c_int32 * max(len(v), 1))(*v)  # noqa: E731
        return lib.mes_kv_copy_pages(ctypes.byref(kv), arr(src), arr(dst), len(src or ()) if n is None else n, None)
    assert call([], []) == 0 and call(None, None, n=0) == 0
    assert call([0], None) == 1 and call(None, [0], n=1) == 1
    assert call([0], [1], n=-1) == 2 and call([0] * 9, [1] * 9) == 2
    assert call([8], [1]) == 9 and call([0], [8]) == 9 and call([-1], [1]) == 9 and call([0], [-1]) == 9
    assert call([0, 1], [2, 2]) == 9 and b"twice" in lib.mes_last_error()
    assert call([0, 1], [1, 2]) == 9 and b"read and written" in lib.mes_last_error()
    assert call([3], [3]) == 9
    assert call([0], [1], kv=_kv(page_tokens=20)) == 2


# ------------------------------------------------------------------------------------------------------ bookkeeping

def _same(pool, ora, max_seqs):
    assert pool.unused() == len(ora.unused())
    table, length = pool.table(range(max_seqs))
    for s in range(max_seqs):
        assert length[s] == ora.length[s] == pool.length(s)
        m = len(ora.pages[s])
        assert table[s, :m].tolist() == ora.pages[s] and not table[s, m:].any()


@pytest.mark.parametrize("seed", range(6))
def test_bookkeeping_follows_its_definition(seed):
    rng = random.Random(seed)
    n_pages, t, seqs, most = rng.choice([(12, 16, 5, 12), (40, 16, 8, 9), (64, 4, 20, 64), (7, 1, 3, 7)])
    pool, ora = mes.PagePool(n_pages, t, seqs, most), Pages(n_pages, t, seqs, most)
    refused = 0
    for _ in range(400):
        op = rng.choice(["grow", "grow", "grow", "fork", "free", "compact"])
        if op == "grow":
            who = rng.sample(range(seqs), rng.randint(1, seqs))
            add = [rng.choice([0, 1, 1, t, rng.randint(0, 3 * t)]) for _ in who]
            if any(ora.length[s] + a > most * t for s, a in zip(who, add)):
                with pytest.raises(mes.MesError) as e:
                    pool.grow(who, add)
                assert e.value.status == 2
            else:
                want = ora.grow(who, add)
                if want is None:
                    refused += 1
                    with pytest.raises(mes.MesError) as e:
                        pool.grow(who, add)
                    assert e.value.status == 9
                else:
                    src, dst = pool.grow(who, add)
                    assert list(zip(src, dst)) == want
        elif op == "fork":
            parent, child = rng.sample(range(seqs), 2)
            if ora.length[child]:
                ora.free(child)
                pool.free(child)
            n = rng.randint(0, ora.length[parent])
            pool.fork(parent, child, n)
            ora.fork(parent, child, n)
        elif op == "free":
            s = rng.randrange(seqs)
            pool.free(s)
            ora.free(s)
        else:
            live = sorted({p for own in ora.pages for p in own})
            src, dst = pool.compact()
            assert len(set(dst)) == len(dst) and not set(src) & set(dst) and set(src) <= set(live) and not set(dst) & set(live)
            move = dict(zip(src, dst))
            ora.pages = [[move.get(p, p) for p in own] for own in ora.pages]
            assert sorted({p for own in ora.pages for p in own}) == list(range(len(live)))
        _same(pool, ora, seqs)
    for s in range(seqs):
        pool.free(s)
    assert pool.unused() == n_pages
    assert refused or n_pages > 30


def test_forks_share_pages_until_one_writes():
    pool = mes.PagePool(10, 16, 4)
    assert pool.grow([0], [40]) == ([], [])
    pool.fork(0, 1)
    pool.fork(0, 2, 32)                                        # on a page's border: nothing is shared that it could write to
    assert pool.unused() == 7
    assert pool.grow([2], [1]) == ([], [])
    assert pool.grow([0, 1], [1, 1]) == ([2], [4])             # the first to write copies, the last holder keeps the page
    table, length = pool.table([0, 1, 2], 3)
    assert table.tolist() == [[0, 1, 4], [0, 1, 2], [0, 1, 3]] and length.tolist() == [41, 41, 33]
    pool.free(0)
    assert pool.unused() == 6
    assert pool.compact() == ([], [])                          # page 4 is free, 0 to 3 are in use


def test_bookkeeping_errors():
    for bad in ((0, 16, 4, 4), (4, 0, 4, 4), (4, 16, 0, 4), (4, 16, 4, 0), (4, 1 << 20, 4, 1 << 20)):
        with pytest.raises(mes.MesError) as e:
            mes.PagePool(*bad)
        assert e.value.status == 2
    assert lib.mes_pages_create(4, 16, 4, 4, None) == 1
    pool = mes.PagePool(4, 16, 3, 3)
    pool.grow([0], [20])
    for call, status in ((lambda: pool.grow([3], [1]), 2), (lambda: pool.grow([-1], [1]), 2), (lambda: pool.grow([0, 0], [1, 1]), 2),
                         (lambda: pool.grow([1, 0], [1, -1]), 2), (lambda: pool.grow([0], [29]), 2), (lambda: pool.grow([0], [2 ** 31 - 1]), 2),
                         (lambda: pool.grow([1], [48]), 9), (lambda: pool.fork(0, 0), 2), (lambda: pool.fork(0, 3), 2), (lambda: pool.fork(1, 0, 0), 2),
                         (lambda: pool.fork(0, 1, 21), 2), (lambda: pool.fork(0, 1, -1), 2), (lambda: pool.free(3), 2), (lambda: pool.table([0], 1), 2),
                         (lambda: pool.table([5], 3), 2)):
        with pytest.raises(mes.MesError) as e:
            call()
        assert e.value.status == status
        assert pool.length(0) == 20 and pool.length(1) == 0 and pool.unused() == 2        # nothing has changed
    n = ctypes.c_int(0)
    one = (ctypes.c_int32 * 1)(0)
    assert lib.mes_pages_grow(None, one, one, 1, one, one, ctypes.byref(n)) == 1
    assert lib.mes_pages_grow(pool.handle, one, None, 1, one, one, ctypes.byref(n)) == 1
    assert lib.mes_pages_fork(None, 0, 1, 0) == 1 and lib.mes_pages_free(None, 0) == 1
    assert lib.mes_pages_compact(pool.handle, None, one, ctypes.byref(n)) == 1
    assert lib.mes_pages_table(pool.handle, one, 1, None, 3, None) == 1
    assert lib.mes_pages_length(None, 0) == -1 and pool.length(7) == -1 and lib.mes_pages_unused(None) == -1


def test_sizes_that_do_not_fit_the_device_indexes():
    for call in (_append, _extend, _decode):
        assert call(seqs=_seqs(table_pages=(1 << 26) + 1)) == 2               # 16-token pages: 2^30 tokens and a page
        assert call(ld_q=(1 << 26) + 8) == 2
    assert _append(T=1 << 24) == 2 and _extend(T=1 << 24) == 2 and _prompt(T=1 << 24) == 2
    assert _prompt(ld_k=(1 << 26) + 8) == 2 and _prompt(ld_v=(1 << 26) + 8) == 2 and _prompt(ld_o=(1 << 26) + 8) == 2
    kv, wide = _kv(n_kv_heads=1024), 1024 * 32 * 64
    assert _decode(kv=kv, seqs=_seqs(n_seqs=513), heads=1024 * 32, ld_q=wide, ld_o=wide, seg=None, pre=None, wsb=1 << 62) == 2   # 513 * 32768 rows
    assert b"heads" in lib.mes_last_error()
