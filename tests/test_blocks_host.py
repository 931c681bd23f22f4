"""Rotary positions in their other forms and the cache in blocks, host side (no GPU): every refusal of the entry points, before any
HIP call."""
import ctypes

import pytest
import torch

import paper_2406_09041_amd as mes
import paper_2406_09041_amd.binding as B
from test_attn_host import FAKE, ODD, _append, _decode, _extend, _kv, _seqs

lib = B.lib
OTHER = 0x20000
NAN, INF = float("nan"), float("inf")


def _angles(**kw):
    d = dict(table=FAKE, n_positions=64, dims=64, layout=0)
    d.update(kw)
    return B.mes_angles(*[d[n] for n, _ in B.mes_angles._fields_])


def _blocks(**kw):
    return _kv(**{**dict(dtype=3, k_scale=FAKE, v_scale=FAKE), **kw})


def _turned(kv=None, layer=0, seqs=None, q=FAKE, k=FAKE, v=FAKE, T=5, heads=4, ld_q=256, ld_k=128, ld_v=128, angles=0, q_out=OTHER, ld_o=256, fresh=0):
    kv, seqs = kv or _blocks(), seqs or _seqs()
    angles = _angles() if angles == 0 else angles
    return lib.mes_kv_append_angles(ctypes.byref(kv), layer, ctypes.byref(seqs), q, k, v, T, heads, ld_q, ld_k, ld_v,
                                    None if angles is None else ctypes.byref(angles), q_out, ld_o, fresh, None)


def _rotary(angles=0, positions=FAKE, q=FAKE, k=FAKE, T=5, heads=4, kvh=2, dim=64, ld_q=256, ld_k=128, dtype=0, transpose=0, q_out=OTHER, ld_qo=256,
            k_out=OTHER, ld_ko=128, fresh=0):
    angles = _angles() if angles == 0 else angles
    return lib.mes_rotary(None if angles is None else ctypes.byref(angles), positions, q, k, T, heads, kvh, dim, ld_q, ld_k, dtype, transpose, q_out, ld_qo,
                          k_out, ld_ko, fresh, None)


def _table(table=FAKE, n=10, dims=64, base=1e4, scaling=0, factor=1.0, context=0, low=1.0, high=32.0, magnitude=1.0):
    return lib.mes_rotary_table(table, n, dims, base, scaling, factor, context, low, high, magnitude, None)


def _read(kv=None, layer=0, seqs=None, T=5, k=FAKE, v=OTHER, ld_k=128, ld_v=128, fresh=0):
    kv, seqs = kv or _blocks(), seqs or _seqs()
    return lib.mes_kv_read(ctypes.byref(kv), layer, ctypes.byref(seqs), T, k, v, ld_k, ld_v, fresh, None)


@pytest.mark.parametrize("call", [_append, _extend, _decode, _turned, _read])
def test_cache_of_blocks_errors(call):
    assert call(kv=_kv(dtype=3)) == 1 and call(kv=_kv(dtype=3, k_scale=FAKE)) == 1 and b"exponent" in lib.mes_last_error()
    assert call(kv=_kv(dtype=2)) == 3 and call(kv=_kv(dtype=4)) == 3
    assert call(kv=_blocks(page_tokens=8)) == 2 and call(kv=_blocks(k=ODD)) == 6 and call(kv=_blocks(head_dim=96)) == 2
    assert call(layer=2) == 2 and call(layer=-1) == 2
    assert call(seqs=_seqs(n_seqs=2049)) == 2 and call(seqs=_seqs(kv_len=None)) == 1


def test_append_with_angles_errors():
    assert _turned(angles=_angles(table=None)) == 1 and _turned(angles=_angles(table=ODD)) == 6
    for dims in (0, 8, 24, 80, -16):
        assert _turned(angles=_angles(dims=dims)) == 2
    assert _turned(angles=_angles(layout=2)) == 2 and _turned(angles=_angles(layout=-1)) == 2
    assert _turned(angles=_angles(n_positions=63)) == 2 and b"rotary" in lib.mes_last_error()
    assert _turned(angles=None) == 1                             # queries only pass through to be turned
    assert _turned(fresh=2) == 2 and _turned(fresh=1, q_out=FAKE) == 2 and _turned(fresh=1, q=None, q_out=None) == 1
    assert _turned(T=-1) == 2 and _turned(T=1 << 24) == 2 and _turned(T=0, q=None, k=None, v=None, q_out=None) == 0
    assert _turned(k=None) == 1 and _turned(v=ODD) == 6 and _turned(ld_k=64) == 2 and _turned(ld_o=258) == 2
    assert _turned(seqs=_seqs(n_seqs=0, kv_len=None, page_table=None)) == 0
    assert _turned(seqs=_seqs(q_offsets=None)) == 5


def test_rotary_errors():
    assert _rotary(angles=None) == 1 and _rotary(angles=_angles(table=None)) == 1 and _rotary(angles=_angles(dims=80)) == 2
    assert _rotary(angles=_angles(n_positions=-1)) == 2 and _rotary(angles=_angles(layout=7)) == 2
    assert _rotary(T=-1) == 2 and _rotary(T=1 << 24) == 2 and _rotary(T=0, q=None, k=None, q_out=None, k_out=None, positions=None) == 0
    assert _rotary(positions=None) == 1 and _rotary(q=None) == 1 and _rotary(q_out=None) == 1
    assert _rotary(k=None) == 1 and _rotary(k_out=None) == 1      # both or neither
    assert _rotary(q=ODD) == 6 and _rotary(k_out=ODD) == 6
    assert _rotary(dtype=2) == 3 and _rotary(transpose=2) == 2 and _rotary(fresh=-1) == 2
    for dim in (0, 8, 72, 528):
        assert _rotary(dim=dim) == 2
    assert _rotary(heads=0) == 2 and _rotary(kvh=0) == 2 and _rotary(heads=65536) == 2
    assert _rotary(ld_q=255) == 2 and _rotary(ld_ko=130) == 2 and _rotary(ld_qo=(1 << 26) + 8) == 2
    assert _rotary(q_out=FAKE, ld_qo=512) == 2 and _rotary(k_out=FAKE, ld_ko=256) == 2
    assert _rotary(q_out=FAKE, fresh=1) == 2 and _rotary(k_out=FAKE, fresh=1) == 2


def test_table_errors():
    assert _table(n=-1) == 2 and _table(n=(1 << 26) + 1) == 2 and _table(n=0, table=None) == 0
    for dims in (0, 8, 40, 528):
        assert _table(dims=dims) == 2
    assert _table(table=None) == 1 and _table(table=ODD) == 6
    for base in (0.0, -1.0, NAN, INF):
        assert _table(base=base) == 2
    assert _table(base=1e-30, dims=128) == 2 and b"frequency" in lib.mes_last_error()
    assert _table(scaling=4) == 2 and _table(scaling=-1) == 2 and _table(magnitude=NAN) == 2
    for scaling in (1, 2, 3):
        for factor in (0.5, NAN, INF, -2.0):
            assert _table(scaling=scaling, factor=factor, context=100) == 2
    assert _table(scaling=3, factor=2.0, context=0) == 2 and _table(scaling=3, factor=2.0, context=9, low=4.0, high=4.0) == 2
    assert _table(scaling=3, factor=2.0, context=9, low=-1.0) == 2 and _table(scaling=3, factor=2.0, context=9, high=INF) == 2


def test_read_errors():
    assert _read(T=-1) == 2 and _read(T=1 << 24) == 2 and _read(T=0, k=None, v=None) == 0
    assert _read(k=None, v=None) == 1 and _read(k=ODD) == 6 and _read(v=ODD) == 6 and _read(ld_k=64) == 2 and _read(ld_v=132) == 2
    assert _read(v=FAKE) == 2 and _read(fresh=3) == 2
    assert _read(seqs=_seqs(q_offsets=None)) == 5
    assert _read(seqs=_seqs(n_seqs=0, kv_len=None, page_table=None)) == 0
    assert _read(kv=_kv(dtype=1)) == 1


def test_the_binding_refuses():
    with pytest.raises(AssertionError, match="scaling"):
        mes.mes_rotary_table(4, 64, scaling="other")
    with pytest.raises(AssertionError):
        mes.Angles(torch.zeros(4, 2, 32))                        # not on a GPU
    with pytest.raises(AssertionError, match="finds its exponents itself"):
        mes.KvCache(1, 4, 16, 2, 64, mes.KV_E4M3_BLOCKS, torch.zeros(1, 2), torch.zeros(1, 2), device="cpu")
