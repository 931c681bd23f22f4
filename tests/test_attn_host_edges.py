"""Attention and its cache, host side (no GPU): refusals beside those of test_attn_host.py."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

import paper_2406_09041_amd as mes
import paper_2406_09041_amd.binding as B
from test_attn_host import FAKE, ODD, _kv, _seqs

lib = B.lib
OTHER = 0x20000


def _fresh(seqs=None, q=FAKE, k=FAKE, T=5, heads=4, ld_o=256, rotary=FAKE, n_pos=64, q_out=OTHER):
    kv, seqs = _kv(), seqs or _seqs()
    return lib.mes_kv_append_fresh(ctypes.byref(kv), 0, ctypes.byref(seqs), q, k, FAKE, T, heads, 256, 128, 128, rotary, n_pos, q_out, ld_o, None)


def test_append_into_fresh_queries_errors():
    assert _fresh(q=None) == 1 and _fresh(q_out=None) == 1 and _fresh(q=None, q_out=None) == 1
    assert _fresh(q_out=FAKE) == 2 and b"mes_kv_append_fresh: q_out is q" in lib.mes_last_error()      # it would be cleared
    assert _fresh(T=0, q=None, q_out=None) == 0
    # the other checks are those of mes_kv_append
    assert _fresh(k=None) == 1 and _fresh(q_out=ODD) == 6 and _fresh(ld_o=255) == 2 and _fresh(n_pos=63) == 2 and _fresh(rotary=None) == 1 and _fresh(heads=0) == 2
    assert _fresh(seqs=_seqs(n_seqs=0, kv_len=None, page_table=None), q_out=ODD) == 6                  # no sequences: all rows are cleared


def test_the_decode_workspace_is_refused_where_no_call_could_use_it():
    cache = lambda kvh=2, dim=64: SimpleNamespace(n_kv_heads=kvh, head_dim=dim, device="cpu", index=-1)  # noqa: E731
    for heads, seqs, c, what in ((4, 2049, cache(), "max_seqs"), (4, -1, cache(), "max_seqs"), (5, 8, cache(), "n_heads"), (130, 8, cache(), "n_heads"),
                                 (0, 8, cache(), "n_heads"), (4, 8, cache(dim=96), "head_dim")):
        with pytest.raises(AssertionError, match=what):
            mes.AttnDecode(c, heads, seqs)
    for seqs in (0, 1, 2048):
        assert mes.AttnDecode(cache(), 4, seqs).ws.numel() == lib.mes_attn_decode_workspace_bytes(max(seqs, 1), 4, 2, 64)


def test_the_prompt_workspace_is_the_packages_own():
    ws = mes.prompt_workspace(5, 1, 4, 2, 64, "cpu")
    assert ws.dtype == torch.uint8 and ws.numel() == lib.mes_attn_prompt_workspace_bytes(5, 1, 4, 2, 64) > 0
