"""How much work one decode call takes, host side (no GPU): as much as its numbers of 32 bits hold."""
import itertools
import math

import pytest

import paper_2406_09041_amd.binding as B
from test_attn_host import _decode, _kv, _seqs

SHAPE = 2


@pytest.mark.parametrize("n_seqs,kvh,page", [(2048, 1, 256), (2048, 8, 16), (700, 3, 256), (100, 8, 64)])
def test_the_largest_call(n_seqs, kvh, page):
    """12 costs for 128 tokens, and for twice as many more, of a sequence and key / value head: 2^32 of them at most."""
    fits = lambda pages: 12 * n_seqs * kvh * (pages * page // 128 + 2) <= 2 ** 32  # noqa: E731
    lo, hi = 1, 2 ** 30 // page + 1                              # the first that does not
    while lo < hi:
        mid = (lo + hi) // 2
        lo, hi = (mid + 1, hi) if fits(mid) else (lo, mid)
    call = lambda pages: _decode(kv=_kv(n_kv_heads=kvh, page_tokens=page), seqs=_seqs(n_seqs=n_seqs, table_pages=pages), heads=kvh, ld_q=64 * kvh, ld_o=64 * kvh, seg=None, pre=None, ws=None)  # noqa: E731
    assert call(lo) == SHAPE and b"more than one call takes" in B.lib.mes_last_error()
    assert call(lo - 1) not in (0, SHAPE) and b"workspace" in B.lib.mes_last_error()


def _line(lens, prefix, group, codes):
    """The costs of one key / value head of one expert's sequences, as the kernel lays them out."""
    wide, per_pass = group > 16, 128 // group
    tile, begin = (4, 8) if wide else (7, 12) if codes else (4, 7)
    many = lambda a, b: begin + tile * -(-(b - a // 64 * 64) // 64) if b > a else 0  # noqa: E731
    own = lambda a, b: many(a, b) if wide else (3 if codes else 2) + -(-(b - a // 32 * 32) // 32) if b > a else 0  # noqa: E731
    shares = sum(n >= prefix > 0 for n in lens) >= 2
    total = sum(own(prefix if shares and n >= prefix else 0, n) for n in lens)
    return total + (math.ceil(len(lens) / per_pass) * many(0, prefix) if shares else 0)


@pytest.mark.parametrize("group,codes", itertools.product([1, 4, 16, 17, 33, 42, 43, 64], [False, True]))
def test_no_batch_has_more(group, codes):
    """Every way for 2 to 9 sequences to be just shorter than the prefix, as long as it, or as long as the table."""
    for pages in (1, 3, 4, 5, 31, 64, 999):
        capacity = 16 * pages
        for n, prefix in itertools.product(range(1, 10), {0, 1, 16, capacity // 2 + 1, capacity - 31, capacity - 1, capacity}):
            for at, short in itertools.product(range(0, n + 1), range(0, n + 1)):
                if at + short <= n and 0 <= prefix <= capacity:
                    lens = [prefix] * at + [max(prefix - 1, 0)] * short + [capacity] * (n - at - short)
                    assert _line(lens, prefix, group, codes) <= 12 * n * (capacity // 128 + 2)
