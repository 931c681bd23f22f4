"""Which token a row of a call is (csrc/mes_place.h), compiled for the host: against the definition where offsets are in order, and, whatever
stands in device memory, rows of a block that are all in the call."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BLOCK = 16

SHIM = r"""
#include "mes_place.h"
using namespace mes;
extern "C" void place(int s, int begin, int end, int len, int capacity, int t, int T, int* out) {
  const Place at = place_of_row(s, begin, end, len, capacity, t, T);
  out[0] = at.seq; out[1] = at.pos; out[2] = at.from; out[3] = at.to;
  if (at.seq < 0 || at.pos < 0 || at.pos >= capacity) return;
  const BlockRows b = block_rows(at, t, 16);
  out[4] = b.begin; out[5] = b.from; out[6] = b.rows; out[7] = b.row0;
}
"""


@pytest.fixture(scope="module")
def place(tmp_path_factory):
    d = tmp_path_factory.mktemp("place")
    src, lib = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-ftrapv", "-shared", "-fPIC", "-o", str(lib), str(src),
                           "-I" + os.path.join(ROOT, "paper_2406_09041_amd", "csrc")])
    entry = ctypes.CDLL(str(lib)).place

    def call(*args):
        out = (ctypes.c_int * 8)(*[-7] * 8)
        entry(*args, out)
        return list(out)

    return call


def _search(offsets, t):
    """The first sequence that ends behind row t."""
    return next((s for s in range(len(offsets) - 1) if offsets[s + 1] > t), len(offsets) - 1)


def test_rows_are_the_last_tokens_of_their_sequences(place):
    """Offsets in order, up to T or past it: every block's rows in the call, found from each of them alike."""
    rng = random.Random(1)
    for _ in range(400):
        n, capacity = rng.randint(1, 5), 16 * rng.randint(1, 6)
        offsets = [0]
        for _ in range(n):
            offsets.append(offsets[-1] + rng.choice([0, 1, rng.randint(1, 50)]))
        T = rng.choice([offsets[-1], offsets[-1] + 3, max(offsets[-1] - rng.randint(1, 20), 0)])
        kv_len = [rng.choice([-3, 0, rng.randint(0, 120), offsets[s + 1] - offsets[s] + rng.randint(0, 30)]) for s in range(n)]
        want = {}                                                # of (sequence, block): its rows
        where = {}
        for t in range(T):
            s = _search(offsets, t)
            if s < n:
                pos = max(kv_len[s], 0) - (offsets[s + 1] - t)
                where[t] = s, pos
                if 0 <= pos < capacity:
                    want.setdefault((s, pos // BLOCK), []).append((t, pos))
        for t in range(T):
            s = _search(offsets, t)
            if s == n:
                continue
            got = place(s, offsets[s], offsets[s + 1], kv_len[s], capacity, t, T)
            assert tuple(got[:2]) == where[t]
            if 0 <= got[1] < capacity:
                rows = want[s, got[1] // BLOCK]
                assert got[4:] == [got[1] // BLOCK * BLOCK, rows[0][1], len(rows), rows[0][0]]


def test_whatever_stands_in_memory_rows_are_in_the_call(place):
    """What the kernel reads and how often it goes round: 1 to 16 rows of [0, T), the row itself among them, positions below the capacity."""
    rng, most = random.Random(2), 2 ** 31 - 1
    some = lambda: rng.choice([-most - 1, -most, -40, -1, 0, 1, rng.randint(0, 60), rng.randint(0, 60), 1000, most - 1, most])  # noqa: E731
    places = 0
    for _ in range(200000):
        T, capacity = rng.choice([1, 5, 40, 2 ** 24 - 1]), rng.choice([16, 48, 2 ** 30])
        t = rng.randrange(min(T, 50))
        got = place(3, some(), some(), some(), capacity, t, T)
        if got[0] < 0 or not 0 <= got[1] < capacity:
            continue
        places += 1
        seq, pos, _, _, begin, start, rows, row0 = got
        assert seq == 3 and begin == pos // BLOCK * BLOCK and 1 <= rows <= BLOCK
        assert begin <= start <= pos < start + rows <= min(begin + BLOCK, capacity)
        assert 0 <= row0 and row0 + rows <= T and t - row0 == pos - start
    assert places > 5000
