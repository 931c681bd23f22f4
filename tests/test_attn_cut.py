"""How the rows of a call are cut over its keys (csrc/mes_attn_cut.h), compiled for the host: every key of every item in one part, and never more parts
than the workspace is laid out for."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include "mes_attn_cut.h"
using namespace mes;
extern "C" {
int block_of(int packed, int R, int columns, int items, int longest, int units) { return cut_block(packed != 0, R, columns, items, longest, units); }
int below(int b, int block, int base, int tiles) { return parts_below(b, block, base, tiles); }
int first(int b, int block, int base) { return first_item(b, block, base); }
int slots(int64_t workgroups) { return cut_slots_of(workgroups); }
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    d = tmp_path_factory.mktemp("cut")
    src, lib = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-ftrapv", "-shared", "-fPIC", "-o", str(lib), str(src),
                           "-I" + os.path.join(ROOT, "paper_2406_09041_amd", "csrc")])
    lib = ctypes.CDLL(str(lib))
    lib.slots.argtypes = [ctypes.c_int64]
    return lib


def test_every_key_is_in_one_part(cut):
    rng = random.Random(1)
    for _ in range(2000):
        base, tiles, block = rng.choice([0, rng.randint(0, 60)]), rng.randint(1, 40), rng.randint(1, 50)
        number = 0
        for b in range(-(-(base + tiles) // block)):
            assert cut.below(b, block, base, tiles) == number
            items = [t for t in range(tiles) if base + t + 1 > b * block]         # that see keys of the block
            assert items == list(range(cut.first(b, block, base), tiles))
            number += len(items)
        assert cut.below(-(-(base + tiles) // block), block, base, tiles) == number


@pytest.mark.parametrize("packed", [False, True])
def test_the_workspace_has_room_for_the_parts(cut, packed):
    rng, cuts = random.Random(2), 0
    for _ in range(30000):
        heads = rng.choice([1, 2, 4])                             # of a workgroup
        R, columns, n = 128 // heads, rng.choice([1, 2, 3, 4, 5, 7, 8, 10, 16, 32, 40, 100, 512]), rng.choice([1, 1, 2, 3, 8, 20, 64])
        most = rng.choice([100, 1000, 4000, 20000])
        rows = [rng.choice([0, 1, rng.randint(1, most), rng.randint(1, max(most // 10, 1))]) for _ in range(n)]
        before = [0 if packed else rng.choice([0, rng.randint(0, 3000), rng.randint(0, rng.choice([20000, 2 ** 24]))]) for _ in range(n)]
        T = sum(rows) + rng.choice([0, 0, 50])
        tiles, base = [-(-x // R) for x in rows], [-(-x // R) for x in before]
        workgroups = (T // R + n) * columns                      # of a call that is not cut
        items = sum(tiles)
        if items == 0 or items * columns > 1024:
            continue
        block = cut.block_of(packed, R, columns, items, max(b + t for b, t in zip(base, tiles) if t), sum(t * b + t * (t + 1) // 2 for b, t in zip(base, tiles)))
        if block == 0:
            continue
        cuts += 1
        assert block * R >= 256 and block * R % 64 == 0
        parts = sum(cut.below(-(-(b + t) // block), block, b, t) for b, t in zip(base, tiles) if t)
        assert parts * columns <= cut.slots(workgroups), (rows, before, R, columns)
    assert cuts > 500
