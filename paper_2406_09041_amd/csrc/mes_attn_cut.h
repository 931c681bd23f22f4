// How a call's rows are cut over its keys (mes_attn_prompt.hip): items are tiles of R rows, keys are counted in units of R: item t of a sequence with
// `base` units before its rows sees about base + t + 1.  Plain C++ without HIP, so that the host tests compile it: what is said here about the
// number of parts is what the workspace is laid out for.
#pragma once

#include <stdint.h>

namespace mes {

constexpr int kHeld = 512;             // workgroups that the chip holds, two per compute unit
constexpr int kMostCut = 1024;         // items of a call that is cut: with more, no compute unit is without work for long
constexpr int kLeastPart = 256;        // keys of a block
constexpr int kCutTile = 64;           // keys of a tile

// Parts of the blocks below block b of a sequence: block i is seen by the items whose keys reach past its beginning.
constexpr int parts_below(int b, int block, int base, int tiles) {
  const int full = b < base / block + 1 ? b : base / block + 1;   // blocks that begin at or before base: all items
  return full * tiles + (b - full) * (tiles + base) - block * ((b - full) * (full + b - 1) / 2);
}
constexpr int first_item(int b, int block, int base) { return b * block > base ? b * block - base : 0; }

// Units of a block, 0: the call is not cut.  columns: workgroups of an item; of the call: its items, the units of the longest and of all.
//
// A tile of keys takes a workgroup 1.1 us alone on its compute unit and 2.3 us beside another; writing and adding up parts about as long
// as 11 tiles (measured: 512 rows behind 4096 tokens 70 us cut and 87 whole; a prompt of 1024 tokens 38 us cut and 24 whole).  The longest item
// either has its compute unit to itself, or, where there are more items than compute units, it has company until the others' share of the work
// is done (8 prompts behind 0 to 4096 tokens of an e4m3 cache, 528 items, longest 72 tiles: 148 us whole, 118 cut).  Packed prompts alone have
// items of every length up to the longest, so that it is alone sooner: there it has to be longer by a quarter (16 heads over 2, one prompt of
// 4000 rows 90 us whole, 101 cut; 8 over 1, of 5800 112 and 102, of 8500 180 and 180, of 10000 228 and 239).
constexpr int cut_block(bool packed, int R, int columns, int items, int longest, int units) {
  if (items * columns > kMostCut) return 0;
  const int places = kHeld / columns > 1 ? kHeld / columns : 1, share = units / places + 1;   // of a workgroup, if all had the same
  const bool beside = items * columns > kHeld / 2 && longest > (packed ? 27 : 21) * share / 16 + (packed ? 24 : 18) * kCutTile / R;
  if (longest <= 21 * share / 8 + 11 * kCutTile / R && !beside) return 0;
  // longer than a share: the workspace has room for no more parts, and they fit the chip at once; whole tiles (R is 32, 64 or 128)
  const int block = share + share / 8 + 1 > kLeastPart / R ? share + share / 8 + 1 : kLeastPart / R;
  return block + (R < kCutTile ? block & 1 : 0);
}
// parts of a call, times columns: one per item, and one per block
constexpr int cut_slots_of(int64_t workgroups) { return (int)(workgroups < kMostCut ? workgroups : kMostCut) + kHeld; }

}  // namespace mes
