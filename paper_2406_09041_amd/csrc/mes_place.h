// Which token of which sequence a row of a call is, from what stands in device memory, of which nothing is taken for granted: offsets
// that reach past the call's rows, that decrease or are negative, lengths that are anything.  Plain C++ without HIP, so that the host
// tests compile it.
#pragma once

namespace mes {

struct Place {
  int seq, pos;                // -1: behind the last sequence; position < 0 or past the capacity: none
  int from, to;                // positions [from, to) of the sequence's rows that are in the call, below the capacity
};
constexpr Place kNoPlace = {-1, -1, 0, 0};

// Row t of a call of T rows (0 <= t < T), if sequence s has rows [begin, end) and len tokens, the rows among them.
constexpr Place place_of_row(int s, int begin, int end, int len, int capacity, int t, int T) {
  if (begin > t || end <= t) return kNoPlace;
  if (begin < 0) begin = 0;
  if (len < 0) len = 0;
  const int cut = end > T ? end - T : 0;         // rows that the call does not have: its last ones
  const int first = len - (end - begin), behind = len - cut;
  return {s, len - (end - t), first > 0 ? first : 0, behind < capacity ? behind : capacity};
}

// The call's rows in the block of `tokens` (a power of two) that row t with a position inside [0, capacity) is in: positions from ..
// from + rows - 1, rows row0 .. row0 + rows - 1 of the call, t among them.
struct BlockRows {
  int begin, from, rows, row0;
};
constexpr BlockRows block_rows(const Place& at, int t, int tokens) {
  const int begin = at.pos & -tokens, from = begin > at.from ? begin : at.from, to = begin + tokens < at.to ? begin + tokens : at.to;
  return {begin, from, to - from, t - (at.pos - from)};
}

}  // namespace mes
