// What the kernels on a paged cache read from the arrays of a tr_sequences, and how a launch's keys are shared out.  Plain C++: constexpr
// functions are both the host's and the device's, so the bounds that keep every access inside the caller's arrays are tested on the host.
#pragma once
#include <stdint.h>

#include "divisor.h"

namespace tr {

struct Sequences {
  const int* table;      // [n][max_pages], rows table_stride apart
  const int* kv_len;
  const int* q_start;
  const int* q_pos;      // or null
  int64_t table_stride;
  int n, max_pages;
  int tokens;            // of the call's tensors (their S)
  int n_pages, page_size;
  Divisor by_page;       // of page_size
};

constexpr int kPosLimit = 1 << 30;
constexpr int clamped(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// A sequence, whatever its entries hold: 0 <= start, start + n <= tokens; 0 <= len <= max_pages * page_size; -2^30 <= pos < 2^30.
struct Sequence { int start, n, len, pos; };
constexpr Sequence sequence(const Sequences& s, int b) {
  Sequence r = {0, 0, 0, 0};
  r.start = clamped(s.q_start[b], 0, s.tokens);
  r.n = clamped(s.q_start[b + 1], r.start, s.tokens) - r.start;
  r.len = clamped(s.kv_len[b], 0, s.max_pages * s.page_size);   // (at most 2^30, see the entry points)
  r.pos = clamped(s.q_pos ? s.q_pos[b] : r.len - r.n, -kPosLimit, kPosLimit - 1);   // (pos + tokens fits)
  return r;
}

// Keys 0 .. visible(...) - 1 are those that token t of a sequence sees.
constexpr int visible(const Sequence& q, int t, bool causal) { return causal ? clamped(q.pos + t + 1, 0, q.len) : q.len; }

// Page (-1: none) and slot of key c, 0 <= c < max_pages * page_size.
struct Slot { int page, slot; };
constexpr Slot slot_of(const Sequences& s, int b, int c) {
  const int i = divide(s.by_page, c), page = s.table[(int64_t)b * s.table_stride + i];
  return Slot{page >= 0 && page < s.n_pages ? page : -1, c - i * s.page_size};
}

// The sequences that a launch serves: those with more than `over` and at most `most` rows a K/V head, in tiles of `tile` rows.
struct RowClass { int tile, over, most; };
constexpr int tiles_of(int rows, RowClass c) { return rows > c.over && rows <= c.most ? (rows + c.tile - 1) / c.tile : 0; }

// Keys of a part, a multiple of kPartStep, so that parts begin on whole steps of a workgroup.
//   work     sum over (sequence, K/V head) of row tiles x steps_of(keys); tiles: of row tiles; longest: largest steps_of(keys)
//   share    how the keys may be shared out
// Uncut, the row tiles take as long as rounds of the longest or, where they are of different lengths, an even share and the longest behind it.  Cut for r rounds of
// `at_once` workgroups a tile's last part is half a part on average, so that parts are work / (r at_once - tiles / 2).  What is estimated to end first is
// taken, costs beside the keys' being those of an item and of the fold, in sixteenths of a step.
// Tiles that are cut have fewer than steps / part + 1 parts: all of them together at most share.slots(tiles).
constexpr int kPartStep = 128, kMostRounds = 4;
constexpr int steps_of(int keys) { return (keys + kPartStep - 1) / kPartStep; }
struct Share {
  int at_once;      // workgroups that run at once, 0: keys are not shared out
  int rounds;       // at most
  int item, fold;   // costs
  constexpr int slots(int64_t tiles) const { return at_once * rounds + (int)(tiles < at_once * rounds ? tiles : at_once * rounds); }
};
constexpr int part_keys(int64_t work, int64_t tiles, int longest, Share share) {
  if (share.at_once <= 0 || work <= 0 || work > 0x3ffffff) return kPosLimit;   // (as many keys as a sequence has at most)
  const unsigned w = (unsigned)work, at_once = (unsigned)share.at_once, n_tiles = (unsigned)(tiles < 0x3ffffff ? tiles : 0x3ffffff);
  const unsigned full = (n_tiles + at_once - 1) / at_once;
  const unsigned even = 16 * w / at_once + 16 * (unsigned)longest, rounds = full < 0x3ff && longest < 0x3fff ? 16 * full * (unsigned)longest : even;
  unsigned best = (even < rounds ? even : rounds) + (unsigned)share.item * (full < 64 ? full : 64);
  int part = kPosLimit;
  for (int r = 1; r <= share.rounds; r++) {
    const unsigned all = (unsigned)r * at_once;
    if (all <= n_tiles / 2) continue;
    const unsigned n = all - n_tiles / 2, steps = (w + n - 1) / n < 2 ? 2 : (w + n - 1) / n;
    const unsigned time = (unsigned)r * (16 * steps + (unsigned)share.item) + (unsigned)share.fold;
    if (steps < (unsigned)longest && time < best) {
      best = time;
      part = (int)steps * kPartStep;
    }
  }
  return part;
}
constexpr int parts_of(int keys, int part) { return keys <= part ? 1 : (keys - 1) / part + 1; }

// Row tiles that the sequences of `tokens` tokens have at most, `group` rows a token: each has at most one that is not full.
constexpr int64_t most_tiles(int64_t tokens, int64_t n_seqs, int64_t group, RowClass c) {
  const int64_t some = tokens * group / (c.over + 1);
  return tokens * group / c.tile + (some < n_seqs ? some : n_seqs);
}

}  // namespace tr
