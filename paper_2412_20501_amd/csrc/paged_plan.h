// What the kernels on a paged cache read from the arrays of a tr_sequences, how a launch's keys are shared out, and the launches of a call.  Plain C++: constexpr
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
// What is estimated to end first is taken, in sixteenths of the time that a step takes a workgroup which has its compute unit to itself:
//   - uncut: rounds of the longest row tile or, where they are of different lengths, an even share and the longest behind it, which then has its unit to itself;
//   - cut for one round of 1 .. most_per_unit workgroups a unit, or for more of them, which then share the work evenly but for the last.  A tile's last part is half a
//     part on average, so that parts are work / (workgroups - tiles / 2).
// (Few rows, K and V at HBM's rate: 1, 2, 3 a unit take 253, 224, 218 us for 64 sequences of up to 16K keys in 8 bits, but each part costs the fold: 1 x 32K keys in
// 8 bits 24.5, 25.4, 32.4.)
// The kernels of a call each make the plan for themselves and have to agree, or the fold reads parts that nobody wrote: floating-point operations are rounded one by one, as they are
// written, not fused where a kernel's code happens to suggest it.  (In whole numbers a step of 16 sequences of five tokens takes 38.3 us for 37.7.)
// Tiles that are cut have fewer than steps / part + 1 parts: all of them together at most share.slots(tiles).
constexpr int kPartStep = 128, kUnits = 256;   // keys; compute units
constexpr int steps_of(int keys) { return (keys + kPartStep - 1) / kPartStep; }
struct Share {
  int most_per_unit;   // workgroups that a compute unit holds, 0: keys are not shared out
  int rounds;          // at most
  int item, fold, part;   // costs of an item beside its steps, of the fold, and of a part there, in sixteenths of a step
  constexpr int most() const { return kUnits * most_per_unit * rounds; }   // items that cutting adds
  constexpr int slots(int64_t tiles) const { return most() + (int)(tiles < most() ? tiles : most()); }
};
constexpr int step_time(int per_unit) { return per_unit <= 1 ? 16 : per_unit == 2 ? 28 : per_unit == 3 ? 41 : 54; }
constexpr int ceil_div(int n, int d) {   // of n < 2^24: the float quotient is at least the whole one
  const int q = (int)((float)n / (float)d);
  return q * d < n ? q + 1 : q;
}
constexpr int part_keys(int64_t work, int64_t tiles, int longest, const Share& share) {
#if defined(__clang__)
#pragma clang fp contract(off)
#endif
  // (As many keys as a sequence has at most.  No grid has 2^24 tiles: only sequences that overlap do, and for fewer work is below 2^47.)
  if (share.most_per_unit <= 0 || work <= 0 || tiles >= (1 << 24)) return kPosLimit;
  int unit = 0;   // work is counted in 2^unit steps, rounded up, which 24 bits hold (one token of 32 heads on 2^21 keys 1.2 ms; left uncut 22.5)
  while (work >= (1 << 24)) {
    work = (work + 1) >> 1;
    longest = (longest + 1) >> 1;
    unit++;
  }
  const int cost_item = share.item >> unit, cost_fold = share.fold >> unit, cost_part = share.part >> unit;
  const int w = (int)work, n_tiles = (int)tiles, most = share.most_per_unit, at_once = kUnits * most, all_busy = step_time(most);
  const int full = n_tiles / at_once, rest = n_tiles - full * at_once;
  const float each = (float)longest, rounds = (float)full * (each * (float)all_busy + (float)cost_item) + (rest > 0 ? each * (float)step_time((rest + kUnits - 1) / kUnits) + (float)cost_item : 0.f);
  const float even = ((float)w * (float)all_busy + (float)n_tiles * (float)cost_item) / (float)at_once + 8.f * each;
  const float alone = 16.f * each + (float)cost_item, at_least = even > alone ? even : alone;
  float best = rounds < at_least ? rounds : at_least;
  int part = kPosLimit;
  for (int c = 1; c < most + share.rounds; c++) {   // (more rounds than one where every unit is full)
    const int per_unit = c < most ? c : most, r = c < most ? 1 : c - most + 1, n = kUnits * per_unit * r - n_tiles / 2;
    if (n <= 0) continue;
    const int least = ceil_div(w, n), steps = least < 2 ? 2 : least;
    if (steps >= longest) continue;
    const float shared = r == 1 ? (float)(steps * step_time(per_unit) + cost_item)
                                : ((float)w * (float)all_busy + ((float)w / (float)steps + (float)(n_tiles / 2)) * (float)cost_item) / (float)at_once + 8.f * (float)steps;
    const float time = shared + (float)(cost_fold + cost_part * ceil_div(longest, steps));
    if (time < best) {
      best = time;
      part = (steps << unit) * kPartStep;
    }
  }
  return part;
}
constexpr int parts_of(int keys, int part) { return keys <= part ? 1 : (keys - 1) / part + 1; }

// Row tiles that the sequences of `tokens` tokens have at most, `group` rows a token: each has at most one that is not full, and over + 1 rows at least for
// a tile (a class that leaves rows out leaves out half a tile at most); where the most rows are one tile's, no sequence has two.
constexpr int64_t most_tiles(int64_t tokens, int64_t n_seqs, int64_t group, RowClass c) {
  const int64_t rows = tokens * group, some = rows / (c.over + 1), full = c.most <= c.tile ? n_seqs : rows / c.tile + n_seqs;
  return some < full ? some : full;
}

// How a call is launched: one launch for each class of sequences.
// Waves a SIMD of the kernel for tiles of 16 * rt rows, which are workgroups (of four waves) a compute unit.
constexpr int paged_few_waves(int D, bool f8, int rt) { return D == 128 ? (rt == 1 && f8 ? 3 : 2) : rt == 1 ? 4 : 3; }
constexpr int kManyRows = 256;   // rows of the tiles of sequences with many
struct PagedLaunch {
  int n;
  struct Part {
    RowClass rows;
    Share share;     // where a workspace is there
    int64_t tiles;   // of all sequences and K/V heads, at most
    int64_t parts;   // of a tile, at most
    // Workgroups with an item, at most, where the keys are shared out by `with` (the share above, or none).
    int64_t items(const Share& with) const {
      const int64_t cut = tiles + with.most(), whole = tiles * (with.most() > 0 ? parts : 1);
      return cut < whole ? cut : whole;
    }
    int64_t floats(int D) const { return (int64_t)share.slots(tiles) * rows.tile * (D + 1); }   // of the workspace
  } part[2];
};
// The launches of a call.  The lengths are not known here, so it goes by the average rows of a sequence and K/V head: up to 32, sequences are taken to be
// of single tokens and drafts, and workgroups of 16 or 32 rows serve them all; a lone sequence of more is one of many rows; several are a mixture,
// a launch for either kind.
inline PagedLaunch paged_launch(int64_t tokens, int64_t n_seqs, int64_t max_keys, int Hkv, int gq, int D, bool f8) {
  PagedLaunch l;
  const int64_t rows = tokens * gq;
  constexpr int any = 0x7fffffff;
  const RowClass few16 = {16, 0, any}, few32 = {32, 0, any}, many = {kManyRows, 0, any};
  const int few = gq <= 4 ? 16 : 32;   // rows of few tokens in a mixture: 16 / gq tokens (4 at groups of 4), 32 / gq beyond (4 at 8, 2 at 16, none above 32)
  const RowClass only_few = {few, 0, few}, only_many = {kManyRows, few, any};
  const bool mixed = rows > 32 * n_seqs && n_seqs > 1;
  l.n = mixed ? 2 : 1;
  l.part[0].rows = mixed ? only_few : rows <= 16 * n_seqs ? few16 : rows <= 32 * n_seqs ? few32 : many;
  l.part[1].rows = only_many;
  for (int i = 0; i < l.n; i++) {
    PagedLaunch::Part& c = l.part[i];
    c.tiles = most_tiles(tokens, n_seqs, gq, c.rows) * Hkv;
    // Workgroups that the registers of each kernel allow a compute unit; what an item, the fold and its parts cost, measured.  A second round only
    // for launches of few rows that may have more row tiles than a part of the first: the launch has workgroups for all that its plan may choose, and
    // those without an item cost 2 us a round of theirs (a mixture of 527 tokens of 16 sequences 99 us with 1300 of them, 108 with 3800).
    const int per_unit = c.rows.tile == kManyRows ? 1 : paged_few_waves(D, f8, c.rows.tile / 16);
    const int rounds = c.rows.tile == kManyRows || 2 * c.tiles <= kUnits * per_unit ? 1 : 2;
    const Share cut = c.rows.tile == kManyRows ? Share{1, 1, 20, 32, 2} : Share{per_unit, rounds, 36, 64, 2};
    const int64_t two_steps = (max_keys + 2 * kPartStep - 1) / (2 * kPartStep);
    c.parts = two_steps < 1 ? 1 : two_steps;
    c.share = c.parts == 1 ? Share{0, 0, 0, 0, 0} : cut;
  }
  return l;
}

}  // namespace tr
