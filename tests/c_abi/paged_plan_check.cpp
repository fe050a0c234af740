// csrc/paged_plan.h on the host: whatever the arrays hold, nothing outside of them and of the pages is addressed, and parts stay within the scratch.
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <vector>

#include "paged_plan.h"

#define EXPECT(x) do { if (!(x)) { printf("FAILED line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

int main() {
  std::mt19937_64 rng(7);
  auto any = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  const int odd[] = {0, 1, -1, 2147483647, -2147483647 - 1, 1 << 30, -(1 << 30), 15, 16, 17};
  for (int round = 0; round < 4000; round++) {
    const int n = (int)any(1, 70), page_size = 16 * (int)any(1, 20), max_pages = (int)any(0, 40), n_pages = (int)any(1, 50), gq = (int)any(1, 16), Hkv = (int)any(1, 8);
    const bool wild = round % 2, with_pos = round % 3 == 0, causal = round % 5 != 0;
    const int tokens = (int)any(0, 600);
    std::vector<int> table((size_t)n * max_pages + 1), len(n), start(n + 1), pos(n);
    for (int& x : table) x = any(0, 9) == 0 ? odd[any(0, 9)] : (int)any(0, n_pages - 1);
    int at = 0;
    for (int b = 0; b < n; b++) {
      len[b] = wild && any(0, 3) == 0 ? odd[any(0, 9)] : (int)any(0, (int64_t)max_pages * page_size);
      start[b] = wild && any(0, 3) == 0 ? odd[any(0, 9)] : at;
      at += (int)any(0, (tokens - at) / 2);
      pos[b] = wild && any(0, 3) == 0 ? odd[any(0, 9)] : (int)any(-100, 1000);
    }
    start[n] = wild && any(0, 3) == 0 ? odd[any(0, 9)] : at;
    tr::Sequences s;
    s.table = table.data(); s.kv_len = len.data(); s.q_start = start.data(); s.q_pos = with_pos ? pos.data() : nullptr;
    s.table_stride = max_pages; s.n = n; s.max_pages = max_pages; s.tokens = tokens; s.n_pages = n_pages; s.page_size = page_size;
    s.by_page = tr::make_divisor((unsigned)page_size);
    for (tr::RowClass tile : {tr::RowClass{16, 0, 1 << 30}, tr::RowClass{32, 0, 1 << 30}, tr::RowClass{32, 0, 32}, tr::RowClass{256, 32, 1 << 30}})
      for (int per_unit : {0, 1, 3}) {
        const tr::Share share = {per_unit, 1 + round % 4, 5 * (round % 7), 10 * (round % 5), round % 3};
        int64_t work = 0, tiles = 0;
        int longest = 0;
        for (int b = 0; b < n; b++) {
          const tr::Sequence q = tr::sequence(s, b);
          EXPECT(q.start >= 0 && q.n >= 0 && q.start + q.n <= tokens && q.len >= 0 && q.len <= max_pages * page_size);
          EXPECT(q.pos >= -(1 << 30) && q.pos < (1 << 30));
          work += (int64_t)tr::tiles_of(q.n * gq, tile) * tr::steps_of(q.len);
          tiles += tr::tiles_of(q.n * gq, tile);
          if (tr::tiles_of(q.n * gq, tile) > 0 && tr::steps_of(q.len) > longest) longest = tr::steps_of(q.len);
          int before = 0;
          for (int t = 0; t < q.n; t++) {
            const int v = tr::visible(q, t, causal);
            EXPECT(v >= 0 && v <= q.len && v >= before);
            before = v;
          }
          for (int i = 0; i < 20 && q.len > 0; i++) {
            const int c = (int)any(0, q.len - 1);
            const tr::Slot at_c = tr::slot_of(s, b, c);   // (a read outside the table is the sanitizer's to find)
            EXPECT(at_c.page >= -1 && at_c.page < n_pages && at_c.slot == c % page_size);
          }
        }
        if (!wild) EXPECT(tiles <= tr::most_tiles(tokens, n, gq, tile));
        const int part = tr::part_keys(work * Hkv, tiles * Hkv, longest, share);
        EXPECT(part > 0 && (part == tr::kPosLimit || part % tr::kPartStep == 0) && (per_unit > 0 || part == tr::kPosLimit));
        int64_t items = 0, slots = 0;
        for (int b = 0; b < n; b++) {
          const tr::Sequence q = tr::sequence(s, b);
          const int parts = tr::parts_of(q.len, part), mine = tr::tiles_of(q.n * gq, tile) * Hkv * parts;
          EXPECT(parts >= 1 && (int64_t)parts * part >= q.len && (parts == 1 || (int64_t)(parts - 1) * part < q.len));
          items += mine;
          if (parts > 1) slots += mine;
        }
        EXPECT(slots <= share.slots(tiles * Hkv));
        EXPECT(items <= tiles * Hkv + share.most());
      }
  }
  printf("paged plan ok\n");
  return 0;
}
