// The launch of a tree's call, on the host: it serves every sequence's rows, has a workgroup for every item that its plan makes of any lengths, and its scratch a slot for every cut one.
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <vector>

#include "paged_plan.h"

#define EXPECT(x) do { if (!(x)) { printf("FAILED line %d: %s (round %d)\n", __LINE__, #x, round); exit(1); } } while (0)

int main() {
  std::mt19937_64 rng(17);
  auto any = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  int cut_calls = 0, cut_of_128 = 0, tiles_met[4] = {};
  for (int round = 0; round < 30000; round++) {
    const int n = (int)any(1, round % 3 ? 12 : 300), gq = (int)any(1, round % 7 ? 9 : 80), Hkv = (int)any(1, 24), max_pages = (int)any(1, (int64_t)1 << any(0, 13)), drafts = (int)any(0, 1 << any(0, 8));
    std::vector<int> start(n + 1), len(n), table(1);
    for (int b = 0; b < n; b++) {
      start[b + 1] = start[b] + (int)(round % 2 ? drafts : any(0, drafts));
      len[b] = (int)any(0, (int64_t)max_pages * 16);
    }
    const int tokens = start[n] + (int)any(0, 3), D = round % 2 ? 64 : 128;
    if (tokens == 0) continue;
    tr::Sequences s = {};
    s.table = table.data(); s.kv_len = len.data(); s.q_start = start.data();
    s.n = n; s.max_pages = max_pages; s.tokens = tokens; s.n_pages = 1; s.page_size = 16;
    const tr::PagedLaunch l = tr::paged_launch(tokens, n, (int64_t)max_pages * 16, Hkv, gq, D, round % 5 == 0, true);
    EXPECT(l.n == 1);
    const tr::PagedLaunch::Part& c = l.part[0];
    tiles_met[c.rows.tile == 16 ? 0 : c.rows.tile == 32 ? 1 : c.rows.tile == 128 ? 2 : 3]++;
    for (bool shared : {true, false}) {
      const tr::Share share = shared ? c.share : tr::Share{0, 0, 0, 0, 0};
      int64_t work = 0, tiles = 0, items = 0, slots = 0, cut = 0;
      int longest = 0;
      for (int b = 0; b < n; b++) {
        const tr::Sequence q = tr::sequence(s, b);
        const int t = tr::tiles_of(q.n * gq, c.rows);
        EXPECT((int64_t)t * c.rows.tile >= (int64_t)q.n * gq);
        work += (int64_t)t * tr::steps_of(q.len);
        tiles += t;
        if (t > 0 && tr::steps_of(q.len) > longest) longest = tr::steps_of(q.len);
        EXPECT(0 <= tr::visible_to_all(q) && tr::visible_to_all(q) <= tr::visible_to_any(q) && tr::visible_to_any(q) <= q.len);
      }
      work *= Hkv;
      tiles *= Hkv;
      EXPECT(tiles <= c.tiles);
      const int part = tr::part_keys(work, tiles, longest, share);
      for (int b = 0; b < n; b++) {
        const tr::Sequence q = tr::sequence(s, b);
        const int64_t mine = (int64_t)tr::tiles_of(q.n * gq, c.rows) * Hkv, parts = tr::parts_of(q.len, part);
        items += mine * parts;
        if (parts > 1) slots += mine * parts, cut += mine;
      }
      EXPECT(items <= c.items(share) && slots <= share.slots(c.tiles) && slots * c.rows.tile * (D + 1) <= c.floats(D));
      EXPECT(shared || cut == 0);
      cut_calls += cut > 0;
      cut_of_128 += cut > 0 && c.rows.tile == 128;
    }
  }
  if (cut_calls < 1000 || cut_of_128 < 100 || !tiles_met[0] || !tiles_met[1] || !tiles_met[2] || !tiles_met[3]) { printf("FAILED: %d cut, %d\n", cut_calls, cut_of_128); return 1; }
  printf("tree launches ok\n");
  return 0;
}
