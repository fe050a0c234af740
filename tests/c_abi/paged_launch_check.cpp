// csrc/paged_plan.h on the host: the launches of a call have a workgroup for every item that its plan makes of any lengths, and its scratch a slot for every cut one.
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <vector>

#include "paged_plan.h"

#define EXPECT(x) do { if (!(x)) { printf("FAILED line %d: %s (round %d)\n", __LINE__, #x, round); exit(1); } } while (0)

int main() {
  std::mt19937_64 rng(13);
  auto any = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  int mixtures = 0, cut_calls = 0;
  bool classes[6] = {};   // of rows, that were met: few 16, few 32, many; a mixture's few 16, few 32, many behind either
  for (int round = 0; round < 60000; round++) {
    const int n = (int)any(1, round % 3 ? 12 : 300), gq = (int)any(1, round % 7 ? 9 : 80), Hkv = (int)any(1, 24), page_size = 16, max_pages = (int)any(1, (int64_t)1 << any(0, 13));
    const int kind = (int)any(0, 3);   // single tokens, drafts, prompts, one prompt among single tokens
    std::vector<int> start(n + 1), len(n), table(1);
    int at = 0;
    for (int b = 0; b < n; b++) {
      start[b] = at;
      at += (int)(kind == 0 ? any(0, 1) : kind == 1 ? any(0, 8) : kind == 2 ? any(0, 900) : b == n / 2 ? any(0, 2000) : 1);
      len[b] = (int)any(0, (int64_t)max_pages * page_size);
      if (round % 4 == 0) len[b] = max_pages * page_size;
    }
    start[n] = at;
    const int tokens = at + (int)any(0, 3), D = round % 2 ? 64 : 128;
    if (tokens == 0) continue;
    tr::Sequences s = {};
    s.table = table.data(); s.kv_len = len.data(); s.q_start = start.data(); s.q_pos = nullptr;
    s.n = n; s.max_pages = max_pages; s.tokens = tokens; s.n_pages = 1; s.page_size = page_size;
    const tr::PagedLaunch l = tr::paged_launch(tokens, n, (int64_t)max_pages * page_size, Hkv, gq, D, round % 5 == 0);
    EXPECT(l.n == 1 || l.n == 2);
    mixtures += l.n == 2;
    for (int i = 0; i < l.n; i++) {
      const tr::RowClass r = l.part[i].rows;
      classes[l.n == 1 ? (r.tile == 16 ? 0 : r.tile == 32 ? 1 : 2) : i == 1 ? 5 : r.tile == 16 ? 3 : 4] = true;
    }
    for (int b = 0; b < n; b++) {   // every sequence's rows are one launch's
      const int rows = (start[b + 1] - start[b]) * gq;
      int in = 0;
      for (int i = 0; i < l.n; i++) {
        const int t = tr::tiles_of(rows, l.part[i].rows);
        in += t > 0;
        EXPECT(t == 0 || (int64_t)t * l.part[i].rows.tile >= rows);
      }
      EXPECT(in == (rows > 0));
    }
    for (int i = 0; i < l.n; i++)
      for (bool shared : {true, false}) {
        const tr::PagedLaunch::Part& c = l.part[i];
        const tr::Share share = shared ? c.share : tr::Share{0, 0, 0, 0, 0};
        int64_t work = 0, tiles = 0, items = 0, slots = 0, cut = 0;
        int longest = 0;
        for (int b = 0; b < n; b++) {
          const tr::Sequence q = tr::sequence(s, b);
          const int t = tr::tiles_of(q.n * gq, c.rows);
          work += (int64_t)t * tr::steps_of(q.len);
          tiles += t;
          if (t > 0 && tr::steps_of(q.len) > longest) longest = tr::steps_of(q.len);
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
        EXPECT(cut <= share.most() || share.most() == 0);
        EXPECT(shared || cut == 0);
        cut_calls += cut > 0;
        // item `id` of the launch, as the kernels number them: each has a workgroup
        const int64_t groups = (c.items(share) + 7) / 8 * 8, each = (items + 7) >> 3;
        EXPECT(8 * each <= groups || items == 0);
      }
  }
  for (bool met : classes)
    if (!met) { printf("FAILED: a class of rows was not met\n"); return 1; }
  if (mixtures < 1000 || cut_calls < 1000) { printf("FAILED: %d mixtures, %d cut\n", mixtures, cut_calls); return 1; }
  printf("launches ok\n");
  return 0;
}
