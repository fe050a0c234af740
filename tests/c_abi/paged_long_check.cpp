// csrc/paged_plan.h on the host: sequences of up to 2^30 keys are shared out as shorter ones are, within the scratch.
#include <stdio.h>
#include <stdlib.h>

#include <initializer_list>

#include "paged_plan.h"

#define EXPECT(x) do { if (!(x)) { printf("FAILED line %d: %s (tiles %d, keys %d, per unit %d)\n", __LINE__, #x, tiles, keys, share.most_per_unit); exit(1); } } while (0)

int main() {
  const tr::Share shares[] = {{1, 1, 20, 32, 2}, {2, 1, 36, 64, 2}, {3, 1, 36, 64, 2}, {4, 2, 36, 64, 2}};   // of many rows; of few
  for (const tr::Share& share : shares)
    for (int tiles : {1, 2, 3, 8, 24, 64, 100, 128}) {
      int64_t was = 0;   // parts of the shorter ones
      for (int64_t k : {(int64_t)100000, (int64_t)1000000, (int64_t)2096961, (int64_t)2097024, (int64_t)2097152, (int64_t)2097153, (int64_t)4194305, (int64_t)12345678, (int64_t)33554432, (int64_t)134217729, (int64_t)268435456,
                        (int64_t)536870913, (int64_t)1 << 30}) {
        const int keys = (int)k, longest = tr::steps_of(keys);
        const int part = tr::part_keys((int64_t)tiles * longest, tiles, longest, share);
        EXPECT(part > 0 && part % tr::kPartStep == 0 && part < keys);
        const int64_t parts = tr::parts_of(keys, part);
        EXPECT((parts - 1) * part < keys && parts * part >= keys);
        EXPECT(tiles * parts <= share.slots(tiles) && tiles * parts <= tiles + share.most());
        // at least half the units have a part, and a longer sequence has hardly fewer than a shorter one
        EXPECT(tiles * parts >= tr::kUnits / 2);
        EXPECT(parts * 10 >= was * 9);
        was = parts;
      }
    }
  // one long sequence among short ones: still cut
  for (const tr::Share& share : shares) {
    const int tiles = 800, keys = 1 << 27, longest = tr::steps_of(keys);
    const int part = tr::part_keys(8 * (int64_t)longest + 792 * 8, tiles, longest, share);
    if (tiles / 2 >= share.most()) EXPECT(part == tr::kPosLimit);   // 800 / 2 >= 256: there is no room for parts beside the tiles' halves
    else EXPECT(part < keys / 8);
  }
  // more tiles than a grid has: only sequences that overlap have them
  const tr::Share share = shares[0];
  const int tiles = 1 << 24, keys = 1 << 30;
  for (int64_t work : {(int64_t)1, (int64_t)1 << 40, (int64_t)1 << 62, (int64_t)-5}) EXPECT(tr::part_keys(work, tiles, tr::steps_of(keys), share) == tr::kPosLimit);
  printf("long keys ok\n");
  return 0;
}
