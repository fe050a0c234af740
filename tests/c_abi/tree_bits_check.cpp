// tree_bits() of csrc/paged_plan.h on the host: the bits are those of the definition, key by key, and no word outside the row is read (each row is an allocation of its own, under a sanitizer).
#include <stdio.h>
#include <stdlib.h>

#include <memory>
#include <random>

#include "paged_plan.h"

int main() {
  std::mt19937_64 rng(5);
  auto any = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  for (int round = 0; round < 200000; round++) {
    const int words = (int)any(1, 5), n = (int)any(0, 170), len = (int)any(0, 400);
    const bool far = round % 10 == 0;
    tr::Sequence q = {0, n, len, far ? (int)any(-(1 << 30), (1 << 30) - 1) : (int)any(-200, 500)};
    std::unique_ptr<unsigned[]> row(new unsigned[words]);
    for (int i = 0; i < words; i++) row[i] = (unsigned)rng();
    const int key0 = far ? (int)any(0, (1 << 30) - 32) : (int)any(0, 420), cut = (int)any(0, 3) ? tr::visible_to_any(q) : (int)any(0, tr::visible_to_any(q));
    const unsigned bits = tr::tree_bits(row.get(), words, q, key0, cut);
    for (int i = 0; i < 32; i++) {
      const int64_t key = (int64_t)key0 + i, j = key - q.pos;
      const bool seen = key < cut && (j < 0 || (j < n && j < 32 * words && (row[j / 32] >> (j % 32) & 1)));
      if (seen != (bits >> i & 1)) { printf("FAILED: round %d, key %d + %d\n", round, key0, i); return 1; }
      if (key < q.len && key < tr::visible_to_all(q) && key < cut && !seen) { printf("FAILED: round %d, a key in front of the drafts\n", round); return 1; }
    }
  }
  printf("tree bits ok\n");
  return 0;
}
