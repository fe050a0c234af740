// Which kernels weigh the keys of a call, on the host: no sequence that may have many rows is left to the kernel for few, whatever the others, their number or the room of the page table.
#include <stdio.h>
#include <stdlib.h>

#include <random>

#include "weigh_plan.h"

#define EXPECT(x) do { if (!(x)) { printf("FAILED line %d: %s (%ld tokens, %ld sequences, group %ld, %ld heads, %ld keys)\n", __LINE__, #x, (long)tokens, (long)n, (long)gq, (long)Hkv, (long)keys); exit(1); } } while (0)

int main() {
  std::mt19937_64 rng(5);
  auto any = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  int met[4] = {};
  for (int round = 0; round < 20000; round++) {
    const int64_t n = any(1, (int64_t)1 << any(0, 10)), gq = any(1, round % 5 ? 8 : 32), Hkv = any(1, 32), keys = 16 * any(1, (int64_t)1 << any(0, 16));
    int64_t tokens = n;
    EXPECT(tr::weigh_form(tokens, n, gq, Hkv, keys) == tr::kWeighFew);   // a decode step
    bool left = false;
    for (int64_t more = 0; more < 300; more++) {   // n - 1 single tokens and a prompt
      tokens = n + more;
      const int64_t rows = (more + 1) * gq;
      const tr::WeighForm form = tr::weigh_form(tokens, n, gq, Hkv, keys);
      met[form]++;
      EXPECT(rows <= tr::kApartRows || form != tr::kWeighFew);
      EXPECT(rows > 32 || form == tr::kWeighFew);
      EXPECT(form != tr::kWeighApart || rows > tr::kApartRows);
      EXPECT(n > 1 || form == (rows <= 32 ? tr::kWeighFew : tr::kWeighMany));
      EXPECT(n == 1 || form != tr::kWeighMany);   // (others beside it may have single tokens)
      EXPECT(!left || form != tr::kWeighFew);   // a token more never goes back
      left |= form != tr::kWeighFew;
    }
  }
  const int64_t tokens = 0, n = 0, gq = 0, Hkv = 0, keys = 0;
  for (int i = 0; i < 4; i++) EXPECT(met[i] > 1000);
  printf("weigh forms ok\n");
  return 0;
}
