// Which kernels weigh the keys of a call (tr_cache_weigh).  Plain C++, tested on the host.
#pragma once
#include "paged_plan.h"

namespace tr {

constexpr int kFewKeys = 256;    // of an item of few rows: 64 a wave
constexpr int kApartRows = 128;  // most rows of a sequence and K/V head that the first of two launches takes

// The lengths lie in device memory, so the launch goes by the call's tokens (`tokens`, of `n` sequences; `gq` query heads a K/V head) and by the keys that the table has room for.
enum WeighForm {
  kWeighFew,     // the kernel for few rows, 16 at a time, for all sequences
  kWeighMany,    // the one for many rows, 32 at a time, for all
  kWeighMixed,   // both in one launch, the first for sequences of up to 32 rows
  kWeighApart    // a launch of each, the first for sequences of up to kApartRows rows
};
// More than 32 rows on average: many in a lone sequence, otherwise a mixture, of which the launch cannot know that it is none (us, all of them as many / as a mixture: 7 sequences of 16K keys with a prompt of 300
// 295 / 82, 3 of 30K with one of 512 389 / 172, 5 of 1000 with one of 500 54 / 22; 2 of 1000 tokens on 8000 keys 139 / 140, 7 of 256 on 256 13.8 / 14.1).
// Few on average: `most` is what one sequence has if all others have a token.  Up to 32, as in a decode step, few it is.  More may be drafts, which the kernel for few rows serves best, or a prompt among single tokens, which
// it would go through 16 rows at a time for every 64 keys, all of them on one XCD: both kernels then, in one launch where the table has room for few keys; else in two, where the first has twice the waves for its loads.
// us as few / in one launch / in two, 8 K/V heads of 128 for 32 (figures of the form taken in brackets):
//   64 sequences of 16K keys, a prompt of 440 1111 / 507 / (507), of up to 16K in 8 bits 916 / 215 / (201); 32 of 8K, 200 269 / 125 / (138); 16 of 300, 97 29.5 / (12.1) / 16, with room for 32K keys 29.2 / 12.1 / (15.6)
//   drafts: 64 of 4 on 4K in 8 bits (three quarters to all of it) 47 / 60 / (50), 16 of 7 on 16K in 8 bits 58.6 / 72 / (60.7), 16 of 5 on 400 7.1 / (7.3) / 9.0, with room for 32K keys 7.1 / 7.3 / (8.8)
//   64 of 4K, a prompt of 30 (118) / 116 / 120.
// (Where some sequences have no tokens one may have more than `most`: up to as many tokens as there are sequences then go as few.)
constexpr WeighForm weigh_form(int64_t tokens, int64_t n, int64_t gq, int64_t Hkv, int64_t max_keys) {
  const int64_t rows = tokens * gq, most = (tokens - n + 1) * gq;
  if (rows > 32 * n) return n == 1 ? kWeighMany : kWeighMixed;
  if (most <= 32) return kWeighFew;
  if (n * Hkv * ((max_keys + kFewKeys - 1) / kFewKeys) <= 512) return kWeighMixed;
  return most <= kApartRows ? kWeighFew : kWeighApart;
}

}  // namespace tr
