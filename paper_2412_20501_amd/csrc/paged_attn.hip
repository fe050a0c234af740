// Launches of the attention on a paged cache.
#include "paged_launch.h"

namespace tr {

#define TR_PAGED(D, F8) extern template hipError_t launch_paged_form<D, F8>(PagedParams&, const PagedLaunch&, float*, hipStream_t);
TR_PAGED(64, false) TR_PAGED(64, true) TR_PAGED(128, false) TR_PAGED(128, true)
#undef TR_PAGED

// The launches of a call.  The lengths are not known here, so it goes by the average rows of a sequence and K/V head: up to 32, sequences are taken to be
// of single tokens and drafts, and workgroups of 16 or 32 rows serve them all; a lone sequence of more is one of many rows; several are a mixture,
// a launch for either kind.
PagedLaunch paged_launch(int64_t tokens, int64_t n_seqs, int64_t max_keys, int Hkv, int gq, int D, bool f8) {
  PagedLaunch l;
  const int64_t rows = tokens * gq;
  constexpr int any = 0x7fffffff;
  const RowClass few16 = {16, 0, any}, few32 = {32, 0, any}, many = {kManyRows, 0, any};
  const int few = gq <= 4 ? 16 : 32;   // in a mixture: four tokens
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
    c.parts = std::max<int64_t>(1, (max_keys + 2 * kPartStep - 1) / (2 * kPartStep));
    c.share = c.parts == 1 ? Share{0, 0, 0, 0, 0} : cut;
  }
  return l;
}

hipError_t launch_paged_attn(PagedParams& p, const PagedLaunch& l, int D, bool f8, float* workspace, hipStream_t stream) {
  if (D == 128) return f8 ? launch_paged_form<128, true>(p, l, workspace, stream) : launch_paged_form<128, false>(p, l, workspace, stream);
  return f8 ? launch_paged_form<64, true>(p, l, workspace, stream) : launch_paged_form<64, false>(p, l, workspace, stream);
}

}  // namespace tr
