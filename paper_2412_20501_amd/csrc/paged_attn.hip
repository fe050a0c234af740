// Launches of the attention on a paged cache.
#include "paged_launch.h"

namespace tr {

constexpr int kUnits = 256;   // compute units

#define TR_PAGED(D, F8) extern template hipError_t launch_paged_form<D, F8>(PagedParams&, const PagedLaunch&, float*, hipStream_t);
TR_PAGED(64, false) TR_PAGED(64, true) TR_PAGED(128, false) TR_PAGED(128, true)
#undef TR_PAGED

// The launches of a call.  The lengths are not known here, so it goes by the average rows of a sequence and K/V head: up to 32, sequences are taken to be
// of single tokens and drafts, and workgroups of 16 or 32 rows serve them all; a lone sequence of more is one of many rows; several are a mixture,
// a launch for either kind.
PagedLaunch paged_launch(int64_t tokens, int64_t n_seqs, int64_t max_keys, int Hkv, int gq, int D) {
  PagedLaunch l;
  const int64_t rows = tokens * gq;
  constexpr int any = 0x7fffffff;
  const RowClass few16 = {16, 0, any}, few32 = {32, 0, any}, many = {kManyRows, 0, any}, only_few = {32, 0, 32}, only_many = {kManyRows, 32, any};
  const bool mixed = rows > 32 * n_seqs && n_seqs > 1;
  l.n = mixed ? 2 : 1;
  l.part[0].rows = mixed ? only_few : rows <= 16 * n_seqs ? few16 : rows <= 32 * n_seqs ? few32 : many;
  l.part[1].rows = only_many;
  for (int i = 0; i < l.n; i++) {
    PagedLaunch::Part& c = l.part[i];
    c.tiles = most_tiles(tokens, n_seqs, gq, c.rows) * Hkv;
    // workgroups that run at once: what the registers of each kernel allow a compute unit (paged_few_waves); what an item and the fold cost, measured
    const Share cut = c.rows.tile == kManyRows ? Share{kUnits, 2, 20, 32} : Share{kUnits * paged_few_waves(D, c.rows.tile / 16), 4, 5, 10};
    c.share = max_keys <= 2 * kPartStep ? Share{0, 0, 0, 0} : cut;
  }
  return l;
}

hipError_t launch_paged_attn(PagedParams& p, const PagedLaunch& l, int D, bool f8, float* workspace, hipStream_t stream) {
  if (D == 128) return f8 ? launch_paged_form<128, true>(p, l, workspace, stream) : launch_paged_form<128, false>(p, l, workspace, stream);
  return f8 ? launch_paged_form<64, true>(p, l, workspace, stream) : launch_paged_form<64, false>(p, l, workspace, stream);
}

}  // namespace tr
