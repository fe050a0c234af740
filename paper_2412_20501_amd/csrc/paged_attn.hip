// Launches of the attention on a paged cache.
#include "paged_launch.h"

namespace tr {

#define TR_PAGED(D, F8) extern template hipError_t launch_paged_form<D, F8>(const PagedParams&, const PagedLaunch&, hipStream_t);
TR_PAGED(64, false) TR_PAGED(64, true) TR_PAGED(128, false) TR_PAGED(128, true)
#undef TR_PAGED

// The form of a launch.  The lengths are not known here, so it goes by the average rows of a sequence and K/V head: up to 32, sequences are taken to be
// of single tokens and drafts, and their keys are read by workgroups of 16 or 32 rows; more, and there are chunks of prompts among them.
PagedLaunch paged_launch(int64_t tokens, int64_t n_seqs, int64_t max_keys, int Hkv, int gq, int D) {
  PagedLaunch l;
  const int64_t rows = tokens * gq;
  l.tile = rows <= 16 * n_seqs ? TileRows{16, 16} : rows <= 32 * n_seqs ? TileRows{32, 32} : kMixed;
  l.tiles = most_tiles(tokens, n_seqs, gq, l.tile) * Hkv;
  l.target = max_keys <= 256 ? 0 : l.tile.many == kMixed.many ? 256 : l.tile.many == 32 ? 512 : 768;
  return l;
}

hipError_t launch_paged_attn(const PagedParams& p, const PagedLaunch& l, int D, bool f8, hipStream_t stream) {
  if (D == 128) return f8 ? launch_paged_form<128, true>(p, l, stream) : launch_paged_form<128, false>(p, l, stream);
  return f8 ? launch_paged_form<64, true>(p, l, stream) : launch_paged_form<64, false>(p, l, stream);
}

}  // namespace tr
