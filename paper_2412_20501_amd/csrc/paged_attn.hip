// Launches of the attention on a paged cache.
#include "paged_attn_kernel.h"

namespace tr {

namespace {
template <int D, bool F8, bool OUT_F32>
hipError_t launch_form(const PagedParams& p, const PagedLaunch& l, hipStream_t stream) {
  const unsigned items = (unsigned)((l.tiles + p.target + 7) / 8 * 8);   // an eighth of the items for every XCD, rounded up
  const hipError_t e = launch_kernel(paged_few_kernel<D, F8, 1, OUT_F32>, dim3(items), dim3(256), Few<D, F8, 1>::LDS, stream, p);
  if (e != hipSuccess || p.target == 0) return e;
  const unsigned cut = (unsigned)(l.tiles < p.target ? l.tiles : p.target);   // a cut tile has two parts at least
  return launch_kernel(paged_fold_kernel<D, 16, OUT_F32>, dim3(cut, 16 * D / 1024), dim3(256), 0, stream, p);
}
}  // namespace

PagedLaunch paged_launch(int64_t tokens, int64_t n_seqs, int64_t max_keys, int Hkv, int gq, int D) {
  PagedLaunch l;
  l.rows = 16;
  l.tiles = most_tiles(tokens, n_seqs, gq, l.rows) * Hkv;
  l.target = max_keys > 256 ? 512 : 0;
  return l;
}

hipError_t launch_paged_attn(const PagedParams& p, const PagedLaunch& l, int D, bool f8, hipStream_t stream) {
#define TR_FORM(d, f) (p.out_f32 ? launch_form<d, f, true>(p, l, stream) : launch_form<d, f, false>(p, l, stream))
  if (D == 128) return f8 ? TR_FORM(128, true) : TR_FORM(128, false);
  return f8 ? TR_FORM(64, true) : TR_FORM(64, false);
#undef TR_FORM
}

}  // namespace tr
