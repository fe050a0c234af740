// Launches of the attention on a paged cache.
#include "paged_launch.h"

namespace tr {

#define TR_PAGED(D, F8)                                                                                                  \
  extern template hipError_t launch_paged_form<D, F8>(PagedParams&, const PagedLaunch&, float*, hipStream_t); \
  extern template hipError_t launch_paged_form<D, F8>(TreeParams&, const PagedLaunch&, float*, hipStream_t);
TR_PAGED(64, false) TR_PAGED(64, true) TR_PAGED(128, false) TR_PAGED(128, true)
#undef TR_PAGED

namespace {
template <typename P>
hipError_t launch(P& p, const PagedLaunch& l, int D, bool f8, float* workspace, hipStream_t stream) {
  if (D == 128) return f8 ? launch_paged_form<128, true>(p, l, workspace, stream) : launch_paged_form<128, false>(p, l, workspace, stream);
  return f8 ? launch_paged_form<64, true>(p, l, workspace, stream) : launch_paged_form<64, false>(p, l, workspace, stream);
}
}  // namespace

hipError_t launch_paged_attn(PagedParams& p, const PagedLaunch& l, int D, bool f8, float* workspace, hipStream_t stream) { return launch(p, l, D, f8, workspace, stream); }
hipError_t launch_paged_attn(TreeParams& p, const PagedLaunch& l, int D, bool f8, float* workspace, hipStream_t stream) { return launch(p, l, D, f8, workspace, stream); }

}  // namespace tr
