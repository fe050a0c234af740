// Attention of trees of drafted tokens on a paged cache at head dim 128, pages of e4m3.
#include "paged_launch.h"

namespace tr {
template hipError_t launch_paged_form<128, true>(TreeParams&, const PagedLaunch&, float*, hipStream_t);
}  // namespace tr
