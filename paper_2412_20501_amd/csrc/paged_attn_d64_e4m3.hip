// Attention on a paged cache at head dim 64, pages of e4m3.
#include "paged_launch.h"

namespace tr {
template hipError_t launch_paged_form<64, true>(PagedParams&, const PagedLaunch&, float*, hipStream_t);
}  // namespace tr
