// Attention on a paged cache at head dim 64, pages of bf16.
#include "paged_launch.h"

namespace tr {
template hipError_t launch_paged_form<64, false>(PagedParams&, const PagedLaunch&, float*, hipStream_t);
}  // namespace tr
