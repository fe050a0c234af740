// Attention on a paged cache at head dim 128, pages of bf16.
#include "paged_launch.h"

namespace tr {
template hipError_t launch_paged_form<128, false>(PagedParams&, const PagedLaunch&, float*, hipStream_t);
}  // namespace tr
