// Launches of one head dim and type of the pages (one .hip each, so that they compile side by side).
#pragma once
#include <algorithm>
#include <atomic>

#include "paged_tile.h"

namespace tr {
namespace {

// A launch that asks for more LDS than the default limit: raised once for each device and kernel.
template <typename Kernel, typename... Args>
hipError_t launch_lds(Kernel kernel, std::atomic<uint64_t>& raised, dim3 grid, dim3 block, int lds_bytes, hipStream_t stream, Args... args) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? (uint64_t)1 << dev : 0;
  if (!(raised.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes);
    if (e != hipSuccess) return e;
    raised.fetch_or(bit, std::memory_order_release);
  }
  return launch_kernel(kernel, grid, block, lds_bytes, stream, args...);
}

template <int D, bool F8, bool OUT_F32>
hipError_t launch_out(PagedParams& p, const PagedLaunch& l, float* workspace, hipStream_t stream) {
  static std::atomic<uint64_t> raised[3];
  for (int i = 0; i < l.n; i++) {
    const PagedLaunch::Part& c = l.part[i];
    p.rows = c.rows;
    p.share = workspace ? c.share : Share{0, 0, 0, 0, 0};
    p.slots = p.share.slots(c.tiles);
    p.part_out = workspace;
    p.part_lse = workspace ? workspace + (int64_t)p.slots * c.rows.tile * D : nullptr;
    if (workspace) workspace += c.floats(D);
    // Workgroups beyond those that have an item cost a microsecond for every four hundred.  (An eighth of the items for every XCD, rounded up.)
    const dim3 items((unsigned)((c.items(p.share) + 7) / 8 * 8));
    hipError_t e;
    if (c.rows.tile == kManyRows) e = launch_lds(paged_many_kernel<D, F8, OUT_F32>, raised[0], items, dim3(512), Tile<D>::LDS, stream, p);
    else if (c.rows.tile == 32) e = launch_lds(paged_few_kernel<D, F8, 2, OUT_F32>, raised[1], items, dim3(256), Few<D, F8, 2, 4>::LDS, stream, p);
    else e = launch_lds(paged_few_kernel<D, F8, 1, OUT_F32>, raised[2], items, dim3(256), Few<D, F8, 1, 4>::LDS, stream, p);
    if (e != hipSuccess) return e;
    if (p.share.most() == 0) continue;
    const unsigned cut = (unsigned)std::min<int64_t>(c.tiles, p.share.most());   // tiles that are cut, at most
    e = launch_kernel(paged_fold_kernel<D, OUT_F32>, dim3(std::min(cut * (unsigned)std::max(1, c.rows.tile * D / 1024), 1024u)), dim3(256), 0, stream, p);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

template <int D, bool F8>
hipError_t launch_paged_form(PagedParams& p, const PagedLaunch& l, float* workspace, hipStream_t stream) {
  return p.out_f32 ? launch_out<D, F8, true>(p, l, workspace, stream) : launch_out<D, F8, false>(p, l, workspace, stream);
}

}  // namespace tr
