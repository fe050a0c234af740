// Launches of one head dim and type of the pages (one .hip each, so that they compile side by side).
#pragma once
#include <algorithm>

#include "launch_lds.h"
#include "paged_tile.h"

namespace tr {
namespace {

template <int D, bool F8, bool OUT_F32>
hipError_t launch_half(const TreeParams& p, std::atomic<uint64_t>& raised, dim3 items, hipStream_t stream) {
  return launch_lds(paged_half_kernel<D, F8, OUT_F32, TreeParams>, raised, items, dim3(256), Tile<D, 4>::LDS, stream, p);
}
template <int D, bool F8, bool OUT_F32>
hipError_t launch_half(const PagedParams&, std::atomic<uint64_t>&, dim3, hipStream_t) { return hipErrorInvalidValue; }   // (trees alone have such rows)
template <int D, bool F8, bool OUT_F32, typename P>
hipError_t launch_out(P& p, const PagedLaunch& l, float* workspace, hipStream_t stream) {
  static std::atomic<uint64_t> raised[4];
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
    if (c.rows.tile == kManyRows) e = launch_lds(paged_many_kernel<D, F8, OUT_F32, P>, raised[0], items, dim3(512), Tile<D, 8>::LDS, stream, p);
    else if (c.rows.tile == kHalfRows) e = launch_half<D, F8, OUT_F32>(p, raised[3], items, stream);
    else if (c.rows.tile == 32) e = launch_lds(paged_few_kernel<D, F8, 2, OUT_F32, P>, raised[1], items, dim3(256), Few<D, F8, 2, 4>::LDS, stream, p);
    else e = launch_lds(paged_few_kernel<D, F8, 1, OUT_F32, P>, raised[2], items, dim3(256), Few<D, F8, 1, 4>::LDS, stream, p);
    if (e != hipSuccess) return e;
    if (p.share.most() == 0) continue;
    const unsigned cut = (unsigned)std::min<int64_t>(c.tiles, p.share.most());   // tiles that are cut, at most
    // Few tiles in more than eight parts each: shared (a tree of 100 rows on 2 heads of 64 and 24K keys, in 94 parts, 38 -> 22 us; but four of 256 rows on 8 heads and 8K keys, in eight, 56 -> 59).
    if (is_tree<P> && std::min<int64_t>(p.share.most() / cut, c.parts) > 8)
      e = launch_kernel(paged_fold_kernel<D, OUT_F32, is_tree<P>, P>, dim3(std::min(cut * (unsigned)(c.rows.tile * D / 256), 1024u)), dim3(256), 0, stream, p);
    else
      e = launch_kernel(paged_fold_kernel<D, OUT_F32, false, P>, dim3(std::min(cut * (unsigned)std::max(1, c.rows.tile * D / 1024 / fold_turns<P>), 1024u)), dim3(256), 0, stream, p);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

template <int D, bool F8, typename P>
hipError_t launch_paged_form(P& p, const PagedLaunch& l, float* workspace, hipStream_t stream) {
  return p.out_f32 ? launch_out<D, F8, true>(p, l, workspace, stream) : launch_out<D, F8, false>(p, l, workspace, stream);
}

}  // namespace tr
