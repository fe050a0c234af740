// Sums over the sequences of a call, taken by every wave for itself: which of them holds a launch's i-th item.  Params: what holds a Sequences `seq`.
#pragma once
#include "paged.h"

namespace tr {
namespace {

template <int CONTROL, int ROWS>
__device__ __forceinline__ int from_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CONTROL, ROWS, 0xf, false); }   // 0 where no lane is
__device__ __forceinline__ int wave_scan(int x) {   // sum over the lanes up to and including this one
  x += from_lane<0x111, 0xf>(x);   // rows of 16 lanes: from 1, 2, 4, 8 below,
  x += from_lane<0x112, 0xf>(x);
  x += from_lane<0x114, 0xf>(x);
  x += from_lane<0x118, 0xf>(x);
  x += from_lane<0x142, 0xa>(x);   // then a row's last lane to the next row,
  x += from_lane<0x143, 0xc>(x);   // and the lower half's to the upper
  return x;
}
template <int CONTROL, int ROWS>
__device__ __forceinline__ int64_t add_from(int64_t x) {
  return x + (int64_t)(((uint64_t)(unsigned)from_lane<CONTROL, ROWS>((int)(x >> 32)) << 32) | (unsigned)from_lane<CONTROL, ROWS>((int)x));
}
__device__ __forceinline__ int64_t wave_sum(int64_t x) {
  x = add_from<0x118, 0xf>(add_from<0x114, 0xf>(add_from<0x112, 0xf>(add_from<0x111, 0xf>(x))));
  x = add_from<0x143, 0xc>(add_from<0x142, 0xa>(x));
  return (int64_t)(((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), 63) << 32) | (unsigned)__builtin_amdgcn_readlane((int)x, 63));
}
__device__ __forceinline__ int wave_max(int x) {   // of numbers that are not negative
  x = max(x, from_lane<0x111, 0xf>(x));
  x = max(x, from_lane<0x112, 0xf>(x));
  x = max(x, from_lane<0x114, 0xf>(x));
  x = max(x, from_lane<0x118, 0xf>(x));
  x = max(x, from_lane<0x142, 0xa>(x));
  return __builtin_amdgcn_readlane(max(x, from_lane<0x143, 0xc>(x)), 63);
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// What the sums are over.  Lane i has sequence i in registers; further ones are loaded when their 64 come up.
struct Plan {
  int n;            // sequences
  int part;         // keys of a part
  Sequence first;   // sequence `lane` (empty if there is none)
};
template <typename Params>
__device__ __forceinline__ Sequence lane_sequence(const Params& p, const Plan& plan, int b0) {
  const int b = b0 + (int)(threadIdx.x & 63);
  return b0 == 0 ? plan.first : b < plan.n ? sequence(p.seq, b) : Sequence{0, 0, 0, 0};
}
// Sums count(sequence) over the sequences up to the one that holds element `at`: true, and its number and the sum before it; false, and the sum of all.
template <typename Params, typename Count>
__device__ __forceinline__ bool locate(const Params& p, const Plan& plan, int at, Count count, int& b, int& before) {
  before = 0;
  for (int b0 = 0; b0 < plan.n; b0 += 64) {
    const int c = count(lane_sequence(p, plan, b0)), upto = wave_scan(c);
    const unsigned long long over = __ballot(at < before + upto);
    if (over) {
      const int i = __builtin_ctzll(over);
      b = b0 + i;
      before += __builtin_amdgcn_readlane(upto - c, i);
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}
// The sum of count over the sequences in front of b.
template <typename Params, typename Count>
__device__ __forceinline__ int sum_before(const Params& p, const Plan& plan, int end, Count count) {
  int sum = 0;
  for (int b0 = 0; b0 < end; b0 += 64) {
    const int c = b0 + (int)(threadIdx.x & 63) < end ? count(lane_sequence(p, plan, b0)) : 0;
    sum += __builtin_amdgcn_readlane(wave_scan(c), 63);
  }
  return sum;
}

}  // namespace
}  // namespace tr
