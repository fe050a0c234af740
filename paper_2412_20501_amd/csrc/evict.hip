// Which keys of a paged cache stay (tr_cache_select), and moving those together (tr_cache_keep).
#include "evict.h"
#include "paged_sums.h"

namespace tr {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---- select.
//
// The k-th largest weight of a row (a sequence's K/V head) by its bits, 11, 11 and 10 at a time: counts of each value of these bits among the keys that have the higher
// bits found so far, in LDS; then the keys above it, and of those equal to it the first ones, in their order.
constexpr int kSelectThreads = 1024, kDigits = 2048;

// Weights in the order of unsigned integers: NaN highest, -0 as 0; 0: on no page.
__device__ __forceinline__ unsigned rank_of(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x == 0.f ? 0.f : x);
  if (x != x) return 0xffffffffu;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// Sum of x over the workgroup's threads in front of this one; all: over all of them.  `waves`: LDS for 17 numbers, free again behind the next barrier.
__device__ __forceinline__ int before_in_group(int x, int* waves, int& all) {
  const int wave = (int)threadIdx.x >> 6, upto = wave_scan(x);
  if ((threadIdx.x & 63) == 63) waves[wave] = upto;
  __syncthreads();
  int before = upto - x;
  all = 0;
#pragma unroll
  for (int i = 0; i < kSelectThreads / 64; i++) {
    const int n = waves[i];
    before += i < wave ? n : 0;
    all += n;
  }
  return before;
}

__global__ void __launch_bounds__(kSelectThreads) select_kernel(const SelectParams p) {
  __shared__ int counts[kDigits];
  __shared__ int waves[2][16];
  __shared__ unsigned found[3];   // digit, keys still to take among those that have it
  const int tid = threadIdx.x;
  for (int64_t row = blockIdx.x; row < (int64_t)p.seq.n * p.heads; row += gridDim.x) {
    const int b = (int)(row / p.heads), h = (int)(row - (int64_t)b * p.heads);
    const int len = clamped(p.seq.kv_len[b], 0, p.seq.max_pages * p.seq.page_size), n = min(len, p.most);
    int* const out = p.keys + (int64_t)b * p.k_sb + (int64_t)h * p.k_sh;
    if (h == 0 && tid == 0) p.count[b] = n;
    if (len <= p.most) {
      for (int i = tid; i < len; i += kSelectThreads) out[i] = i;
      continue;
    }
    const int from = p.first, to = len - p.last;   // first + last <= most < len
    auto four = [&](int key, unsigned (&u)[4]) __attribute__((always_inline)) {   // keys key .. key + 3, key a multiple of 4 and below len
      const Slot at = slot_of(p.seq, b, key);
#pragma unroll
      for (int i = 0; i < 4; i++) u[i] = 0;
      if (at.page < 0) return;
      const f32x4 x = *reinterpret_cast<const f32x4*>(p.weights + (int64_t)at.page * p.w_sp + (int64_t)h * p.w_sh + at.slot);
#pragma unroll
      for (int i = 0; i < 4; i++) u[i] = rank_of(x[i]);
    };
    int take = p.most - p.first - p.last;   // of those between
    unsigned prefix = 0, known = 0;         // bits found, and which
    if (take > 0) {
#pragma unroll 1
      for (int pass = 0; pass < 3; pass++) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const unsigned digits = pass < 2 ? 2047u : 1023u;
        for (int i = tid; i < kDigits; i += kSelectThreads) counts[i] = 0;
        __syncthreads();
        for (int key = (from & ~3) + 4 * tid; key < to; key += 4 * kSelectThreads) {
          unsigned u[4];
          four(key, u);
#pragma unroll
          for (int i = 0; i < 4; i++)
            if (key + i >= from && key + i < to && (u[i] & known) == prefix) atomicAdd(&counts[u[i] >> shift & digits], 1);
        }
        __syncthreads();
        // from the highest digit down: thread t has digits 2047 - 2 t and the one below
        const int hi = counts[kDigits - 1 - 2 * tid], lo = counts[kDigits - 2 - 2 * tid];
        int all;
        const int above = before_in_group(hi + lo, waves[0], all);
        if (above < take && above + hi + lo >= take) {
          const bool in_hi = above + hi >= take;
          found[0] = kDigits - 1 - 2 * tid - (in_hi ? 0 : 1);
          found[1] = take - above - (in_hi ? 0 : hi);
        }
        __syncthreads();
        prefix |= found[0] << shift;
        known |= digits << shift;
        take = (int)found[1];
        __syncthreads();
      }
    }
    // keys above the bits found, and the first `take` of those equal to them
    int kept = 0, same = 0;
    int turn = 0;
    for (int key0 = 0; key0 < len; key0 += 4 * kSelectThreads) {
      const int key = key0 + 4 * tid;
      unsigned u[4] = {0, 0, 0, 0};
      if (key < len) four(key, u);
      bool stays[4], equal[4];
      int sum = 0;   // keys that stay, and in the upper half those that are equal
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const bool there = key + i < len, between = key + i >= from && key + i < to;
        equal[i] = there && between && known != 0 && u[i] == prefix;
        stays[i] = there && (!between || (known != 0 && u[i] > prefix));
        sum += (stays[i] ? 1 : 0) + (equal[i] ? 1 << 16 : 0);
      }
      int all;
      const int before = before_in_group(sum, waves[turn], all);
      turn ^= 1;
      // equal ones in front of this thread's, which stay while there are fewer than `take`
      int eq = same + (before >> 16), at = kept + (before & 0xffff) + min(eq, take) - min(same, take);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const bool stay = stays[i] || (equal[i] && eq < take);
        if (equal[i]) eq++;
        if (stay) out[at++] = key + i;
      }
      const int equals = all >> 16;
      kept += (all & 0xffff) + min(same + equals, take) - min(same, take);
      same += equals;
    }
    __syncthreads();
  }
}

// ---- keep.
//
// In place: a place may be the source of an entry in front of it, so that rows are read before any is written there.  A list rises and moves nothing up, so a workgroup that goes through a list in its order, reading
// some rows, waiting for all its reads, and writing them, never writes what it has yet to read.  Workgroups share out sequences, heads, K and V, and pieces of the rows.
constexpr int kKeepThreads = 512, kKeepAhead = 8;   // 16-byte pieces of a thread at a time

struct KeepList {
  const int* keys;
  int n, start, len;
};
__device__ __forceinline__ KeepList list_of(const KeepParams& p, int b, int h) {
  KeepList l;
  l.keys = p.keys + (int64_t)b * p.k_sb + (int64_t)h * p.k_sh;
  l.n = clamped(p.count[b], 0, p.most);
  l.start = p.start ? clamped(p.start[b], -kPosLimit, kPosLimit - 1) : 0;
  l.len = clamped(p.seq.kv_len[b], 0, p.seq.max_pages * p.seq.page_size);
  return l;
}
// Where entry i comes from and goes to; false: it is skipped, or stays where it is.
__device__ __forceinline__ bool entry(const KeepParams& p, const KeepList& l, int b, int i, Slot& from, Slot& to) {
  if (i >= l.n) return false;
  const int key = l.keys[i], place = l.start + i;
  if (place < 0 || place >= key || key >= l.len) return false;
  from = slot_of(p.seq, b, key);
  to = slot_of(p.seq, b, place);
  return from.page >= 0 && to.page >= 0;
}

// LANES threads move 16 bytes each of a row's piece.
template <int LANES>
__device__ __forceinline__ void move_rows(const KeepParams& p, const KeepList& l, int b, char* pages, int64_t at_head) {
  constexpr int ROWS = kKeepThreads / LANES;
  const int r = (int)threadIdx.x / LANES, c = (int)threadIdx.x % LANES;
  char* const base = pages + at_head + c * 16;
#pragma unroll 1
  for (int i0 = 0; i0 < l.n; i0 += ROWS * kKeepAhead) {
    u32x4 x[kKeepAhead];
    int64_t to[kKeepAhead];
#pragma unroll
    for (int j = 0; j < kKeepAhead; j++) {
      Slot s, d;
      to[j] = -1;
      if (entry(p, l, b, i0 + j * ROWS + r, s, d)) {
        to[j] = (int64_t)d.page * p.page_b + (int64_t)d.slot * p.slot_b;
        x[j] = *reinterpret_cast<const u32x4*>(base + (int64_t)s.page * p.page_b + (int64_t)s.slot * p.slot_b);
      }
    }
    __builtin_amdgcn_s_waitcnt(0);   // the rows are here, not only asked for
    asm volatile("" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kKeepAhead; j++)
      if (to[j] >= 0) *reinterpret_cast<u32x4*>(base + to[j]) = x[j];
  }
}
__device__ __forceinline__ void move_scales(const KeepParams& p, const KeepList& l, int b, int h) {   // and weights
#pragma unroll 1
  for (int i0 = 0; i0 < l.n; i0 += kKeepThreads * kKeepAhead) {
    unsigned char ks[kKeepAhead], vs[kKeepAhead];
    float w[kKeepAhead];
    Slot d[kKeepAhead];
    bool moves[kKeepAhead];
#pragma unroll
    for (int j = 0; j < kKeepAhead; j++) {
      Slot s;
      moves[j] = entry(p, l, b, i0 + j * kKeepThreads + (int)threadIdx.x, s, d[j]);
      if (moves[j] && p.k_scales) {
        const int64_t at = (int64_t)s.page * p.scale_sp + (int64_t)h * p.scale_sh + s.slot;
        ks[j] = p.k_scales[at];
        vs[j] = p.v_scales[at];
      }
      if (moves[j] && p.weights) w[j] = p.weights[(int64_t)s.page * p.w_sp + (int64_t)h * p.w_sh + s.slot];
    }
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kKeepAhead; j++) {
      if (moves[j] && p.k_scales) {
        const int64_t at = (int64_t)d[j].page * p.scale_sp + (int64_t)h * p.scale_sh + d[j].slot;
        p.k_scales[at] = ks[j];
        p.v_scales[at] = vs[j];
      }
      if (moves[j] && p.weights) p.weights[(int64_t)d[j].page * p.w_sp + (int64_t)h * p.w_sh + d[j].slot] = w[j];
    }
  }
}

// blockIdx.x: piece of the rows of K, of V, and behind them scales and weights; y: sequence and head.
template <int LANES>
__global__ void __launch_bounds__(kKeepThreads) keep_kernel(const KeepParams p, const int pieces) {
  for (int64_t y = blockIdx.y; y < (int64_t)p.seq.n * p.heads; y += gridDim.y) {
    const int b = (int)(y / p.heads), h = (int)(y - (int64_t)b * p.heads), x = (int)blockIdx.x;
    const KeepList l = list_of(p, b, h);
    if (x >= 2 * pieces) move_scales(p, l, b, h);
    else move_rows<LANES>(p, l, b, x >= pieces ? p.v_pages : p.k_pages, (int64_t)h * p.head_b + (x >= pieces ? x - pieces : x) * (LANES * 16));
  }
}

}  // namespace

hipError_t launch_cache_select(const SelectParams& p, hipStream_t stream) {
  const int64_t rows = (int64_t)p.seq.n * p.heads;
  return launch_kernel(select_kernel, dim3((unsigned)(rows < 65536 ? rows : 65536)), dim3(kSelectThreads), 0, stream, p);
}

hipError_t launch_cache_keep(const KeepParams& p, hipStream_t stream) {
  const int64_t lists = (int64_t)p.seq.n * p.heads;
  const unsigned y = (unsigned)(lists < 65535 ? lists : 65535), side = p.k_scales || p.weights ? 1 : 0;
  const int pieces = lists * 2 >= 256 || p.row_bytes < 128 ? 1 : p.row_bytes / 64, lanes = p.row_bytes / pieces / 16;
  const dim3 grid(2 * pieces + side, y), block(kKeepThreads);
  if (lanes == 16) return launch_kernel(keep_kernel<16>, grid, block, 0, stream, p, pieces);
  if (lanes == 8) return launch_kernel(keep_kernel<8>, grid, block, 0, stream, p, pieces);
  return launch_kernel(keep_kernel<4>, grid, block, 0, stream, p, pieces);
}

}  // namespace tr
