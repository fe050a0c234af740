// Which keys of a paged cache stay (tr_cache_select), and moving those together (tr_cache_keep).
#include "evict.h"
#include "launch_lds.h"
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

// Weights in the order of unsigned integers: NaN highest, -0 as 0.  Above them all those keys that stay anyway, below them 0: no key, or on no page.
constexpr unsigned kStays = 0xffffffffu, kZero = 0x80000000u;
__device__ __forceinline__ unsigned rank_of(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x == 0.f ? 0.f : x);
  return x != x ? kStays - 1 : b & 0x80000000u ? ~b : b | 0x80000000u;
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

// The last key that stays: its rank, and how many of those that are equal to it stay, the first ones.
struct Border {
  unsigned rank;
  int take;
};
__device__ __forceinline__ int sum_four(const Border& border, const u32x4 u) {   // keys above the border, and in the upper half those equal to it
  int sum = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) sum += (u[i] > border.rank ? 1 : 0) + (u[i] == border.rank ? 1 << 16 : 0);
  return sum;
}
__device__ __forceinline__ void write_four(int* out, const Border& border, int key, const u32x4 u, int above, int same) {   // above, same: of the keys in front
  int at = above + min(same, border.take);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const bool equal = u[i] == border.rank, stays = u[i] > border.rank || (equal && same < border.take);
    if (stays) out[at] = key + i;
    at += stays ? 1 : 0;
    same += equal ? 1 : 0;
  }
}

// A row's ranks are held in LDS, where they fit (`room` of them, a multiple of a turn's), and are read again from memory in every pass where they do not.
constexpr int kTurn = 4 * kSelectThreads, kTurns = 9;   // keys of a turn of the workgroup; turns that LDS has room for beside the counts
__global__ void __launch_bounds__(kSelectThreads, 8) select_kernel(const SelectParams p, const int room) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ int counts[kDigits];
  __shared__ int waves[2][16];
  __shared__ int totals[kTurns * 16];
  __shared__ int found[2];   // digit, keys still to take among those that have it
  u32x4* const ranks = reinterpret_cast<u32x4*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  for (int64_t row = blockIdx.x; row < (int64_t)p.seq.n * p.heads; row += gridDim.x) {
    const int b = (int)(row / p.heads), h = (int)(row - (int64_t)b * p.heads);
    const int len = uniform(clamped(p.seq.kv_len[b], 0, p.seq.max_pages * p.seq.page_size)), n = min(len, p.most);
    int* const out = p.keys + (int64_t)b * p.k_sb + (int64_t)h * p.k_sh;
    if (h == 0 && tid == 0) p.count[b] = n;
    if (len <= p.most) {
      for (int i = tid; i < len; i += kSelectThreads) out[i] = i;
      continue;
    }
    if (p.most == 0) continue;
    auto fetch = [&](int key) __attribute__((always_inline)) -> u32x4 {   // keys key .. key + 3, key a multiple of 4
      u32x4 u = {0, 0, 0, 0};
      if (key >= len) return u;
      const Slot at = slot_of(p.seq, b, key);
      if (at.page >= 0) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(p.weights + (int64_t)at.page * p.w_sp + (int64_t)h * p.w_sh + at.slot);
#pragma unroll
        for (int i = 0; i < 4; i++) u[i] = rank_of(x[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; i++) u[i] = key + i >= len ? 0 : key + i < p.first || key + i >= len - p.last ? kStays : u[i];
      return u;
    };
    const bool held = len <= room;
    const int turns = (len + kTurn - 1) / kTurn;
    if (held) {
#pragma unroll 4
      for (int t = 0; t < turns; t++) ranks[t * kSelectThreads + tid] = fetch(t * kTurn + 4 * tid);   // (each thread reads what it wrote)
    }
    auto four = [&](int t) __attribute__((always_inline)) -> u32x4 { return held ? ranks[t * kSelectThreads + tid] : fetch(t * kTurn + 4 * tid); };
    Border border = {0, p.most};   // (at least one of the keys goes: len > most)
    unsigned known = 0;            // bits of the rank that are found
#pragma unroll 1
    for (int pass = 0; pass < 3; pass++) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const unsigned digits = pass < 2 ? 2047u : 1023u;
      for (int i = tid; i < kDigits; i += kSelectThreads) counts[i] = 0;
      __syncthreads();
      int zeros = 0, none = 0;   // (most weights may be 0: they are counted by the wave, 64 additions to one place are 64 turns)
      for (int t = 0; t < turns; t++) {
        const u32x4 x = four(t);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const bool here = (x[i] & known) == border.rank;
          zeros += __popcll(__ballot(here && x[i] == kZero));
          none += __popcll(__ballot(here && x[i] == 0));
          if (here && (x[i] & ~kZero) != 0) atomicAdd(&counts[x[i] >> shift & digits], 1);
        }
      }
      if (lane == 0 && zeros > 0) atomicAdd(&counts[kZero >> shift & digits], zeros);
      if (lane == 0 && none > 0) atomicAdd(&counts[0], none);
      __syncthreads();
      // from the highest digit down: thread t has digits 2047 - 2 t and the one below
      const int hi = counts[kDigits - 1 - 2 * tid], lo = counts[kDigits - 2 - 2 * tid];
      int all;
      const int above = before_in_group(hi + lo, waves[0], all);
      if (above < border.take && above + hi + lo >= border.take) {
        const bool in_hi = above + hi >= border.take;
        found[0] = kDigits - 1 - 2 * tid - (in_hi ? 0 : 1);
        found[1] = border.take - above - (in_hi ? 0 : hi);
      }
      __syncthreads();
      border.rank |= (unsigned)found[0] << shift;
      known |= digits << shift;
      border.take = found[1];
    }
    if (held) {   // sums within the waves, then one scan over those of all turns and waves
      for (int t = 0; t < turns; t++) {
        const int upto = wave_scan(sum_four(border, four(t)));
        if (lane == 63) totals[t * 16 + wave] = upto;
      }
      __syncthreads();
      int base = 0, scan[(kTurns * 16 + 63) / 64];
#pragma unroll
      for (int e = 0; e < (kTurns * 16 + 63) / 64; e++) {
        const int mine = e * 64 + lane < turns * 16 ? totals[e * 64 + lane] : 0, upto = wave_scan(mine);
        scan[e] = base + upto - mine;
        base += __builtin_amdgcn_readlane(upto, 63);
      }
      for (int t = 0; t < turns; t++) {
        const u32x4 x = four(t);
        const int at = t * 16 + wave, sum = sum_four(border, x), mine = at < 64 ? scan[0] : at < 128 ? scan[1] : scan[2];
        const int sums = __builtin_amdgcn_readlane(mine, at & 63) + wave_scan(sum) - sum;
        write_four(out, border, t * kTurn + 4 * tid, x, sums & 0xffff, (int)((unsigned)sums >> 16));
      }
    } else {
      int above = 0, same = 0;
      for (int t = 0; t < turns; t++) {
        const u32x4 x = four(t);
        int all;
        const int before = before_in_group(sum_four(border, x), waves[t & 1], all);
        write_four(out, border, t * kTurn + 4 * tid, x, above + (before & 0xffff), same + (before >> 16));
        above += all & 0xffff;
        same += all >> 16;
      }
    }
    __syncthreads();
  }
}

// ---- keep.
//
// In place: a place may be the source of an entry in front of it, so that rows are read before any is written there.  A list rises and moves nothing up, so a workgroup that goes through a list in its order, reading
// some rows, waiting for all its reads, and writing them, never writes what it has yet to read.  Workgroups share out sequences, heads, K and V, and pieces of the rows.
constexpr int kKeepThreads = 512, kKeepAhead = 8;   // entries of a thread of those that move scales and weights, at a time

struct KeepList {
  const int* keys;
  int n, start, len;
};
__device__ __forceinline__ KeepList list_of(const KeepParams& p, int b, int h) {
  KeepList l;
  l.keys = p.keys + (int64_t)b * p.k_sb + (int64_t)h * p.k_sh;
  l.n = uniform(clamped(p.count[b], 0, p.most));
  l.start = p.start ? uniform(clamped(p.start[b], -kPosLimit, kPosLimit - 1)) : 0;
  l.len = uniform(clamped(p.seq.kv_len[b], 0, p.seq.max_pages * p.seq.page_size));
  return l;
}
__device__ __forceinline__ int key_of(const KeepList& l, int i) { return i < l.n ? l.keys[i] : -1; }
// Where entry i, of key `key`, comes from and goes to; false: it is skipped, or stays where it is.
__device__ __forceinline__ bool entry(const KeepParams& p, const KeepList& l, int b, int i, int key, Slot& from, Slot& to) {
  const int place = l.start + i;   // (of two numbers below 2^30)
  if (place < 0 || place >= key || key >= l.len) return false;
  from = slot_of(p.seq, b, key);
  to = slot_of(p.seq, b, place);
  return from.page >= 0 && to.page >= 0;
}
__device__ __forceinline__ int64_t from_other(int64_t x, int lane) {
  return (int64_t)(((uint64_t)(unsigned)__shfl((int)(x >> 32), lane) << 32) | (unsigned)__shfl((int)x, lane));
}

// Every wave has 64 entries at a time: lane i finds the places of the i-th, and a row's piece is 16 bytes of LANES lanes.  While rows are on their way, so are the pages of
// the next entries and the keys of those behind them.
template <int LANES>
__device__ __forceinline__ void move_rows(const KeepParams& p, const KeepList& l, int b, char* pages, int64_t at_head) {
  constexpr int ROWS = 64 / LANES;   // at once
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), c = lane % LANES;
  char* const base = pages + at_head + c * 16;
  int key = key_of(l, wave * 64 + lane), key_next = key_of(l, kKeepThreads + wave * 64 + lane);
  Slot s = {0, 0}, d = {0, 0};
  bool moves = entry(p, l, b, wave * 64 + lane, key, s, d);
#pragma unroll 1
  for (int i0 = wave * 64; i0 < l.n + wave * 64; i0 += kKeepThreads) {   // (as often in every wave)
    const int64_t from = moves ? (int64_t)s.page * p.page_b + (int64_t)s.slot * p.slot_b : -1, to = moves ? (int64_t)d.page * p.page_b + (int64_t)d.slot * p.slot_b : -1;
    key = key_next;
    key_next = key_of(l, i0 + 2 * kKeepThreads + lane);
    moves = entry(p, l, b, i0 + kKeepThreads + lane, key, s, d);
    u32x4 x[LANES];
#pragma unroll
    for (int j = 0; j < LANES; j++) {
      const int64_t at = from_other(from, j * ROWS + lane / LANES);
      if (at >= 0) x[j] = *reinterpret_cast<const u32x4*>(base + at);
    }
    __builtin_amdgcn_s_waitcnt(0);   // the rows are here, not only asked for
    asm volatile("" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < LANES; j++) {
      const int64_t at = from_other(to, j * ROWS + lane / LANES);
      if (at >= 0) *reinterpret_cast<u32x4*>(base + at) = x[j];
    }
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
      const int i = i0 + j * kKeepThreads + (int)threadIdx.x;
      moves[j] = entry(p, l, b, i, key_of(l, i), s, d[j]);
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
  const dim3 grid((unsigned)(rows < 65536 ? rows : 65536)), block(kSelectThreads);
  // LDS for the rows that the table has room for: a compute unit then holds two workgroups on up to 16384 keys, one on more.
  const int64_t max_keys = (int64_t)p.seq.max_pages * p.seq.page_size, turns = (max_keys + kTurn - 1) / kTurn;
  const int room = (int)(turns < kTurns ? turns : kTurns) * kTurn;
  static std::atomic<uint64_t> raised;
  const hipError_t e = raise_lds(select_kernel, raised, kTurns * kTurn * 4);
  return e != hipSuccess ? e : launch_kernel(select_kernel, grid, block, room * 4, stream, p, room);
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
