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
// bits found so far, in LDS; then the keys above it, and of those equal to it the first ones, in their order.  A row is one workgroup's: keys that stay anyway are ranked above all others, so that
// nothing else has to know about them.
constexpr int kDigits = 2048;

// Weights in the order of unsigned integers: NaN highest, -0 as 0.  Above them all those keys that stay anyway, below them 0: no key, or on no page.
constexpr unsigned kStays = 0xffffffffu, kZero = 0x80000000u;
__device__ __forceinline__ unsigned rank_of(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x == 0.f ? 0.f : x);
  return x != x ? kStays - 1 : b & 0x80000000u ? ~b : b | 0x80000000u;
}
// One wave: the digit of the take-th largest among counts, from the highest digit (DIGITS - 1) down, and how many of those that have it are still to take; false: there are fewer than `take`
// in all, which are taken off.
template <int DIGITS>
__device__ __forceinline__ bool find_digit(const int* counts, int& take, unsigned& digit) {
  constexpr int EACH = DIGITS / 64;   // lane i has digits DIGITS - 1 - EACH i and the EACH - 1 below
  const int lane = threadIdx.x & 63;
  const u32x4* const mine = reinterpret_cast<const u32x4*>(counts) + (63 - lane) * (EACH / 4);
  int sum = 0;
#pragma unroll
  for (int i = 0; i < EACH / 4; i++) {
    const u32x4 x = mine[(i + lane) % (EACH / 4)];   // (lanes begin on different banks)
    sum += (int)(x[0] + x[1] + x[2] + x[3]);
  }
  const int upto = wave_scan(sum), all = __builtin_amdgcn_readlane(upto, 63);
  if (all < take) {
    take -= all;
    return false;
  }
  const int first = __builtin_ctzll(__ballot(upto >= take));   // the lane that has it
  take -= __builtin_amdgcn_readlane(upto - sum, first);
  const int top = DIGITS - 1 - EACH * first, one = lane < EACH ? counts[top - lane] : 0, below = wave_scan(one);
  const int at = __builtin_ctzll(__ballot(below >= take));
  take -= __builtin_amdgcn_readlane(below - one, at);
  digit = top - at;
  return true;
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

// A wave has a stretch of the row's keys, 256 at a time.  Ranks are held in LDS, as many as fit (`room`), and those behind them in registers (EXTRA); what is left is read from memory again where it is
// needed.  Those that share the first digit with the border, mostly a few hundredths of them, are held once more as a list, unless it is too long.  Bound: the instructions of one compute unit, and its barriers
// (512 rows of 4608 keys: 10 us of a workgroup's time, 3 of them for the weights to come; 8 of 32768: 21; 8 of 65536 30, with all ranks read again where LDS does not hold them 55).
constexpr int kRoom = 32768, kList = 2048;   // ranks that LDS has room for; entries of the list
template <int THREADS, int EXTRA>   // EXTRA: pieces of four ranks behind those that a thread holds in registers
__global__ void __launch_bounds__(THREADS, EXTRA > 0 ? 4 : 8) select_kernel(const SelectParams p, const int room) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ __attribute__((aligned(16))) int counts[2 * kDigits + kDigits / 2];   // of the three passes
  __shared__ unsigned list[kList];
  __shared__ int sums[2][THREADS / 64];
  __shared__ int n_list, n_zeros, found[2];   // found: digit, keys still to take among those that have it
  u32x4* const ranks = reinterpret_cast<u32x4*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  for (int64_t row = blockIdx.x; row < (int64_t)p.seq.n * p.heads; row += gridDim.x) {
    const int b = (int)(row / p.heads), h = (int)(row - (int64_t)b * p.heads);
    const int len = uniform(clamped(p.seq.kv_len[b], 0, p.seq.max_pages * p.seq.page_size)), n = min(len, p.most);
    int* const out = p.keys + (int64_t)b * p.k_sb + (int64_t)h * p.k_sh;
    if (h == 0 && tid == 0) p.count[b] = n;
    if (len <= p.most) {
      for (int i = tid; i < len; i += THREADS) out[i] = i;
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
      if (key < p.first || key + 3 >= len - p.last) {
#pragma unroll
        for (int i = 0; i < 4; i++) u[i] = key + i >= len ? 0 : key + i < p.first || key + i >= len - p.last ? kStays : u[i];
      }
      return u;
    };
    const int steps = (len + 4 * THREADS - 1) / (4 * THREADS), piece0 = wave * steps * 64 + lane;   // of a wave; pieces of four keys are piece0 + 64 i
    const int in_lds = min(steps, room / (4 * THREADS)), behind = in_lds + EXTRA;                   // pieces in LDS; those from `behind` on are held nowhere
    u32x4* const mine = ranks + wave * in_lds * 64 + lane;   // (each thread reads what it wrote)
    u32x4 kept[EXTRA > 0 ? EXTRA : 1];
    auto over = [&](auto body) __attribute__((always_inline)) {   // all pieces: body(i, ranks)
      for (int i = 0; i < in_lds; i++) body(i, mine[64 * i]);
      if constexpr (EXTRA > 0) {
#pragma unroll
        for (int j = 0; j < EXTRA; j++)
          if (in_lds + j < steps) body(in_lds + j, kept[j]);
      }
#pragma unroll 1
      for (int i = behind; i < steps; i++) body(i, fetch(4 * (piece0 + 64 * i)));
    };
    Border border = {0, p.most};   // (at least one of the keys goes: len > most)
    auto find = [&](int pass, int shift) __attribute__((always_inline)) -> bool {
      __syncthreads();
      if (wave == 0) {
        unsigned digit = 0;
        int take = border.take;
        const bool there = pass < 2 ? find_digit<kDigits>(counts + pass * kDigits, take, digit) : find_digit<kDigits / 2>(counts + 2 * kDigits, take, digit);
        if (lane == 0) {
          found[0] = there ? (int)digit : -1;
          found[1] = take;
        }
      }
      __syncthreads();
      const int digit = uniform(found[0]);
      border.take = uniform(found[1]);
      if (digit < 0) return false;   // there are too few keys on pages: the border is among the others
      border.rank |= (unsigned)digit << shift;
      return true;
    };
    if (tid == 0) n_list = n_zeros = 0;
    for (int i = tid; i < (2 * kDigits + kDigits / 2) / 4; i += THREADS) reinterpret_cast<u32x4*>(counts)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
    int zeros = 0;   // (most weights may be 0: they are counted apart, 64 additions to one place are 64 turns)
    auto count = [&](const u32x4 x) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < 4; k++) {
        zeros += x[k] == kZero ? 1 : 0;
        if ((x[k] & ~kZero) != 0) atomicAdd(&counts[x[k] >> 21], 1);
      }
    };
#pragma unroll 4
    for (int i = 0; i < in_lds; i++) {
      const u32x4 x = fetch(4 * (piece0 + 64 * i));
      mine[64 * i] = x;
      count(x);
    }
    if constexpr (EXTRA > 0) {
#pragma unroll
      for (int j = 0; j < EXTRA; j++)
        if (in_lds + j < steps) kept[j] = fetch(4 * (piece0 + 64 * (in_lds + j)));
#pragma unroll
      for (int j = 0; j < EXTRA; j++)
        if (in_lds + j < steps) count(kept[j]);
    }
#pragma unroll 4
    for (int i = behind; i < steps; i++) count(fetch(4 * (piece0 + 64 * i)));
    zeros = __builtin_amdgcn_readlane(wave_scan(zeros), 63);
    if (lane == 0 && zeros > 0) {
      atomicAdd(&counts[kZero >> 21], zeros);
      atomicAdd(&n_zeros, zeros);
    }
    if (find(0, 21)) {
      const unsigned digit = border.rank >> 21;
      over([&](int, const u32x4 x) __attribute__((always_inline)) {
        int have = 0;
#pragma unroll
        for (int k = 0; k < 4; k++) have += x[k] >> 21 == digit && x[k] != kZero ? 1 : 0;
        if (!__any(have != 0)) return;
        const int upto = wave_scan(have);
        int at = 0;
        if (lane == 63) at = atomicAdd(&n_list, upto);
        at = __builtin_amdgcn_readlane(at, 63) + upto - have;
#pragma unroll
        for (int k = 0; k < 4; k++)
          if (x[k] >> 21 == digit && x[k] != kZero) {
            atomicAdd(&counts[kDigits + (x[k] >> 10 & 2047)], 1);
            if (at < kList) list[at] = x[k];
            at++;
          }
      });
      if (tid == 0 && digit == kZero >> 21) atomicAdd(&counts[kDigits + (kZero >> 10 & 2047)], n_zeros);
      find(1, 10);
      const unsigned high = border.rank >> 10;
      if (n_list <= kList) {
        for (int i = tid; i < n_list; i += THREADS)
          if (list[i] >> 10 == high) atomicAdd(&counts[2 * kDigits + (list[i] & 1023)], 1);
      } else {
        over([&](int, const u32x4 x) __attribute__((always_inline)) {
#pragma unroll
          for (int k = 0; k < 4; k++)
            if (x[k] >> 10 == high && x[k] != kZero) atomicAdd(&counts[2 * kDigits + (x[k] & 1023)], 1);
        });
      }
      if (tid == 0 && high == kZero >> 10) atomicAdd(&counts[2 * kDigits], n_zeros);
      find(2, 0);
    }
    // what the waves in front have: keys above the border, and those equal to it
    int above = 0, same = 0;
    over([&](int, const u32x4 x) __attribute__((always_inline)) {
      const int sum = sum_four(border, x);
      above += sum & 0xffff;
      same += sum >> 16;
    });
    above = wave_scan(above);
    same = wave_scan(same);
    if (lane == 63) {
      sums[0][wave] = above;
      sums[1][wave] = same;
    }
    __syncthreads();
    above = lane < wave ? sums[0][lane] : 0;
    same = lane < wave ? sums[1][lane] : 0;
    above = __builtin_amdgcn_readlane(wave_scan(above), 63);
    same = __builtin_amdgcn_readlane(wave_scan(same), 63);
    over([&](int i, const u32x4 x) __attribute__((always_inline)) {
      const int sum = sum_four(border, x), upto = wave_scan(sum), before = upto - sum, all = __builtin_amdgcn_readlane(upto, 63);
      write_four(out, border, 4 * (piece0 + 64 * i), x, above + (before & 0xffff), same + (before >> 16));
      above += all & 0xffff;
      same += all >> 16;
    });
    __syncthreads();
  }
}

// ---- keep.
//
// In place: a place may be the source of an entry in front of it, so that rows are read before any is written there.  A list rises and moves nothing up, so a workgroup that goes through a list in its order, reading
// some rows, waiting for all its reads, and writing them, never writes what it has yet to read.  Workgroups share out sequences, heads, K and V, and, where those are few, pieces of the rows.  Bound: HBM: 64
// sequences of 4.6K keys on 8 heads of 128 in 8 bits back to 4096 238 us, 4.65 TB/s (with keys and pages looked up in front of each load 338); one long list: the instructions that find its entries.
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

// Every wave has SETS times 64 entries at a time: lane i finds the places of the i-th of each, and a row's piece is 16 bytes of LANES lanes.  While rows are on their way, so are the pages of
// the next entries and the keys of those behind them.
template <int LANES, int SETS>
__device__ __forceinline__ void move_rows(const KeepParams& p, const KeepList& l, int b, char* pages, int64_t at_head) {
  constexpr int ROWS = 64 / LANES, ALL = SETS * kKeepThreads;   // rows at once; entries of the workgroup
  const int lane = threadIdx.x & 63, first = uniform((int)threadIdx.x >> 6) * 64 * SETS, c = lane % LANES;
  char* const base = pages + at_head + c * 16;
  int key_next[SETS];
  int64_t from[SETS], to[SETS];   // of the next entries, -1: none
  auto find = [&](int k, int i, int key) __attribute__((always_inline)) {
    Slot s, d;
    from[k] = to[k] = -1;
    if (entry(p, l, b, i, key, s, d)) {
      from[k] = (int64_t)s.page * p.page_b + (int64_t)s.slot * p.slot_b;
      to[k] = (int64_t)d.page * p.page_b + (int64_t)d.slot * p.slot_b;
    }
  };
#pragma unroll
  for (int k = 0; k < SETS; k++) {
    const int i = first + k * 64 + lane;
    key_next[k] = key_of(l, i + ALL);
    find(k, i, key_of(l, i));
  }
#pragma unroll 1
  for (int i0 = 0; i0 < l.n; i0 += ALL) {
    int64_t src[SETS], dst[SETS];
#pragma unroll
    for (int k = 0; k < SETS; k++) {
      const int i = i0 + ALL + first + k * 64 + lane, key = key_next[k];
      src[k] = from[k];
      dst[k] = to[k];
      key_next[k] = key_of(l, i + ALL);
      find(k, i, key);
    }
    u32x4 x[SETS][LANES];
#pragma unroll
    for (int k = 0; k < SETS; k++)
#pragma unroll
      for (int j = 0; j < LANES; j++) {
        const int64_t at = from_other(src[k], j * ROWS + lane / LANES);
        if (at >= 0) x[k][j] = *reinterpret_cast<const u32x4*>(base + at);
      }
    __builtin_amdgcn_s_waitcnt(0);   // the rows are here, not only asked for
    asm volatile("" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SETS; k++)
#pragma unroll
      for (int j = 0; j < LANES; j++) {
        const int64_t at = from_other(dst[k], j * ROWS + lane / LANES);
        if (at >= 0) *reinterpret_cast<u32x4*>(base + at) = x[k][j];
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
template <int LANES, int SETS>
__global__ void __launch_bounds__(kKeepThreads) keep_kernel(const KeepParams p, const int pieces) {
  for (int64_t y = blockIdx.y; y < (int64_t)p.seq.n * p.heads; y += gridDim.y) {
    const int b = (int)(y / p.heads), h = (int)(y - (int64_t)b * p.heads), x = (int)blockIdx.x;
    const KeepList l = list_of(p, b, h);
    if (x >= 2 * pieces) move_scales(p, l, b, h);
    else move_rows<LANES, SETS>(p, l, b, x >= pieces ? p.v_pages : p.k_pages, (int64_t)h * p.head_b + (x >= pieces ? x - pieces : x) * (LANES * 16));
  }
}

}  // namespace

namespace {
template <int THREADS, int EXTRA>
hipError_t launch_select(const SelectParams& p, int room, dim3 grid, hipStream_t stream) {
  static std::atomic<uint64_t> raised;
  const hipError_t e = raise_lds(select_kernel<THREADS, EXTRA>, raised, kRoom * 4);
  return e != hipSuccess ? e : launch_kernel(select_kernel<THREADS, EXTRA>, grid, dim3(THREADS), room * 4, stream, p, room);
}
}  // namespace

hipError_t launch_cache_select(const SelectParams& p, hipStream_t stream) {
  const int64_t rows = (int64_t)p.seq.n * p.heads;
  const dim3 grid((unsigned)(rows < 65536 ? rows : 65536));
  const int64_t max_keys = (int64_t)p.seq.max_pages * p.seq.page_size;
  const int room = (int)(max_keys < kRoom ? (max_keys + 4095) / 4096 * 4096 : kRoom);   // LDS for what the table has room for
  // With a row for every compute unit, smaller workgroups, two a unit, are less work, as long as LDS holds the ranks of two: 512 rows of 4608 keys 12.7 us, with 1024 threads about 1 more, with 256 1.5; 8 rows of
  // 32768 keys 21.7, with 512 threads 7 more, with 256 28; 512 rows of 14500 33.3 with 512 threads, 28.2 with 1024.  Registers for another 32768 ranks, where the table has room for so many: 8 rows of 65536 keys 42.7 -> 30.3, 256 of 40000 42.3 -> 30.
  // What the rows need lies on the device, so a table with room for more costs short rows: with room for 16K (64K) keys 512 rows of 4608 take 18.7 us (19.4) for 12.6, of 1000 keys 13.6 (14.8) for 7.8, 8 of 4608 9.1 (9.7) for 9.1.
  constexpr int kTwoRows = 12288;
  if (max_keys > kRoom) return launch_select<1024, 8>(p, room, grid, stream);
  return rows >= 256 && max_keys <= kTwoRows ? launch_select<512, 0>(p, room, grid, stream) : launch_select<1024, 0>(p, room, grid, stream);
}

namespace {
template <int LANES, int SETS>
hipError_t launch_keep(const KeepParams& p, int pieces, hipStream_t stream) {
  const int64_t lists = (int64_t)p.seq.n * p.heads;
  const dim3 grid(2 * pieces + (p.k_scales || p.weights ? 1 : 0), (unsigned)(lists < 65535 ? lists : 65535));
  return launch_kernel(keep_kernel<LANES, SETS>, grid, dim3(kKeepThreads), 0, stream, p, pieces);
}
}  // namespace

hipError_t launch_cache_keep(const KeepParams& p, hipStream_t stream) {
  const int pieces = (int64_t)p.seq.n * p.heads * 2 >= 256 || p.row_bytes < 128 ? 1 : p.row_bytes / 64, lanes = p.row_bytes / pieces / 16;
  // Long lists: more entries between two barriers, if fewer workgroups share a compute unit (64 lists of up to 4608 keys on 8 heads of 128 bytes 247 -> 238 us, of 256 bytes 467 -> 456, one of 32768 53 -> 46).
  // Their length lies on the device, so lists with room for more than they hold lose: 64 of 600 keys in 8 bits 28 -> 44, of 2000 96 -> 109, 8 of 600 9.3 -> 13.5.
  const bool many = p.most > 2048;
  if (lanes == 16) return many ? launch_keep<16, 2>(p, pieces, stream) : launch_keep<16, 1>(p, pieces, stream);
  if (lanes == 8) return many ? launch_keep<8, 4>(p, pieces, stream) : launch_keep<8, 1>(p, pieces, stream);
  return many ? launch_keep<4, 4>(p, pieces, stream) : launch_keep<4, 1>(p, pieces, stream);
}

}  // namespace tr
