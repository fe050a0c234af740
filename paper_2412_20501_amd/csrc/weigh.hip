// The attention weight that each key of a paged cache gets from the new tokens (tr_cache_weigh).
//
// weights[c] += sum over rows r that see c of exp(scale <q_r, K_c> - lse_r), a row being a (token, query head of the K/V head) pair: half of an attention's products, one
// exponential a score, and sums down the rows instead of along the keys.  A workgroup has some keys and goes through all rows that see them, so that a
// key's sum is one workgroup's, in one order, and K is read once.
#include <type_traits>

#include "evict.h"
#include "paged_sums.h"
#include "weigh_plan.h"

namespace tr {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kFewWaves = 4;     // a SIMD, of few rows
constexpr int kTogetherBelow = 192, kTogetherInMixture = 128, kSmallMixture = 8;   // items of many rows; sequences
constexpr int kManyKeys = 256;   // of many rows: 64 a wave, or, where that leaves compute units without an item, 64 that the waves have together

// Items: (sequence, K/V head, stretch of keys) of the launch's sequences, numbered so that those of a head lie together, and each XCD has a contiguous eighth of all.
struct WeighItem {
  int b, hk, k0;   // its keys: k0 .. min(k0 + width, seen) - 1
  int seen;        // keys that some row of the sequence sees (or that start from 0)
  Sequence q;
};
__device__ __forceinline__ int seen_keys(const WeighParams& p, const Sequence& q) { return visible(q, q.n - 1, p.causal); }
template <int WIDTH>
__device__ __forceinline__ int tiles_of_keys(const WeighParams& p, const RowClass& c, const Sequence& q) {   // of a K/V head
  return tiles_of(q.n * p.gq, c) > 0 ? (seen_keys(p, q) + WIDTH - 1) / WIDTH : 0;
}
__device__ __forceinline__ Plan sums_plan(const WeighParams& p) {
  Plan plan = {p.seq.n, 0, Sequence{0, 0, 0, 0}};
  const int lane = threadIdx.x & 63;
  if (lane < plan.n) plan.first = sequence(p.seq, lane);
  return plan;
}
template <int WIDTH>
__device__ __forceinline__ int all_items(const WeighParams& p, const RowClass& c, const Plan& plan) {
  int b = 0, total;
  locate(p, plan, 0x7fffffff, [&](const Sequence& q) { return tiles_of_keys<WIDTH>(p, c, q) * p.Hkv; }, b, total);
  return total;
}
template <int WIDTH>
__device__ __forceinline__ void item_at(const WeighParams& p, const RowClass& c, const Plan& plan, int at, WeighItem& w) {   // at: below all_items()
  int b = 0, before;
  locate(p, plan, at, [&](const Sequence& q) { return tiles_of_keys<WIDTH>(p, c, q) * p.Hkv; }, b, before);
  w.b = uniform(b);
  if (w.b < 64) {   // a lane has it
    const Sequence& q = plan.first;
    w.q = Sequence{__builtin_amdgcn_readlane(q.start, w.b), __builtin_amdgcn_readlane(q.n, w.b), __builtin_amdgcn_readlane(q.len, w.b), __builtin_amdgcn_readlane(q.pos, w.b)};
  } else {
    const Sequence q = sequence(p.seq, w.b);
    w.q = Sequence{uniform(q.start), uniform(q.n), uniform(q.len), uniform(q.pos)};
  }
  const int tiles = uniform(tiles_of_keys<WIDTH>(p, c, w.q)), i = uniform(at - before);
  w.hk = uniform(i / tiles);
  w.k0 = (i - w.hk * tiles) * WIDTH;
  w.seen = uniform(seen_keys(p, w.q));
}
// Adds to a key's weight, if it has a page.
__device__ __forceinline__ void add_weight(const WeighParams& p, const WeighItem& w, int key, float sum) {
  if (key >= w.seen) return;
  const Slot at = slot_of(p.seq, w.b, key);
  if (at.page < 0) return;
  float* const to = p.weights + (int64_t)at.page * p.w_sp + (int64_t)w.hk * p.w_sh + at.slot;
  const bool starts = p.fresh && key >= w.q.pos && key < w.q.pos + w.q.n;
  *to = starts ? sum : *to + sum;
}

// Few rows (a decode step, drafts): every wave has 64 keys, straight from memory into registers as the B operand of S = Q K^T; lane (i = lane % 16, g = lane / 16) then has
// scores of key i with rows 4 g .. 4 g + 3 of 16, so that a key's sum is four additions and two exchanges between lanes.  More rows than 16 are gone through with the keys held.  The pages of the next item's
// keys are on their way beside this one's keys (found one after the other, table, then keys: 173 us for the 139 below).  Bound: HBM: a token of 64 sequences of 0.8K to 16K keys on 8 heads of 128 in 8 bits
// 135 us, 4.5 TB/s of K and weights; of 16 of 8K in bf16 44.5 us, 6.2 TB/s.
template <int D, bool F8>
__device__ __forceinline__ void weigh_few(const WeighParams& p, const RowClass& c, const Plan& plan, int turn) {   // turn: of the XCD's workgroups, the items' order
  constexpr int QS = D / 32, KL = F8 ? D / 64 : D / 32;
  const int total = uniform(all_items<kFewKeys>(p, c, plan)), each = (total + 7) >> 3, base = ((int)blockIdx.x & 7) * each, end = min(each, total - base);
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
  const float c2 = p.scale * kLog2e;
  WeighItem w, next;
  Slot mine = {-1, 0};   // of key key0 + lane
  auto find = [&](int at, WeighItem& item, Slot& slot) __attribute__((always_inline)) {
    slot = Slot{-1, 0};
    if (at >= end) return;
    item_at<kFewKeys>(p, c, plan, base + at, item);
    const int key = item.k0 + wave * 64 + lane;
    if (key < item.seen) slot = slot_of(p.seq, item.b, key);
  };
  find(turn, next, mine);
  for (int at = turn; at < end; at += (int)gridDim.x >> 3) {
    w = next;
    const Slot slot_now = mine;
    const int key0 = w.k0 + wave * 64, rows = w.q.n * p.gq;
    u32x4 kr[4][KL];
    unsigned k_scale[4];
#pragma unroll
    for (int h = 0; h < 4; h++) {   // 16 keys lie on one page
      const int page = __builtin_amdgcn_readlane(slot_now.page, 16 * h), slot = __builtin_amdgcn_readlane(slot_now.slot, 16 * h);
      k_scale[h] = 127;
      if (page >= 0) {
        const char* const kp = p.k_pages + (int64_t)page * p.page_b + (int64_t)w.hk * p.head_b + (int64_t)slot * p.slot_b;
        const unsigned off = (unsigned)(i16 * p.slot_b + g * 16);   // (slot_b is at most 2^25)
#pragma unroll
        for (int l = 0; l < KL; l++) kr[h][l] = *reinterpret_cast<const u32x4*>(kp + off + l * 64);
        if constexpr (F8) k_scale[h] = (p.k_scales + ((int64_t)page * p.scale_sp + (int64_t)w.hk * p.scale_sh + slot))[(unsigned)i16];
      } else {
#pragma unroll
        for (int l = 0; l < KL; l++) kr[h][l] = u32x4{0, 0, 0, 0};
      }
    }
    float old = 0.f;
    float* to = nullptr;
    if (slot_now.page >= 0) {
      to = p.weights + (int64_t)slot_now.page * p.w_sp + (int64_t)w.hk * p.w_sh + slot_now.slot;
      const bool starts = p.fresh && key0 + lane >= w.q.pos && key0 + lane < w.q.pos + w.q.n;
      if (!starts) old = *to;
    }
    float sum = 0.f;   // of key key0 + lane
    for (int r0 = 0; r0 < rows; r0 += 16) {
      bf16x8 qf[QS];
      const int row = r0 + i16, t = divide(p.by_gq, min(row, rows - 1)), head = w.hk * p.gq + min(row, rows - 1) - t * p.gq;
      const __bf16* const src = p.q + (int64_t)head * p.q_sh + (int64_t)(w.q.start + t) * p.q_ss;
#pragma unroll
      for (int s = 0; s < QS; s++)   // d's in the order of the K loads
        qf[s] = *reinterpret_cast<const bf16x8*>(src + (F8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8));
      const float lse = p.lse[(int64_t)head * p.l_sh + (int64_t)(w.q.start + t) * p.l_ss];
      if (r0 == 0) find(at + ((int)gridDim.x >> 3), next, mine);   // (in front of what waits for the keys)
      // the lane's row: what its exponents have taken off, and the keys that it sees, from key0 on
      const bool live = row < rows && fabsf(lse) < INFINITY;
      const float my_ref = live ? lse * kLog2e : INFINITY;
      const int my_limit = live ? visible(w.q, t, p.causal) - key0 : 0;
      const bool masked = __any(my_limit < 64);
      float ref[4];
      int limit[4];
#pragma unroll
      for (int r = 0; r < 4; r++) {
        ref[r] = __shfl(my_ref, 4 * g + r);
        limit[r] = __shfl(my_limit, 4 * g + r);
      }
#pragma unroll
      for (int h = 0; h < 4; h++) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < QS; ks++) {
          bf16x8 b;
          if constexpr (F8) {
            const u32x4 x = kr[h][ks >> 1];
            const unsigned lo = x[(ks & 1) * 2], hi = x[(ks & 1) * 2 + 1], e = k_scale[h];
            b = __builtin_bit_cast(bf16x8, u32x4{f8_pair(lo, false, e), f8_pair(lo, true, e), f8_pair(hi, false, e), f8_pair(hi, true, e)});
          } else {
            b = __builtin_bit_cast(bf16x8, kr[h][ks]);
          }
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[ks], b, s, 0, 0, 0);
        }
        float part = 0.f;
#pragma unroll
        for (int r = 0; r < 4; r++) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, -ref[r]));
          part += masked && 16 * h + i16 >= limit[r] ? 0.f : e;
        }
        part += __shfl_xor(part, 16);
        part += __shfl_xor(part, 32);
        sum += g == h ? part : 0.f;
      }
    }
    if (to) *to = old + sum;
  }
}

// Many rows (a prompt's chunk): every wave has 64 keys in registers, as the A operand of S^T = K Q^T with 32x32x16 products, and goes through the rows 32 at a time, which the workgroup brings into
// LDS.  A lane then has one row's scores with 32 of the keys, so one reference a tile, and sums of its own for each key, which are added up over the lanes once at the end.  The keys' two blocks of 32 take
// turns: one's exponentials run beside the other's products.
// Bound: the vector unit: 64 scores at D 128 take the matrix core of a SIMD 16 cycles and its vector unit 24, an exponential of 16 and a fused multiply-add and an addition of 4 each, with about a quarter more
// for rows and masks.  2048 tokens of 32 heads of 128 on 32K keys 547 us, 0.98 PFLOP/s (exponentials behind all products of a tile 655; four waves of 32 keys
// a SIMD, which overlap by themselves, 631).
// Where few keys meet many rows (a prompt's first chunk) 256 keys a workgroup leave compute units without any: the waves then have the same 64 keys and every fourth tile of rows, whose operands they
// read from memory themselves (2048 tokens on themselves 171 -> 67 us, 500 50 -> 21; but 2048 on 8192 keys, an item for every unit, 189 -> 264).
template <int D>
struct Many {
  static constexpr int RB = 2 * D, TILE = 32 * RB;             // bytes of a row, of a tile of rows
  static constexpr int SUMS = 4 * 64 * 33 * 4;                 // where the waves add up their lanes' sums
  static constexpr int LDS = 2 * TILE > SUMS ? 2 * TILE : SUMS;
};
// Every 32nd or 128th row of an item, a (token, query head) pair: where it is, by additions.
struct RowStep {
  int t, j;
  int64_t off, wrap;
};
__device__ __forceinline__ RowStep row_step(const WeighParams& p, int rows, int64_t sh, int64_t ss) {
  const int t = uniform(divide(p.by_gq, rows)), j = rows - t * p.gq;
  return RowStep{t, j, j * sh + t * ss, ss - p.gq * sh};
}
struct Row {
  int t, j;
  int64_t off;
};
__device__ __forceinline__ Row row_at(const WeighParams& p, int r, int64_t sh, int64_t ss) {
  const int t = divide(p.by_gq, r), j = r - t * p.gq;
  return Row{t, j, j * sh + t * ss};
}
__device__ __forceinline__ void advance(const WeighParams& p, Row& r, const RowStep& by) {
  r.t += by.t;
  r.off += by.off;
  if (by.j == 0) return;
  r.j += by.j;
  if (r.j >= p.gq) {
    r.j -= p.gq;
    r.t++;
    r.off += by.wrap;
  }
}
template <int D, bool F8, bool TOGETHER>   // TOGETHER: the waves of a workgroup have the same 64 keys, and every fourth tile of rows, which they read for themselves
__device__ __forceinline__ void weigh_rows(const WeighParams& p, const RowClass& c, const Plan& plan, char* lds) {
  typedef Many<D> M;
  constexpr int KS = D / 16, CPR = D / 8, LOADS = M::TILE / 4096, EACH = 16 / KS;   // 16-byte loads a thread and tile; exponentials a product
  constexpr int WIDTH = TOGETHER ? 64 : kManyKeys, STEP = TOGETHER ? 4 : 1;         // keys of an item; from a wave's tile to its next one
  const int total = uniform(all_items<WIDTH>(p, c, plan)), each = (total + 7) >> 3, base = ((int)blockIdx.x & 7) * each;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));   // (or what follows from it is held, in a mixture, over the few rows' turn)
  const int lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, hf = lane >> 5;
  const float c2 = p.scale * kLog2e;
  const RowStep q_step = row_step(p, 32 * STEP, p.q_sh, p.q_ss), l_step = row_step(p, 32 * STEP, p.l_sh, p.l_ss);
#pragma unroll 1
  for (int at = (int)blockIdx.x >> 3; at < each && base + at < total; at += (int)gridDim.x >> 3) {
    WeighItem w;
    item_at<WIDTH>(p, c, plan, base + at, w);
    const int key0 = TOGETHER ? w.k0 : w.k0 + wave * 64, rows = w.q.n * p.gq;
    // rows from the first that sees the item's first key
    const int first = (p.causal ? clamped(w.k0 - w.q.pos, 0, w.q.n) * p.gq / 32 : 0) + (TOGETHER ? wave : 0), tiles = (rows + 31) / 32;
    const __bf16* const q_base = p.q + (int64_t)w.hk * p.gq * p.q_sh + (int64_t)w.q.start * p.q_ss;
    const float* const l_base = p.lse + (int64_t)w.hk * p.gq * p.l_sh + (int64_t)w.q.start * p.l_ss;
    Row q_row[TOGETHER ? 1 : LOADS], l_row = row_at(p, first * 32 + l32, p.l_sh, p.l_ss);   // of the next tile to be fetched
#pragma unroll
    for (int i = 0; i < (TOGETHER ? 1 : LOADS); i++) q_row[i] = row_at(p, first * 32 + (TOGETHER ? l32 : (i * 256 + tid) / CPR), p.q_sh, p.q_ss);
    u32x4 coming[LOADS];
    const __bf16* lane_row = q_base;   // together: the lane's row of the next tile
    float lse_coming;
    int t_coming;
    auto fetch = [&]() __attribute__((always_inline)) {   // (in the place of rows behind the last the first is read)
      if constexpr (TOGETHER) {
        lane_row = q_base + (q_row[0].t < w.q.n ? q_row[0].off : 0) + (F8 ? 16 : 8) * hf;
        advance(p, q_row[0], q_step);
      }
#pragma unroll
      for (int i = 0; i < LOADS && !TOGETHER; i++) {
        const int64_t off = q_row[i].t < w.q.n ? q_row[i].off : 0;
        coming[i] = *reinterpret_cast<const u32x4*>(q_base + off + tid % CPR * 8);
        advance(p, q_row[i], q_step);
      }
      t_coming = l_row.t;
      lse_coming = l_base[l_row.t < w.q.n ? l_row.off : 0];
      advance(p, l_row, l_step);
    };
    auto put = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LOADS; i++) {
        const int r = (i * 256 + tid) / CPR, c = tid % CPR;
        *reinterpret_cast<u32x4*>(lds + (tile & 1) * M::TILE + r * M::RB + ((c ^ (r % CPR)) << 4)) = coming[i];
      }
    };
    // of the lane's row: what its exponents have taken off (infinity: it adds nothing), and the keys that it sees, from key0 on
    struct Shown { float ref; int limit; };
    auto shown = [&]() __attribute__((always_inline)) -> Shown {
      const bool live = t_coming < w.q.n && fabsf(lse_coming) < INFINITY;
      return Shown{live ? lse_coming * kLog2e : INFINITY, live ? visible(w.q, t_coming, p.causal) - key0 : 0};
    };
    const unsigned operand0 = l32 * M::RB + ((l32 % CPR ^ (F8 ? 2 * hf : hf)) << 4);   // of the lane's chunk 0
    auto operand = [&](unsigned tile0, int ks) __attribute__((always_inline)) -> bf16x8 {
      const int c = F8 ? 4 * (ks >> 1) + (ks & 1) : 2 * ks;
      if constexpr (TOGETHER) return *reinterpret_cast<const bf16x8*>(lane_row + 8 * c);
      return *reinterpret_cast<const bf16x8*>(lds + (tile0 ^ (c << 4)));
    };

    bf16x8 kf[2][KS];   // lane (l, hf): K[l][d's of the load order]
#pragma unroll
    for (int h = 0; h < 2; h++) {
      Slot s = {-1, 0};
      if (key0 + 32 * h + l32 < w.seen) s = slot_of(p.seq, w.b, key0 + 32 * h + l32);
      const char* const kp = p.k_pages + (int64_t)max(s.page, 0) * p.page_b + (int64_t)w.hk * p.head_b + (int64_t)s.slot * p.slot_b + hf * 16;
      unsigned e = 127;
      if (F8 && s.page >= 0) e = p.k_scales[(int64_t)s.page * p.scale_sp + (int64_t)w.hk * p.scale_sh + s.slot];
#pragma unroll
      for (int l = 0; l < (F8 ? KS / 2 : KS); l++) {
        u32x4 x = {0, 0, 0, 0};
        if (s.page >= 0) x = *reinterpret_cast<const u32x4*>(kp + 32 * l);
        if constexpr (F8) {   // 16 d's: those of two products
          kf[h][2 * l] = __builtin_bit_cast(bf16x8, u32x4{f8_pair(x[0], false, e), f8_pair(x[0], true, e), f8_pair(x[1], false, e), f8_pair(x[1], true, e)});
          kf[h][2 * l + 1] = __builtin_bit_cast(bf16x8, u32x4{f8_pair(x[2], false, e), f8_pair(x[2], true, e), f8_pair(x[3], false, e), f8_pair(x[3], true, e)});
        } else {
          kf[h][l] = __builtin_bit_cast(bf16x8, x);
        }
      }
    }
    float acc[2][16];
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int i = 0; i < 16; i++) acc[h][i] = 0.f;

    __syncthreads();   // the sums of the item before have been read
    fetch();
    if constexpr (!TOGETHER) put(first);
    Shown now = shown();
    if constexpr (!TOGETHER) {
      fetch();
      __syncthreads();
    }
    f32x16 s[2];     // scores of the two blocks of 32 keys: one's exponentials beside the other's products
    bf16x8 qf[KS];   // operands of the rows whose products come next
#pragma unroll
    for (int ks = 0; ks < KS; ks++) qf[ks] = operand(operand0 + (first & 1) * M::TILE, ks);
#pragma unroll
    for (int i = 0; i < 16; i++) s[0][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0][ks], qf[ks], s[0], 0, 0, 0);
    // Exponentials of tile t: the first block's beside the second's products with the same rows, the second's beside the first's with the next ones, whose operands are fetched in between.
    auto step = [&](int t, auto masked_c) __attribute__((always_inline)) {
      constexpr bool MASKED = decltype(masked_c)::value;
      const unsigned tile0 = operand0 + ((t + 1) & 1) * M::TILE;
      float ref = now.ref;
      asm volatile("" : "+v"(ref));   // (or, as at the sums, the compiler draws what both kinds of steps have in common out of them, and spills registers)
#pragma unroll
      for (int h = 0; h < 2; h++) {
#pragma unroll
        for (int i = 0; i < 16; i++) s[1 - h][i] = 0.f;
        float x[16];
        auto take = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
          for (int i = i0; i < i0 + EACH; i++) {
            acc[h][i] += !MASKED || 32 * h + 8 * (i >> 2) + 4 * hf + (i & 3) < now.limit ? x[i] : 0.f;
            asm volatile("" : "+v"(acc[h][i]));
          }
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
          s[1 - h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[1 - h][ks], qf[ks], s[1 - h], 0, 0, 0);
          if (h == 0) qf[ks] = operand(tile0, ks);
#pragma unroll
          for (int i = ks * EACH; i < (ks + 1) * EACH; i++) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][i], c2, -ref));
          if (ks > 0) take((ks - 1) * EACH);
          __builtin_amdgcn_sched_barrier(0);
        }
        take(16 - EACH);
      }
    };
    int t = first;
    auto turn = [&](auto masked_c) __attribute__((always_inline)) {
      // (behind the last tile: rows that add nothing)
      if constexpr (TOGETHER) {
        fetch();
        step(t, masked_c);
        now = shown();
      } else {
        put(t + 1);
        const Shown next = shown();
        fetch();
        __syncthreads();
        step(t, masked_c);
        now = next;
      }
      t += STEP;
    };
    while (t < tiles) {   // (a loop for either kind: where they meet the compiler moves all sums from some registers to others)
#pragma unroll 1
      while (t < tiles && !__any(now.limit < 64)) turn(std::false_type{});
#pragma unroll 1
      while (t < tiles && __any(now.limit < 64)) turn(std::true_type{});
    }
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(lds) + wave * 64 * 33;
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int i = 0; i < 16; i++) sums[(32 * h + 8 * (i >> 2) + 4 * hf + (i & 3)) * 33 + l32] = acc[h][i];
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; i++) sum += sums[lane * 33 + i];
    if constexpr (TOGETHER) {
      __syncthreads();
      float* const of_waves = reinterpret_cast<float*>(lds);
      of_waves[tid] = sum;
      __syncthreads();
      if (wave == 0) add_weight(p, w, key0 + lane, (of_waves[lane] + of_waves[64 + lane]) + (of_waves[128 + lane] + of_waves[192 + lane]));
    } else {
      add_weight(p, w, key0 + lane, sum);
    }
  }
}
template <int D, bool F8>
__device__ __forceinline__ void weigh_many(const WeighParams& p, const RowClass& c, const Plan& plan, int together_below, char* lds) {
  if (uniform(all_items<kManyKeys>(p, c, plan)) < together_below) weigh_rows<D, F8, true>(p, c, plan, lds);
  else weigh_rows<D, F8, false>(p, c, plan, lds);
}

// In a mixture half of the workgroups begin with one kind of sequences and half with the other, so that the loads of few rows and the products of many run at
// the same time (a prompt of 700 tokens among 15 single ones, 24 heads of 64, 4000 keys: 51 us, in two launches 56).
// Few keys meet many rows sooner here (8 heads of 128 for 32: a prompt of 512 on 2000 keys among 15 54 -> 32 us with 64 keys a workgroup, of 256 on 3900 45 -> 42, but on 5000 44 -> 51), unless the
// sequences are a handful, which may all have many (2 of 100 tokens on 4000 keys 13 us, with the other limit 20, 4 of 128 on 1000 17.6 and 19.9; mixtures lose by that: 7 with a prompt of 256 on 4500 42 and 36).
constexpr RowClass kAny = {32, 0, 0x7fffffff}, kFewRows = {32, 0, 32}, kManyMore = {32, 32, 0x7fffffff};
template <int D, bool F8, bool APART>   // APART: the other launch has the other sequences
__global__ void __launch_bounds__(256, kFewWaves) weigh_few_kernel(const WeighParams p) {
  weigh_few<D, F8>(p, APART ? RowClass{32, 0, kApartRows} : kAny, sums_plan(p), (int)blockIdx.x >> 3);
}
template <int D, bool F8, bool APART>
__global__ void __launch_bounds__(256, 2) weigh_many_kernel(const WeighParams p) {
  __shared__ __attribute__((aligned(1024))) char lds[Many<D>::LDS];
  weigh_many<D, F8>(p, APART ? RowClass{32, kApartRows, 0x7fffffff} : kAny, sums_plan(p), kTogetherBelow, lds);
}
template <int D, bool F8>
__global__ void __launch_bounds__(256, 2) weigh_mixed_kernel(const WeighParams p) {
  __shared__ __attribute__((aligned(1024))) char lds[Many<D>::LDS];
  const Plan plan = sums_plan(p);
  const int first = (int)blockIdx.x >> 3 & 1;
#pragma unroll 1
  for (int turn = 0; turn < 2; turn++) {
    if (turn == first) weigh_many<D, F8>(p, kManyMore, plan, p.seq.n < kSmallMixture ? kTogetherBelow : kTogetherInMixture, lds);
    else weigh_few<D, F8>(p, kFewRows, plan, ((int)gridDim.x - 1 - (int)blockIdx.x) >> 3);   // (from the last workgroup on: where there are few items, none has one of either kind)
  }
}

template <int D, bool F8>
hipError_t launch_form(const WeighParams& p, hipStream_t stream) {
  const int64_t max_keys = (int64_t)p.seq.max_pages * p.seq.page_size;
  const WeighForm form = weigh_form(p.seq.tokens, p.seq.n, p.gq, p.Hkv, max_keys);
  auto items = [&](int64_t width) { return (int64_t)p.seq.n * p.Hkv * ((max_keys + width - 1) / width); };
  auto grid = [](int64_t wanted, int64_t most) { return dim3((unsigned)((wanted < most ? wanted : most) + 7) / 8 * 8); };   // most: workgroups that the compute units hold
  const dim3 block(256), few = grid(items(kFewKeys), 256 * kFewWaves), many = grid(items(64), 512), both = grid(items(64) + 8, 512);   // (a mixture's two kinds are rounded up apart)
  if (form == kWeighFew) return launch_kernel(weigh_few_kernel<D, F8, false>, few, block, 0, stream, p);
  if (form == kWeighMany) return launch_kernel(weigh_many_kernel<D, F8, false>, many, block, 0, stream, p);
  if (form == kWeighMixed) return launch_kernel(weigh_mixed_kernel<D, F8>, both, block, 0, stream, p);
  const hipError_t e = launch_kernel(weigh_few_kernel<D, F8, true>, few, block, 0, stream, p);
  return e != hipSuccess ? e : launch_kernel(weigh_many_kernel<D, F8, true>, many, block, 0, stream, p);
}

}  // namespace

hipError_t launch_cache_weigh(const WeighParams& p, int D, bool f8, hipStream_t stream) {
  if (D == 128) return f8 ? launch_form<128, true>(p, stream) : launch_form<128, false>(p, stream);
  return f8 ? launch_form<64, true>(p, stream) : launch_form<64, false>(p, stream);
}

}  // namespace tr
