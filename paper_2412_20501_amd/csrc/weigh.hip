// The attention weight that each key of a paged cache gets from the new tokens (tr_cache_weigh).
//
// weights[c] += sum over rows r that see c of exp(scale <q_r, K_c> - lse_r), a row being a (token, query head of the K/V head) pair: half of an attention's products, one
// exponential a score, and sums down the rows instead of along the keys.  A workgroup has some keys and goes through all rows that see them, so that a
// key's sum is one workgroup's, in one order, and K is read once.
#include "evict.h"
#include "paged_sums.h"

namespace tr {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kFewWaves = 4;     // a SIMD, of few rows
constexpr int kFewKeys = 256;    // of an item of few rows: 64 a wave
constexpr int kManyKeys = 256;   // of many rows

// Items: (sequence, K/V head, stretch of keys) of the launch's sequences, numbered so that those of a head lie together, and each XCD has a contiguous eighth of all.
struct WeighItem {
  int b, hk, k0;   // its keys: k0 .. min(k0 + width, seen) - 1
  int seen;        // keys that some row of the sequence sees (or that start from 0)
  Sequence q;
};
__device__ __forceinline__ int seen_keys(const WeighParams& p, const Sequence& q) { return visible(q, q.n - 1, p.causal); }
template <int WIDTH>
__device__ __forceinline__ int tiles_of_keys(const WeighParams& p, const Sequence& q) {   // of a K/V head
  const int rows = q.n * p.gq;
  return rows > p.rows.over && rows <= p.rows.most ? (seen_keys(p, q) + WIDTH - 1) / WIDTH : 0;
}
__device__ __forceinline__ Plan sums_plan(const WeighParams& p) {
  Plan plan = {p.seq.n, 0, Sequence{0, 0, 0, 0}};
  const int lane = threadIdx.x & 63;
  if (lane < plan.n) plan.first = sequence(p.seq, lane);
  return plan;
}
template <int WIDTH>
__device__ __forceinline__ int all_items(const WeighParams& p, const Plan& plan) {
  int b = 0, total;
  locate(p, plan, 0x7fffffff, [&](const Sequence& q) { return tiles_of_keys<WIDTH>(p, q) * p.Hkv; }, b, total);
  return total;
}
template <int WIDTH>
__device__ __forceinline__ void item_at(const WeighParams& p, const Plan& plan, int at, WeighItem& w) {   // at: below all_items()
  int b = 0, before;
  locate(p, plan, at, [&](const Sequence& q) { return tiles_of_keys<WIDTH>(p, q) * p.Hkv; }, b, before);
  w.b = uniform(b);
  if (w.b < 64) {   // a lane has it
    const Sequence& q = plan.first;
    w.q = Sequence{__builtin_amdgcn_readlane(q.start, w.b), __builtin_amdgcn_readlane(q.n, w.b), __builtin_amdgcn_readlane(q.len, w.b), __builtin_amdgcn_readlane(q.pos, w.b)};
  } else {
    const Sequence q = sequence(p.seq, w.b);
    w.q = Sequence{uniform(q.start), uniform(q.n), uniform(q.len), uniform(q.pos)};
  }
  const int tiles = uniform(tiles_of_keys<WIDTH>(p, w.q)), i = uniform(at - before);
  w.hk = uniform(i / tiles);
  w.k0 = (i - w.hk * tiles) * WIDTH;
  w.seen = uniform(seen_keys(p, w.q));
}
// What a row's exponents have taken off, in powers of two; infinity for rows that add nothing.
__device__ __forceinline__ float row_reference(const WeighParams& p, const WeighItem& w, int r, int rows) {
  if (r >= rows) return INFINITY;
  const int t = divide(p.by_gq, r);
  const float lse = p.lse[(int64_t)(w.hk * p.gq + r - t * p.gq) * p.l_sh + (int64_t)(w.q.start + t) * p.l_ss];
  return fabsf(lse) < INFINITY ? lse * kLog2e : INFINITY;
}
__device__ __forceinline__ const __bf16* row_of(const WeighParams& p, const WeighItem& w, int r) {
  const int t = divide(p.by_gq, r);
  return p.q + (int64_t)(w.hk * p.gq + r - t * p.gq) * p.q_sh + (int64_t)(w.q.start + t) * p.q_ss;
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
// scores of key i with rows 4 g .. 4 g + 3 of 16.  The pages of the next item's keys are on their way beside this one's.  Bound: HBM.
template <int D, bool F8>
__global__ void __launch_bounds__(256, kFewWaves) weigh_few_kernel(const WeighParams p) {
  constexpr int QS = D / 32, KL = F8 ? D / 64 : D / 32;
  const Plan plan = sums_plan(p);
  const int total = uniform(all_items<kFewKeys>(p, plan)), each = (total + 7) >> 3, base = ((int)blockIdx.x & 7) * each, end = min(each, total - base);
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
  const float c2 = p.scale * kLog2e;
  WeighItem w, next;
  Slot mine = {-1, 0};   // of key key0 + lane
  auto find = [&](int at, WeighItem& item, Slot& slot) __attribute__((always_inline)) {
    slot = Slot{-1, 0};
    if (at >= end) return;
    item_at<kFewKeys>(p, plan, base + at, item);
    const int key = item.k0 + wave * 64 + lane;
    if (key < item.seen) slot = slot_of(p.seq, item.b, key);
  };
  find((int)blockIdx.x >> 3, next, mine);
  for (int at = (int)blockIdx.x >> 3; at < end; at += (int)gridDim.x >> 3) {
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

// Many rows (a prompt's chunk): every wave has 64 keys in registers, as the A operand of S^T = K Q^T, and goes through the rows 32 at a time, which the workgroup brings into LDS.
template <int D>
struct Many {
  static constexpr int RB = 2 * D, TILE = 32 * RB;             // bytes of a row, of a tile of rows
  static constexpr int SUMS = 4 * 64 * 33 * 4;                 // where the waves add up their lanes' sums
  static constexpr int LDS = 2 * TILE > SUMS ? 2 * TILE : SUMS;
};
template <int D, bool F8>
__global__ void __launch_bounds__(256, 2) weigh_many_kernel(const WeighParams p) {
  typedef Many<D> M;
  constexpr int KS = D / 16, CPR = D / 8, LOADS = M::TILE / 4096;   // 16-byte loads a thread and tile
  __shared__ __attribute__((aligned(1024))) char lds[M::LDS];
  const Plan plan = sums_plan(p);
  const int total = uniform(all_items<kManyKeys>(p, plan)), each = (total + 7) >> 3, base = ((int)blockIdx.x & 7) * each;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, hf = lane >> 5;
  const float c2 = p.scale * kLog2e;
  for (int at = (int)blockIdx.x >> 3; at < each && base + at < total; at += (int)gridDim.x >> 3) {
    WeighItem w;
    item_at<kManyKeys>(p, plan, base + at, w);
    const int key0 = w.k0 + wave * 64, rows = w.q.n * p.gq;
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

    // rows from the first that sees the item's first key
    const int first = p.causal ? clamped(w.k0 - w.q.pos, 0, w.q.n) * p.gq / 32 : 0, tiles = (rows + 31) / 32;
    u32x4 next[LOADS];
    float next_ref;
    int next_limit;
    auto fetch = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LOADS; i++) {
        const int n = i * 256 + tid, r = n / CPR, c = n % CPR;
        next[i] = *reinterpret_cast<const u32x4*>(row_of(p, w, min(tile * 32 + r, rows - 1)) + 8 * c);
      }
      const int r = tile * 32 + l32;
      next_ref = row_reference(p, w, r, rows);
      next_limit = next_ref == INFINITY ? 0 : visible(w.q, divide(p.by_gq, r), p.causal) - key0;
    };
    auto put = [&](int half) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LOADS; i++) {
        const int n = i * 256 + tid, r = n / CPR, c = n % CPR;
        *reinterpret_cast<u32x4*>(lds + half * M::TILE + r * M::RB + ((c ^ (r % CPR)) << 4)) = next[i];
      }
    };
    __syncthreads();   // the sums of the item before have been read
    if (first < tiles) {
      fetch(first);
      put(first & 1);
    }
    float ref = next_ref;
    int limit = next_limit;
    for (int t = first; t < tiles; t++) {
      if (t + 1 < tiles) fetch(t + 1);
      __syncthreads();
      if (__any(limit > 0)) {
        bf16x8 qf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
          const int c = F8 ? 4 * (ks >> 1) + 2 * hf + (ks & 1) : 2 * ks + hf;
          qf[ks] = *reinterpret_cast<const bf16x8*>(lds + (t & 1) * M::TILE + l32 * M::RB + ((c ^ (l32 % CPR)) << 4));
        }
        const bool masked = __any(limit < 64);
#pragma unroll
        for (int h = 0; h < 2; h++) {
          f32x16 s;
#pragma unroll
          for (int i = 0; i < 16; i++) s[i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < KS; ks++) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[h][ks], qf[ks], s, 0, 0, 0);
          if (masked) {
#pragma unroll
            for (int i = 0; i < 16; i++) {
              const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c2, -ref));
              acc[h][i] += 32 * h + 8 * (i >> 2) + 4 * hf + (i & 3) < limit ? e : 0.f;
            }
          } else {
#pragma unroll
            for (int i = 0; i < 16; i++) acc[h][i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c2, -ref));
          }
        }
      }
      if (t + 1 < tiles) {
        put((t + 1) & 1);
        ref = next_ref;
        limit = next_limit;
      }
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
    add_weight(p, w, key0 + lane, sum);
  }
}

template <int D, bool F8>
hipError_t launch_form(WeighParams& p, hipStream_t stream) {
  const int64_t tokens = p.seq.tokens, n = p.seq.n, max_keys = (int64_t)p.seq.max_pages * p.seq.page_size;
  constexpr int any = 0x7fffffff;
  const int64_t rows = tokens * p.gq;
  const bool mixed = rows > 32 * n && n > 1, few = rows <= 32 * n;
  for (int part = 0; part < (mixed ? 2 : 1); part++) {
    const bool many = mixed ? part == 1 : !few;
    p.rows = mixed ? (many ? RowClass{32, 32, any} : RowClass{32, 0, 32}) : RowClass{32, 0, any};
    const int64_t width = many ? kManyKeys : kFewKeys, seqs = rows / (p.rows.over + 1) < n ? rows / (p.rows.over + 1) : n;
    const int64_t items = seqs * p.Hkv * ((max_keys + width - 1) / width), most = many ? 512 : 256 * kFewWaves;
    if (items == 0) continue;
    const dim3 grid((unsigned)((items < most ? items : most) + 7) / 8 * 8);
    const hipError_t e = many ? launch_kernel(weigh_many_kernel<D, F8>, grid, dim3(256), 0, stream, p) : launch_kernel(weigh_few_kernel<D, F8>, grid, dim3(256), 0, stream, p);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_cache_weigh(WeighParams& p, int D, bool f8, hipStream_t stream) {
  if (D == 128) return f8 ? launch_form<128, true>(p, stream) : launch_form<128, false>(p, stream);
  return f8 ? launch_form<64, true>(p, stream) : launch_form<64, false>(p, stream);
}

}  // namespace tr
