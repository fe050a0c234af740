// Attention of new tokens on a paged cache (tr_paged_attn) for gfx950.
#pragma once
#include "paged.h"

namespace tr {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
// Largest sum of the 8 or 16 weights that a lane takes at a time before the row's reference is replaced.  Weights and their sums would allow 2^80 and more, but the accumulators
// hold weight * V: with at most 2^20 a weight, sums over n keys are finite for |V| * n up to 2^107 (e4m3 pages hold values up to 2^128).  A score
// has to pass the first ones' largest by 13 (natural units) before a reference is replaced.  Against a cap of 2^80: scores of deviation 1 no difference (500 tokens at 12K 115.2 and 115.2 us), of
// deviation 6 119.5 for 117.6, 2048 tokens at 30K in 8 bits 990 for 983, few rows none.
constexpr float kSumCap = 0x1p20f;

// ---- Which work a workgroup has.
//
// The lengths lie in device memory, so the launch does not know them: it has as many workgroups as the shapes allow work items, and every
// workgroup finds its own item, by sums over the sequences that each of its waves takes for itself (64 sequences a load).  An item
// is a row tile of a K/V head of a sequence on one part of the keys (part_keys).
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
__device__ __forceinline__ Sequence lane_sequence(const PagedParams& p, const Plan& plan, int b0) {
  const int b = b0 + (int)(threadIdx.x & 63);
  return b0 == 0 ? plan.first : b < plan.n ? sequence(p.seq, b) : Sequence{0, 0, 0, 0};
}
__device__ __forceinline__ Plan make_plan(const PagedParams& p) {
  Plan plan;
  const int lane = threadIdx.x & 63;
  plan.n = p.seq.n;
  plan.first = Sequence{0, 0, 0, 0};
  if (lane < plan.n) plan.first = sequence(p.seq, lane);
  int64_t work = 0, tiles = 0;
  int longest = 0;
  if (p.share.most_per_unit > 0) {
    for (int b0 = 0; b0 < plan.n; b0 += 64) {
      const Sequence q = lane_sequence(p, plan, b0);
      const int n = tiles_of(q.n * p.gq, p.rows);
      work += (int64_t)n * steps_of(q.len);
      tiles += n;
      if (n > 0) longest = max(longest, steps_of(q.len));
    }
    work = wave_sum(work) * p.Hkv;
    tiles = wave_sum(tiles) * p.Hkv;
    longest = wave_max(longest);
  }
  plan.part = uniform(part_keys(work, tiles, longest, p.share));
  return plan;
}

// Sums count(sequence) over the sequences up to the one that holds element `at`: true, and its number and the sum before it; false, and the sum of all.
template <typename Count>
__device__ __forceinline__ bool locate(const PagedParams& p, const Plan& plan, int at, Count count, int& b, int& before) {
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
template <typename Count>
__device__ __forceinline__ int sum_before(const PagedParams& p, const Plan& plan, int end, Count count) {
  int sum = 0;
  for (int b0 = 0; b0 < end; b0 += 64) {
    const int c = b0 + (int)(threadIdx.x & 63) < end ? count(lane_sequence(p, plan, b0)) : 0;
    sum += __builtin_amdgcn_readlane(wave_scan(c), 63);
  }
  return sum;
}

struct Item {
  int rows;                         // of the sequence and a K/V head
  int b, hk, tile, part, n_parts;   // n_parts: live ones, those whose keys some row of the tile sees, and the first one
  int k0, k1;                       // its keys
  int slot;                         // of the scratch, if n_parts > 1
  Sequence q;
};

// Rows of a tile see keys 0 .. limit(row) - 1; row r of a sequence and K/V head is query head r mod gq of token r / gq.
__device__ __forceinline__ int row_limit(const PagedParams& p, const Sequence& q, int r) { return visible(q, divide(p.by_gq, r), p.causal); }
__device__ __forceinline__ Sequence uniform_sequence(const PagedParams& p, int b) {   // (loaded by vectors, in scalar registers from here on)
  const Sequence q = sequence(p.seq, b);
  return Sequence{uniform(q.start), uniform(q.n), uniform(q.len), uniform(q.pos)};
}

// Item `id` of the launch; false: none (it lies behind the last one, or its part has no live keys).  The items of a K/V head and part lie next to each
// other, and each XCD has a contiguous eighth of all, so that row tiles which read the same keys mostly share an L2.
__device__ __forceinline__ bool find_item(const PagedParams& p, const Plan& plan, int id, Item& w) {
  const int part = plan.part;
  auto items = [&](const Sequence& q) { return tiles_of(q.n * p.gq, p.rows) * parts_of(q.len, part) * p.Hkv; };
  int before, b = 0;
  locate(p, plan, 0x7fffffff, items, b, before);
  const int total = before, each = (total + 7) >> 3, at = (id & 7) * each + (id >> 3);
  if ((id >> 3) >= each || at >= total) return false;
  if (!locate(p, plan, at, items, b, before)) return false;
  w.b = uniform(b);
  w.q = uniform_sequence(p, w.b);
  w.rows = uniform(w.q.n * p.gq);
  const int parts = uniform(parts_of(w.q.len, part)), tiles = uniform(tiles_of(w.rows, p.rows)), i = uniform(at - before);
  const int unit = uniform(i / tiles);        // K/V head, part
  w.tile = tiles - 1 - (i - unit * tiles);    // the last tiles, which see the most keys, first
  w.hk = uniform(unit / parts);
  w.part = unit - w.hk * parts;
  const int last = min((w.tile + 1) * p.rows.tile, w.rows) - 1;
  const int seen = uniform(row_limit(p, w.q, last));
  w.n_parts = parts_of(seen, part);
  w.k0 = w.part * part;
  w.k1 = w.part + 1 < w.n_parts ? w.k0 + part : seen;
  if (w.part >= w.n_parts) return false;
  w.slot = 0;
  if (parts > 1) {   // its scratch slot: among the items of sequences whose keys are cut
    const int base = sum_before(p, plan, w.b, [&](const Sequence& q) {
      const int n = parts_of(q.len, part);
      return n > 1 ? tiles_of(q.n * p.gq, p.rows) * n * p.Hkv : 0;
    });
    w.slot = base + (w.hk * tiles + w.tile) * parts + w.part;
    if (w.slot < 0 || w.slot >= p.slots) return false;   // (only where sequences overlap)
  }
  return true;
}

// Of two bf16: the top bit of each half whose exponent is all ones.  (In integers: as conditions, many of them spill the scalar registers.)
__device__ __forceinline__ unsigned not_finite(unsigned pair) { return ((pair & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// 16 bytes (fp32) of a row's result, piece c of row row0 + r of the item, to where they belong; with piece 0 the row's lse (NaN: a weight was one).
template <int D, bool OUT_F32>
__device__ __forceinline__ void store_piece(const PagedParams& p, const Item& w, int row0, int slot_row, int r, int c, f32x4 o, float lse) {
  if (w.n_parts > 1) {
    const int64_t at = (int64_t)slot_row + r;
    *reinterpret_cast<f32x4*>(p.part_out + at * D + 4 * c) = o;
    if (c == 0) p.part_lse[at] = lse;
    return;
  }
  const int t = divide(p.by_gq, row0 + r), head = w.hk * p.gq + row0 + r - t * p.gq;
  const int64_t at = (int64_t)head * p.o_sh + (int64_t)(w.q.start + t) * p.o_ss + 4 * c;
  if constexpr (OUT_F32) {
    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(p.out) + at) = o;
  } else {
    bf16x4 ob;
#pragma unroll
    for (int k = 0; k < 4; k++) ob[k] = (__bf16)o[k];
    *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(p.out) + at) = ob;
  }
  if (c == 0) p.lse[(int64_t)head * p.l_sh + (int64_t)(w.q.start + t) * p.l_ss] = lse != lse ? -INFINITY : lse;
}

// ---- Few rows.
//
// Items of at most 16 * RT rows (a decode step's query heads of a K/V head, drafted tokens).  Each of the four waves takes every fourth
// stretch of 32 keys on its own, straight from memory into registers, and the waves' results are added up at the end.  Scores are computed
// transposed, S^T = K Q^T, with 16x16x32 products: A is K as it lies in memory, lane (i = lane % 16, g = lane / 16) then holds
// scores of row i for keys 4g .. 4g + 3 of each 16.  In this order the exponentials are the B operand of O^T = V^T P^T (a contraction index may
// be permuted if both operands agree): its A operand needs 8 keys of one d in a lane, and a lane that loads D / 16 adjacent d's of those 8 keys has them after
// one exchange of 16-bit halves.  No LDS, no barrier inside the loop.  Bound: HBM, and where few keys are left to a workgroup the latency of its set-up and
// loads.  64 sequences of 0.8K to 16K keys on 8 K/V heads of 128: in 8 bits 215 us, 5.2 TB/s; 4 of 8K in bf16 27 us, 4.7 TB/s; a step of 128 keys takes a workgroup that
// has its unit to itself 1.1 us at D 128, 0.73 at D 64, the rest of it 5 (32 rows: 1.16 and 0.75).
template <int D, bool F8, int RT, int W>
struct Few {
  static constexpr int TILE = 16 * RT, DL = D / 16;              // rows of a tile; d's of a lane in V
  static constexpr int KL = F8 ? D / 64 : D / 32, VW = (F8 ? DL : 2 * DL) / 4;   // 16-byte loads of a K row's quarter, words of V a key
  static constexpr int LDS = W * TILE * (D + 2) * 4;
};

template <int D, bool F8, int RT, int W, bool AHEAD, bool OUT_F32>   // AHEAD: the next stretch is on its way beside the products (it takes registers)
__device__ __forceinline__ void few_rows(const PagedParams& p, const Item& w, int row0, int slot_row, char* lds) {
  typedef Few<D, F8, RT, W> F;
  constexpr int STEP = 32 * W;   // keys of a step of the workgroup
  constexpr int TILE = F::TILE, DL = F::DL, KL = F::KL, VW = F::VW, QS = D / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), i16 = lane & 15, g = lane >> 4;
  const int rows = min(TILE, w.q.n * p.gq - row0);
  const int limit_lo = row_limit(p, w.q, row0), limit_hi = min(w.k1, row_limit(p, w.q, row0 + rows - 1));

  bf16x8 qf[RT][QS];
  int limit[RT];
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    const int r = row0 + min(rt * 16 + i16, rows - 1), t = divide(p.by_gq, r);
    limit[rt] = min(w.k1, visible(w.q, t, p.causal));
    const __bf16* const src = p.q + (int64_t)(w.hk * p.gq + r - t * p.gq) * p.q_sh + (int64_t)(w.q.start + t) * p.q_ss;
#pragma unroll
    for (int s = 0; s < QS; s++)   // d's in the order of the K loads
      qf[rt][s] = *reinterpret_cast<const bf16x8*>(src + (F8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8));
  }
  const char* const kb = p.k_pages + (int64_t)w.hk * p.head_b;
  const char* const vb = p.v_pages + (int64_t)w.hk * p.head_b;
  const unsigned char* const ksb = p.k_scales + (int64_t)w.hk * p.scale_sh;
  const unsigned char* const vsb = p.v_scales + (int64_t)w.hk * p.scale_sh;
  const int k_lane = i16 * p.slot_b + g * 16, v_lane = g * 4 * p.slot_b + i16 * VW * 4;

  // Pages of the wave's groups of 16 keys, 32 stretches ahead: lane 2 j + h has those of group h of stretch j.
  const int steps = (w.k1 - w.k0 + STEP - 1) / STEP;
  Slot at = {-1, 0};
  auto find_pages = [&](int step) __attribute__((always_inline)) {
    const int key = w.k0 + (step + (lane >> 1)) * STEP + wave * 32 + (lane & 1) * 16;
    at = Slot{-1, 0};
    if (key < w.k1) at = slot_of(p.seq, w.b, key);
  };
  // A stretch's K and V, each renewed as soon as its product has been taken: K of the next stretch is on its way beside this one's weights and second
  // product, V beside the next one's first.
  u32x4 kr[2][KL];
  unsigned vr[8][VW], k_scale[2], v_scale[2];
  bool k_there[2];     // the two groups of 16 keys lie on pages
  auto load_k = [&](int step) __attribute__((always_inline)) {
    if ((step & 31) == 0) find_pages(step);
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int page = __builtin_amdgcn_readlane(at.page, ((step & 31) << 1) + h), slot = __builtin_amdgcn_readlane(at.slot, ((step & 31) << 1) + h);
      k_there[h] = page >= 0;
      if (page >= 0) {
        const char* const kp = kb + (int64_t)page * p.page_b + (int64_t)slot * p.slot_b;
#pragma unroll
        for (int l = 0; l < KL; l++) kr[h][l] = *reinterpret_cast<const u32x4*>(kp + k_lane + l * 64);
        if constexpr (F8) k_scale[h] = ksb[(int64_t)page * p.scale_sp + slot + i16];
      } else {
#pragma unroll
        for (int l = 0; l < KL; l++) kr[h][l] = u32x4{0, 0, 0, 0};
        if constexpr (F8) k_scale[h] = 127;
      }
    }
  };
  auto load_v = [&](int step) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int page = __builtin_amdgcn_readlane(at.page, ((step & 31) << 1) + h), slot = __builtin_amdgcn_readlane(at.slot, ((step & 31) << 1) + h);
      if (page >= 0) {
        const char* const vp = vb + (int64_t)page * p.page_b + (int64_t)slot * p.slot_b;
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const char* const src = vp + v_lane + e * p.slot_b;
          if constexpr (VW == 4) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(src);
#pragma unroll
            for (int i = 0; i < 4; i++) vr[4 * h + e][i] = x[i];
          } else if constexpr (VW == 2) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(src);
            vr[4 * h + e][0] = x[0];
            vr[4 * h + e][1] = x[1];
          } else {
            vr[4 * h + e][0] = *reinterpret_cast<const unsigned*>(src);
          }
        }
        if constexpr (F8) v_scale[h] = *reinterpret_cast<const unsigned*>(vsb + (int64_t)page * p.scale_sp + slot + 4 * g);
      } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
#pragma unroll
          for (int i = 0; i < VW; i++) vr[4 * h + e][i] = 0;
        if constexpr (F8) v_scale[h] = 0x7f7f7f7f;
      }
    }
  };

  f32x4 acc[RT][DL];
  float m_ref[RT], mc[RT], l_run[RT];
  const float c2 = p.scale * kLog2e;
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    m_ref[rt] = mc[rt] = -INFINITY;
    l_run[rt] = 0.f;
#pragma unroll
    for (int j = 0; j < DL; j++) acc[rt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  unsigned taken_out = 0;
  if (AHEAD && steps > 0) {
    load_k(0);
    load_v(0);
  }
#pragma unroll 1
  for (int step = 0; step < steps; step++) {
    const int key0 = w.k0 + step * STEP + wave * 32;
    if (!AHEAD) load_k(step);
    const bool there[2] = {k_there[0], k_there[1]};
    const bool edge = key0 + 32 > limit_lo || key0 + 32 > limit_hi || !there[0] || !there[1];
    // scores
    f32x4 s[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int ks = 0; ks < QS; ks++) {
        bf16x8 a;
        if constexpr (F8) {
          const u32x4 x = kr[h][ks >> 1];
          const unsigned lo = x[(ks & 1) * 2], hi = x[(ks & 1) * 2 + 1], e = k_scale[h];
          a = __builtin_bit_cast(bf16x8, u32x4{f8_pair(lo, false, e), f8_pair(lo, true, e), f8_pair(hi, false, e), f8_pair(hi, true, e)});
        } else {
          a = __builtin_bit_cast(bf16x8, kr[h][ks]);
        }
#pragma unroll
        for (int rt = 0; rt < RT; rt++) s[rt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[rt][ks], s[rt][h], 0, 0, 0);
      }
    if (AHEAD && step + 1 < steps) load_k(step + 1);
    if (edge) {
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int r = 0; r < 4; r++)
#pragma unroll
          for (int rt = 0; rt < RT; rt++)
            if (key0 + 16 * h + 4 * g + r >= limit[rt] || !there[h]) s[rt][h][r] = -INFINITY;
    }
    // Weights relative to a reference that is not the running maximum: any gives the same result, and one that the
    // first scores set is replaced only where a sum of weights passes kSumCap (fp32 and bf16 hold them as well as small ones).  A row without one has -inf there: its
    // weights are infinite or NaN.
    bf16x8 pf[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
      float e[8], sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][i >> 2][i & 3], c2, -mc[rt]));
        sum += e[i];
      }
      if (__any(!(sum <= kSumCap))) {
        float top = s[rt][0][0];
#pragma unroll
        for (int i = 1; i < 8; i++) top = fmaxf(top, s[rt][i >> 2][i & 3]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m_ref[rt], top);
        const float a = m_ref[rt] == m_new ? 1.f : __builtin_amdgcn_exp2f((m_ref[rt] - m_new) * c2);
        l_run[rt] *= a;
        // acc holds this lane's row in every element, so the factor is the lane's own
#pragma unroll
        for (int j = 0; j < DL; j++)
#pragma unroll
          for (int r = 0; r < 4; r++) acc[rt][j][r] *= a;
        m_ref[rt] = m_new;
        mc[rt] = m_new * c2;
        const float by = m_new == -INFINITY ? 0.f : mc[rt];
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i++) {
          e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][i >> 2][i & 3], c2, -by));
          sum += e[i];
        }
      }
      l_run[rt] += sum;   // (the sums take the weights as they are: rounded ones would put 2^-9 of error into lse)
      // bf16 is what the second product takes: each weight is off by up to 2^-8 of itself, which makes the result's error 2.3e-3 of its size where the result's own rounding to bf16 is 1.7e-3.
#pragma unroll
      for (int i = 0; i < 8; i++) pf[rt][i] = (__bf16)e[i];
    }
    if (!AHEAD) load_v(step);
    // What no row sees takes part in the second product with weight 0: not a value that times 0 is NaN.
    if (edge) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const bool seen = key0 + 16 * (e >> 2) + 4 * g + (e & 3) < limit_hi;
#pragma unroll
        for (int n = 0; n < VW; n++) vr[e][n] = seen ? vr[e][n] : 0;
        if (F8) v_scale[e >> 2] = seen ? v_scale[e >> 2] : v_scale[e >> 2] & ~(128u << 8 * (e & 3));   // (no scale of NaN)
      }
    }
    // A key that some rows see and others do not, with an infinity or NaN in V: taken out of the product, and added below to the rows that see it.
    if (limit_lo < min(key0 + 32, limit_hi)) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
#pragma unroll
        for (int n = 0; n < VW; n++) {
          if constexpr (F8) {
#pragma unroll
            for (int u = 0; u < 2; u++) {
              const unsigned nf = not_finite(f8_pair(vr[e][n], u, v_scale[e >> 2] >> (8 * (e & 3)) & 255));
              taken_out |= nf;
              vr[e][n] &= ~(((nf >> 15 & 1) * 0xffu | (nf >> 31) * 0xff00u) << 16 * u);
            }
          } else {
            const unsigned nf = not_finite(vr[e][n]);
            taken_out |= nf;
            vr[e][n] &= ~(nf | (nf - (nf >> 15)));
          }
        }
        if (F8 && (v_scale[e >> 2] >> (8 * (e & 3)) & 255) == 255) v_scale[e >> 2] &= ~(128u << 8 * (e & 3));   // (all of the row is out)
      }
    }
    // V^T: d's 2 n and 2 n + 1 of a key lie in one word; pairs of keys of one d are what the product takes
#pragma unroll
    for (int n = 0; n < DL / 2; n++) {
      unsigned vt[2][4];
#pragma unroll
      for (int m = 0; m < 4; m++) {
        unsigned a, b;
        if constexpr (F8) {
          const int h = m >> 1;
          a = f8_pair(vr[2 * m][n >> 1], n & 1, v_scale[h] >> (16 * (m & 1)) & 255);
          b = f8_pair(vr[2 * m + 1][n >> 1], n & 1, v_scale[h] >> (16 * (m & 1) + 8) & 255);
        } else {
          a = vr[2 * m][n];
          b = vr[2 * m + 1][n];
        }
        vt[0][m] = __builtin_amdgcn_perm(b, a, 0x05040100);
        vt[1][m] = __builtin_amdgcn_perm(b, a, 0x07060302);
      }
#pragma unroll
      for (int j = 0; j < 2; j++)
#pragma unroll
        for (int rt = 0; rt < RT; rt++)
          acc[rt][2 * n + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{vt[j][0], vt[j][1], vt[j][2], vt[j][3]}), pf[rt], acc[rt][2 * n + j], 0, 0, 0);
    }
    if (AHEAD && step + 1 < steps) load_v(step + 1);
  }
  if (__any(taken_out != 0)) {   // (the rows they reach are infinite or NaN whatever else adds up)
#pragma unroll 1
    for (int key = w.k0 + wave * 32; key < limit_hi; key += (key & 31) == 31 ? STEP - 31 : 1) {
      if (limit_lo >= min((key | 31) + 1, limit_hi)) continue;
      const Slot one = slot_of(p.seq, w.b, key);
      if (one.page < 0) continue;
      const char* const vp = vb + (int64_t)one.page * p.page_b + (int64_t)one.slot * p.slot_b + g * 16 * VW;
      const unsigned scale = F8 ? vsb[(int64_t)one.page * p.scale_sp + one.slot] : 0;
#pragma unroll
      for (int i = 0; i < 4 * VW; i++) {   // the lane's 4 * DL values, d = 4 g DL + ...
        const unsigned x = reinterpret_cast<const unsigned*>(vp)[i];
#pragma unroll
        for (int n = 0; n < (F8 ? 2 : 1); n++) {
          const unsigned pair = F8 ? f8_pair(x, n, scale) : x;
          const int e = F8 ? 4 * i + 2 * n : 2 * i;
#pragma unroll
          for (int rt = 0; rt < RT; rt++) {
            if (key < limit[rt] && (pair & 0x7f80u) == 0x7f80u) acc[rt][e % DL][e / DL] += __builtin_bit_cast(float, pair << 16);
            if (key < limit[rt] && (pair & 0x7f800000u) == 0x7f800000u) acc[rt][e % DL + 1][e / DL] += __builtin_bit_cast(float, pair & 0xffff0000u);
          }
        }
      }
    }
  }

  // ---- the waves' results, added up in LDS: [wave][row][D] (16-byte pieces exchanged among each other by the row), then reference and sum of each
  float* const ml = reinterpret_cast<float*>(lds + W * TILE * D * 4);
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    float l = l_run[rt];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const int r = rt * 16 + i16;
    if (g == 0) {
      ml[(wave * TILE + r) * 2] = m_ref[rt];
      ml[(wave * TILE + r) * 2 + 1] = l;
    }
    char* const at_row = lds + (wave * TILE + r) * D * 4;
#pragma unroll
    for (int q = 0; q < 4; q++)
#pragma unroll
      for (int j = 0; j < DL; j += 4) {
        const int c = ((4 * g + q) * DL + j) / 4;
        *reinterpret_cast<f32x4*>(at_row + ((c ^ (r & 15)) << 4)) = f32x4{acc[rt][j][q], acc[rt][j + 1][q], acc[rt][j + 2][q], acc[rt][j + 3][q]};
      }
  }
  __syncthreads();
  constexpr int PIECES = D / 4;
  for (int i = tid; i < rows * PIECES; i += 64 * W) {
    const int r = i / PIECES, c = i % PIECES;
    float m[W], l[W], top = -INFINITY, total = 0.f;
#pragma unroll
    for (int v = 0; v < W; v++) {
      m[v] = ml[(v * TILE + r) * 2];
      l[v] = ml[(v * TILE + r) * 2 + 1];
      top = fmaxf(top, m[v]);
    }
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < W; v++) {
      const float a = m[v] == -INFINITY ? 0.f : m[v] == top ? 1.f : __builtin_amdgcn_exp2f((m[v] - top) * c2);
      const f32x4 x = *reinterpret_cast<const f32x4*>(lds + (v * TILE + r) * D * 4 + ((c ^ (r & 15)) << 4));
      total += a * l[v];
#pragma unroll
      for (int k = 0; k < 4; k++) o[k] += a * x[k];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const float lse = total > 0.f ? top * p.scale + logf(total) : -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; k++) o[k] *= inv;
    store_piece<D, OUT_F32>(p, w, row0, slot_row, r, c, o, total != total ? __builtin_nanf("") : lse);
  }
}

template <int D, bool F8, int RT, bool OUT_F32>
__global__ void __launch_bounds__(256, paged_few_waves(D, F8, RT)) paged_few_kernel(const PagedParams p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  Item w;
  if (!find_item(p, make_plan(p), (int)blockIdx.x, w)) return;
  few_rows<D, F8, RT, 4, true, OUT_F32>(p, w, w.tile * 16 * RT, w.slot * 16 * RT, lds);
}

// ---- Row tiles whose keys were cut (6 us for 32 tiles of 16 rows in 16 parts, 13 for 64 of 256 rows in four, 34 MB): out = sum of exp(lse_i - lse) out_i over their live parts, in their order.
// A workgroup has pieces of 1024 / D rows of a tile, D / 4 lanes a row.  What bounds it is latency: the lanes of a row
// fetch the lse of one part each, and pieces of eight parts are on their way at a time.
template <int D, bool OUT_F32>
__global__ void __launch_bounds__(256) paged_fold_kernel(const PagedParams p) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES, AHEAD = 8;
  const Plan plan = make_plan(p);
  const int part = plan.part, size = p.rows.tile, pieces = max(1, size / ROWS);
  auto cut_tiles = [&](const Sequence& q) { return parts_of(q.len, part) > 1 ? tiles_of(q.n * p.gq, p.rows) * p.Hkv : 0; };
  for (int at = (int)blockIdx.x;; at += (int)gridDim.x) {
  int b, before;
  if (!locate(p, plan, at / pieces, cut_tiles, b, before)) return;
  Item w;
  w.q = uniform_sequence(p, uniform(b));
  w.rows = uniform(w.q.n * p.gq);
  const int base = sum_before(p, plan, uniform(b), [&](const Sequence& q) { return cut_tiles(q) * parts_of(q.len, part); });
  const int parts = uniform(parts_of(w.q.len, part)), tiles = uniform(tiles_of(w.rows, p.rows)), i = uniform(at / pieces - before);
  w.hk = uniform(i / tiles);
  const int row0 = (i - w.hk * tiles) * size, rows = min(size, w.rows - row0);
  const int n_live = uniform(parts_of(row_limit(p, w.q, row0 + rows - 1), part));
  if (n_live == 1) continue;   // one part: written already
  if (base < 0 || base + (i + 1) * parts > p.slots) continue;   // (only where sequences overlap)
  w.n_parts = 1;   // what follows is stored for good
  const int c = (int)threadIdx.x % LANES;
  const int r = at % pieces * ROWS + (int)threadIdx.x / LANES;
  if (r < rows) {
    const int64_t slot_row = ((int64_t)base + (int64_t)i * parts) * size + r;
    const float* const ls = p.part_lse + slot_row;
    const float* const out = p.part_out + slot_row * D + 4 * c;
    float top = -INFINITY;
    bool nan = false;
    for (int k = c; k < n_live; k += LANES) {
      const float x = ls[(int64_t)k * size];
      nan |= x != x;
      top = fmaxf(top, x);
    }
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) {
      top = fmaxf(top, __shfl_xor(top, d));
      nan |= __shfl_xor((int)nan, d) != 0;
    }
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    for (int k0 = 0; k0 < n_live; k0 += LANES) {
      float mine = -INFINITY;   // weight of part k0 + c; -inf, in its place, of a part without a visible key, whose result says nothing
      if (k0 + c < n_live) mine = ls[(int64_t)(k0 + c) * size];
      mine = mine == -INFINITY ? 0.f : expf(mine - top);
      for (int k1 = k0; k1 < min(k0 + LANES, n_live); k1 += AHEAD) {
        f32x4 y[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; j++) y[j] = *reinterpret_cast<const f32x4*>(out + (int64_t)min(k1 + j, n_live - 1) * size * D);
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
          const float a = k1 + j < n_live ? __shfl(mine, k1 - k0 + j, LANES) : 0.f;
          total += a;
#pragma unroll
          for (int e = 0; e < 4; e++) o[e] += a == 0.f ? 0.f : a * y[j][e];
        }
      }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] *= inv;
    store_piece<D, OUT_F32>(p, w, row0, 0, r, c, o, nan ? __builtin_nanf("") : total > 0.f ? top + logf(total) : -INFINITY);
  }
  }
}

}  // namespace
}  // namespace tr
