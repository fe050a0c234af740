// Attention on a paged cache: items of many rows (a chunk of a prompt).
#pragma once
#include "paged_attn_kernel.h"

namespace tr {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;

template <int N>
using IC = std::integral_constant<int, N>;

__device__ __forceinline__ void swap_halves(float x, float& lo, float& hi) {   // of a wave: x of lane % 32 and of 32 + lane % 32, in every lane
  float a = x, b = x;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));   // (the builtin's second result is folded into the first at -O3)
  lo = a;
  hi = b;
}
__device__ __forceinline__ float halves_max(float x) {
  float lo, hi;
  swap_halves(x, lo, hi);
  return fmaxf(lo, hi);
}
__device__ __forceinline__ float halves_sum(float x) {
  float lo, hi;
  swap_halves(x, lo, hi);
  return lo + hi;
}

// Many rows.
//
// The block attention kernel's way (256 rows in eight waves of 32, or 128 in four, S^T = K Q^T with 32x32x16 products, P in registers as the B operand of O^T = V^T P^T,
// V read from LDS with the transposing read, one softmax sub-tile behind the products in one instruction stream, rings of four 16 KiB tiles of K
// and of V), on rows that are (token, query head of a K/V head) pairs and with tiles that are gathered from pages: a wave's share of a tile, 8 keys
// at D 128 and 16 at D 64, lies on one page, whose address is found with scalar loads a tile ahead.  bf16 goes straight from memory into LDS, e4m3 through
// registers, where each value is converted once for all 256 rows.  Bound: MFMA and power, as there.  An item takes 1.1 us for 64 keys at D 128 on an idle chip (1.7 on a
// full one), 1.55 for 128 at D 64, and 11 and 8 for its set-up and epilogue; 2048 tokens of 32 heads behind 30K keys in 8 bits 1.06 to 1.19 PFLOP/s (cards differ).
//
// What is rare takes another way: an item with a page that is none, or with an infinity or NaN in V at a key that only some of its rows see, is computed
// by few_rows, 16 rows at a time, which holds nothing of either against it and takes five times as long (500 tokens on 12500 keys 114 us, with one entry that is no page 619).
template <int D, int WAVES>
struct Tile {
  static constexpr int RB = 2 * D, BN = (D == 64 ? 16 : 8) * WAVES, NS = 4, TILE_BYTES = BN * RB, ROWS = 32 * WAVES;
  static constexpr int RINGS = 2 * NS * TILE_BYTES, FLAG = RINGS, OFF = RINGS + 64, LDS = OFF + ROWS * 8;
  static_assert(TILE_BYTES == 2048 * WAVES && WAVES * 32 * 4 * D <= RINGS, "the waves' results lie where the rings were");
};

template <int D>
__device__ __forceinline__ int k_tile_off(int row, int c) {   // byte of 16-byte chunk c of a row of a K tile: chunks exchanged by the row, so that reads hit all banks
  constexpr int RB = 2 * D;
  return row * RB + ((c ^ ((row / (256 / RB)) % (RB / 16))) << 4);
}
template <int D>
__device__ __forceinline__ int v_tile_off(int row, int c) {   // the same of a V tile, whose transposing reads take four rows: pairs of chunks are exchanged
  const int slot = (c >> 1) ^ (D == 128 ? (row & 3) << 1 : row & 2);
  return row * 2 * D + (slot << 5) + ((c & 1) << 4);
}

// true: done; false: the item needs the other way (nothing has been written)
template <int D, bool F8, bool OUT_F32, int WAVES, typename P>
__device__ __forceinline__ bool tile_rows(const P& p, const Item& w, int slot_row, char* lds) {
  typedef Tile<D, WAVES> T;
  constexpr int RB = T::RB, BN = T::BN, NS = T::NS, TILE_BYTES = T::TILE_BYTES, KS = D / 16, DB = D / 32, CPR = D / 8, SUB = 32, NSW = BN / SUB;
  constexpr int RPI = 1024 / RB, IPW = 2, SHARE = IPW * RPI;   // rows of a wave-wide 16-byte load; loads of a wave, tile and tensor; its rows
  static_assert(BN / SHARE == WAVES, "the waves load a tile");
  // Tiles are sent in pairs, K of tile a and V of tile a - BEHIND.  Where a tile is a single sub-tile, K is read a tile earlier, and sent a tile earlier too (bf16, whose loads are on their way for a tile).
  constexpr int BEHIND = NSW == 1 && !F8 ? 2 : 1;
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, ql = lane & 31, hf = lane >> 5;
  const int row0 = w.tile * T::ROWS, n_rows = min(T::ROWS, w.q.n * p.gq - row0), qw0 = wave * 32;   // (rows counted within the item)
  const int limit_first = first_limit(p, w.q, row0), end = min(w.k1, last_limit(p, w.q, row0 + n_rows - 1));
  const int n_keys = end - w.k0, n_tiles = uniform((max(n_keys, 0) + BN - 1) / BN), last_tile = n_tiles - 1;

  if (tid == 0) *reinterpret_cast<int*>(lds + T::FLAG) = 0;

  // ---- tiles on their way: page and slot of this wave's share of a tile, in scalar registers
  const char* const kb = p.k_pages + (int64_t)w.hk * p.head_b;
  const char* const vb = p.v_pages + (int64_t)w.hk * p.head_b;
  typedef const int __attribute__((address_space(4)))* const_ptr;
  const const_ptr table = (const_ptr)(uintptr_t)(p.seq.table + (int64_t)w.b * p.seq.table_stride);
  const int share0 = w.k0 + wave * SHARE;   // first key of this wave's share of tile 0
  struct Place { int page, slot; };
  // Tiles up to the last one; there a share behind the end takes the last keys' place.  In the place of a page that is none the last one is read, and the
  // result is not kept (below).
  const unsigned last_page = p.seq.n_pages - 1;
  auto place_of = [&](int t) __attribute__((always_inline)) -> Place {
    int key = (share0 + t * BN) & ~15;
    key = min(key, (end - 1) & ~15);
    const int i = divide(p.seq.by_page, uniform(key));
    return Place{(int)min((unsigned)table[i], last_page), key - i * p.seq.page_size};
  };
  auto last_slot = [&](int row) __attribute__((always_inline)) -> int {   // of a row of the last tile in its group
    const int first = (share0 + last_tile * BN) & ~15, group = min(first, (end - 1) & ~15);
    return min(w.k0 + last_tile * BN + row, end - 1) - group;
  };
  const unsigned lds_base = (unsigned)(unsigned long)(lds_ptr_t)lds;
  // Byte offsets of the lane's loads from its group of 16 keys.  In the last tile rows behind the end take the last key's place; what that changes is counted
  // anew there, to be held in no register (at D 128 there is none left), like a lane's place in e4m3 tiles: 16 values of a row, whose slot is also its scale's.
  constexpr int L8 = D / 16;
  typedef const unsigned char __attribute__((address_space(1)))* global_bytes;
  typedef const u32x4 __attribute__((address_space(1)))* global_u32x4;
  unsigned k_off[IPW], v_off[IPW];
  auto lane_anew = [&]() __attribute__((always_inline)) -> int {
    unsigned zero = 0;
    asm volatile("" : "+v"(zero));
    return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
  };
  auto offset = [&](int i, bool v, bool last) __attribute__((always_inline)) -> unsigned {
    const int l = last ? lane_anew() : lane;
    const int row = wave * SHARE + i * RPI + l / CPR, pc = l % CPR;
    const int swz = D == 128 ? (row & 3) << 1 : row & 2, c = v ? (((pc >> 1) ^ swz) << 1) | (pc & 1) : pc ^ ((row / (256 / RB)) % CPR);
    return (last ? last_slot(row) : row & 15) * p.slot_b + c * 16;
  };
#pragma unroll
  for (int i = 0; i < IPW; i++) {
    k_off[i] = offset(i, false, false);
    v_off[i] = offset(i, true, false);
  }
  // (inline asm, and what follows for m0 and for the waits: see the block attention kernel's staging)
  auto dma16 = [&](const char* base, unsigned off, unsigned lds_off) __attribute__((always_inline)) {
    const unsigned m0v = __builtin_amdgcn_readfirstlane(lds_base + lds_off);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(m0v), "v"(off), "s"(base) : "memory");
  };
  auto uniform_at = [&](const auto* base, int64_t off) __attribute__((always_inline)) {
    const uint64_t x = (uint64_t)(base + off);
    return (decltype(base))(((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((unsigned)(x >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((unsigned)x));
  };
  // Tiles go out in pairs, K of tile a and V of tile a - BEHIND (one that is not there is left out): the place of V's tile is one that K's had.
  const int edge_tile = min(limit_first >= end ? n_tiles : max(0, limit_first - w.k0) / BN, n_keys % BN ? last_tile : n_tiles);   // from here on tiles hold keys that some rows do not see
  unsigned bad = 0;
  auto look = [&](u32x4 x) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; i++) bad |= not_finite(x[i]);
  };
  struct Raw { u32x4 x; unsigned scale; };   // e4m3: 16 values of a row
  auto load8 = [&](const char* base, const unsigned char* scales, Place at, bool last, int l, Raw& r) __attribute__((always_inline)) {
    const int row = wave * SHARE + l / L8, slot = last ? last_slot(row) : row & 15;
    const char* const src = uniform_at(base, (int64_t)at.page * p.page_b + (int64_t)at.slot * p.slot_b);
    const unsigned char* const s = uniform_at(scales, (int64_t)w.hk * p.scale_sh + (int64_t)at.page * p.scale_sp + at.slot);
    // (global memory's, which the compiler cannot see: flat loads wait for each other, and for LDS)
    r.x = *(global_u32x4)((global_bytes)(uintptr_t)src + (unsigned)(slot * p.slot_b + l % L8 * 16));
    r.scale = ((global_bytes)(uintptr_t)s)[(unsigned)slot];
  };
  auto put8 = [&](const Raw& r, int tile, int l, auto is_v_c, bool edge) __attribute__((always_inline)) {
    constexpr bool V = decltype(is_v_c)::value != 0;
    const u32x4 lo = {f8_pair(r.x[0], false, r.scale), f8_pair(r.x[0], true, r.scale), f8_pair(r.x[1], false, r.scale), f8_pair(r.x[1], true, r.scale)};
    const u32x4 hi = {f8_pair(r.x[2], false, r.scale), f8_pair(r.x[2], true, r.scale), f8_pair(r.x[3], false, r.scale), f8_pair(r.x[3], true, r.scale)};
    const int row = wave * SHARE + l / L8, to = V ? v_tile_off<D>(row, l % L8 * 2) : k_tile_off<D>(row, l % L8 * 2);
    *reinterpret_cast<u32x4*>(lds + tile + to) = lo;
    *reinterpret_cast<u32x4*>(lds + tile + (to ^ 16)) = hi;   // the chunk beside it, in either order
    if (V && edge) {
      look(lo);
      look(hi);
    }
  };
  auto send = [&](const char* base, Place at, bool last, const unsigned (&off)[IPW], bool v, int lds_off) __attribute__((always_inline)) {
    const char* const src = uniform_at(base, (int64_t)at.page * p.page_b + (int64_t)at.slot * p.slot_b);
    if (last) {
#pragma unroll
      for (int i = 0; i < IPW; i++) dma16(src, offset(i, v, true), lds_off + (wave * IPW + i) * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < IPW; i++) dma16(src, off[i], lds_off + (wave * IPW + i) * 1024);
    }
  };
  // bf16: pl_k is the place of tile a, pl_v of tile a - BEHIND, pl_n of the one between.  e4m3, whose values are a pair ahead in registers: of a + 1 and a.
  int a = 0;
  Place pl_k = {0, 0}, pl_v = {0, 0}, pl_n = {0, 0};
  Raw k_raw = {{0, 0, 0, 0}, 127}, v_raw = {{0, 0, 0, 0}, 127};
  auto pair = [&](int k_slot, int v_slot, auto inner_c) __attribute__((always_inline)) {
    constexpr bool INNER = decltype(inner_c)::value != 0;   // both tiles lie in front of the last, and the two behind them
    if constexpr (F8) {
      const int l = lane_anew();
      if (INNER || a <= last_tile) put8(k_raw, k_slot * TILE_BYTES, l, IC<0>{}, false);
      if (INNER || (a >= 1 && a - 1 <= last_tile)) put8(v_raw, (NS + v_slot) * TILE_BYTES, l, IC<1>{}, !INNER && a - 1 >= edge_tile);
      if (INNER || a + 1 <= last_tile) load8(kb, p.k_scales, pl_k, !INNER && a + 1 == last_tile, l, k_raw);
      if (INNER || a <= last_tile) load8(vb, p.v_scales, pl_v, !INNER && a == last_tile, l, v_raw);
      pl_v = pl_k;
      if (INNER || a + 2 <= last_tile) pl_k = place_of(a + 2);
    } else {
      if (INNER || a <= last_tile) send(kb, pl_k, !INNER && a == last_tile, k_off, false, k_slot * TILE_BYTES);
      if (INNER || (a >= 1 && a - BEHIND <= last_tile)) send(vb, pl_v, !INNER && a - BEHIND == last_tile, v_off, true, (NS + v_slot) * TILE_BYTES);
      if constexpr (BEHIND == 2) {
        pl_v = pl_n;
        pl_n = pl_k;
      } else {
        pl_v = pl_k;
      }
      if (INNER || a + 1 <= last_tile) pl_k = place_of(a + 1);
    }
    a++;
  };

  // ---- prologue: K_0 .. K_2, V_0, V_1 into the rings, the wave's Query rows into registers
  if (n_tiles > 0) {
    if constexpr (F8) {
      const int n = n_tiles;
      const Place p0 = place_of(0), p1 = place_of(min(1, last_tile)), p2 = place_of(min(2, last_tile)), p3 = place_of(min(3, last_tile));
      Raw k0, k1, k2, v0, v1;
      load8(kb, p.k_scales, p0, n == 1, lane, k0);
      load8(kb, p.k_scales, p1, n <= 2, lane, k1);   // (tiles behind the last one: the last one once more, never read)
      load8(vb, p.v_scales, p0, n == 1, lane, v0);
      load8(kb, p.k_scales, p2, n <= 3, lane, k2);
      load8(vb, p.v_scales, p1, n <= 2, lane, v1);
      if (n > 3) load8(kb, p.k_scales, p3, n == 4, lane, k_raw);
      if (n > 2) load8(vb, p.v_scales, p2, n == 3, lane, v_raw);
      put8(k0, 0, lane, IC<0>{}, false);
      put8(v0, NS * TILE_BYTES, lane, IC<1>{}, edge_tile <= 0);
      put8(k1, TILE_BYTES, lane, IC<0>{}, false);
      put8(k2, 2 * TILE_BYTES, lane, IC<0>{}, false);
      put8(v1, (NS + 1) * TILE_BYTES, lane, IC<1>{}, n > 1 && edge_tile <= 1);
      a = 3;
      pl_v = p3;
      if (n > 4) pl_k = place_of(4);
    } else {
      // (all places at once: each is a load that the next would wait behind)
      const Place p0 = place_of(0), p1 = place_of(min(1, last_tile)), p2 = place_of(min(2, last_tile)), p3 = place_of(min(3, last_tile));
      send(kb, p0, last_tile == 0, k_off, false, 0);
      send(vb, p0, last_tile == 0, v_off, true, NS * TILE_BYTES);
      if (last_tile >= 1) send(kb, p1, last_tile == 1, k_off, false, TILE_BYTES);
      if (last_tile >= 2) send(kb, p2, last_tile == 2, k_off, false, 2 * TILE_BYTES);
      if (last_tile >= 1) send(vb, p1, last_tile == 1, v_off, true, (NS + 1) * TILE_BYTES);
      a = 3;
      pl_k = p3;
      pl_v = p2;
      if constexpr (BEHIND == 2) {
        if (last_tile >= 3) send(kb, p3, last_tile == 3, k_off, false, 3 * TILE_BYTES);
        a = 4;
        pl_n = p3;
        if (last_tile >= 4) pl_k = place_of(4);
      }
    }
  }
  const int qrow = row0 + min(qw0 + ql, n_rows - 1), q_tok = divide(p.by_gq, qrow);
  bf16x8 qf[KS];   // lane (q, hf): Q[q][16 ks + 8 hf ..]
  {
    const __bf16* const qp = p.q + (int64_t)(w.hk * p.gq + qrow - q_tok * p.gq) * p.q_sh + (int64_t)(w.q.start + q_tok) * p.q_ss + 8 * hf;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + 16 * ks);
  }
  // pages that are none, among all of the item's keys
  for (int key = w.k0 + tid * 16; key < end; key += WAVES * 64 * 16) bad |= slot_of(p.seq, w.b, key).page < 0 ? 1u : 0u;
  // keys that the lane's row, and the first and the last row of the wave, see (in keys from k0 on)
  int lane_end = 0;
  if constexpr (is_tree<P>) *reinterpret_cast<int64_t*>(lds + T::OFF + (qw0 + ql) * 8) = (int64_t)(w.q.start + q_tok) * p.tree_stride;   // (the row's bits; both halves write it)
  else lane_end = min(w.k1, visible(w.q, q_tok, p.causal)) - w.k0;
  const bool rows_here = qw0 < n_rows;
  const int wave_lo = uniform(min(w.k1, first_limit(p, w.q, row0 + min(qw0, n_rows - 1))) - w.k0);
  const int wave_hi = uniform(rows_here ? min(w.k1, last_limit(p, w.q, row0 + min(qw0 + 31, n_rows - 1))) - w.k0 : 0);
  const int jw = (max(wave_hi, 0) + SUB - 1) / SUB;      // sub-tiles this wave has visible keys in
  const int kmask_from = wave_lo - SUB;                  // a sub-tile from kstart on needs a mask iff kstart > kmask_from
  const int jw_first = jw, jw_in = min(jw, NSW * n_tiles - 1);

  unsigned k_rd[KS], v_rd[DB];   // LDS addresses of the lane's operands (see the block attention kernel)
#pragma unroll
  for (int ks = 0; ks < KS; ks++) k_rd[ks] = lds_base + k_tile_off<D>(ql, 2 * ks + hf);
  {
    const int i16 = lane & 15, g2 = (lane >> 4) & 1, row = 4 * hf + (i16 >> 2);
#pragma unroll
    for (int db = 0; db < DB; db++) v_rd[db] = lds_base + NS * TILE_BYTES + v_tile_off<D>(row, 4 * db + 2 * g2) + (i16 & 3) * 8;
  }
  f32x16 o_acc[DB];
#pragma unroll
  for (int db = 0; db < DB; db++)
#pragma unroll
    for (int i = 0; i < 16; i++) o_acc[db][i] = 0.f;
  float m_ref = -INFINITY, mc = -INFINITY, l_run = 0.f;   // as in few_rows
  const float c2 = p.scale * kLog2e;

  // One step, as in the block attention kernel: S_{j+1} = K_{j+1} Q^T and O += V_{j-1}^T P_{j-1}^T beside the weights of sub-tile j, in the order
  // in which it is to issue.
  constexpr int NPV = 2 * DB, NQK = KS;
  typedef const s16x4 __attribute__((address_space(3)))* lds_tr_ptr;
  typedef const bf16x8 __attribute__((address_space(3)))* lds_b128_ptr;
  auto load_k = [&](int ks, unsigned imm) __attribute__((always_inline)) -> bf16x8 { return *(lds_b128_ptr)(unsigned long)(k_rd[ks] + imm); };
  auto load_v = [&](int i, unsigned imm) __attribute__((always_inline)) -> bf16x8 {
    const unsigned at = v_rd[i % DB] + imm + 16 * (i / DB) * RB;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(lds_tr_ptr)(unsigned long)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(lds_tr_ptr)(unsigned long)(at + 8 * RB));
    return __builtin_shufflevector(__builtin_bit_cast(bf16x4, lo), __builtin_bit_cast(bf16x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  bf16x8 pre[NQK];
  auto step = [&](int kstart, auto first_c, auto v_imm_c, auto k_imm_next_c, f32x16& s_in, f32x16& s_out, bf16x8 (&p_in)[2], bf16x8 (&p_out)[2],
                  auto inner_c) __attribute__((always_inline)) {
    constexpr bool FIRST = decltype(first_c)::value != 0, INNER = decltype(inner_c)::value != 0;
    constexpr int n_mfma = FIRST ? NQK : NQK + NPV, EPM = 16 / n_mfma;
    constexpr unsigned v_imm = decltype(v_imm_c)::value, k_imm_next = decltype(k_imm_next_c)::value;
    if (!INNER && kstart > kmask_from) {
      if constexpr (is_tree<P>) {
        const int64_t row = *reinterpret_cast<const int64_t*>(lds + T::OFF + (qw0 + ql) * 8);
        const unsigned seen = tree_bits(p.tree + row, p.words, w.q, w.k0 + kstart, end) >> 4 * hf;
#pragma unroll
        for (int i = 0; i < 16; i++)
          if (!(seen >> (8 * (i >> 2) + (i & 3)) & 1)) s_in[i] = -INFINITY;
      } else {
#pragma unroll
        for (int i = 0; i < 16; i++)
          if (kstart + 8 * (i >> 2) + 4 * hf + (i & 3) >= lane_end) s_in[i] = -INFINITY;
      }
    }
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; i++) acc[i] = 0.f;
    bf16x8 pv_ops[NPV], nxt[NQK];
    float tq[16], ex[16], ps0 = 0.f, ps1 = 0.f;
    unsigned pw[8];
    auto stage_a = [&](int g) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < EPM; k++) tq[g * EPM + k] = __builtin_fmaf(s_in[g * EPM + k], c2, -mc);
    };
    auto stage_b = [&](int g) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < EPM; k++) ex[g * EPM + k] = __builtin_amdgcn_exp2f(tq[g * EPM + k]);
    };
    auto stage_c = [&](int g) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < EPM; k++) {
        const int e = g * EPM + k;
        if (e & 1) {
          ps1 += ex[e];
          // (bf16 is what the second product takes: a weight is off by up to 2^-8 of itself, its sum and the results are held in 32 bits)
          asm volatile("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(pw[e >> 1]) : "v"(ex[e - 1]), "v"(ex[e]));
        } else {
          ps0 += ex[e];
        }
      }
    };
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < n_mfma; i++) {
      if (i < NQK) {
        if (FIRST) nxt[i] = load_k(i, k_imm_next);
        else pv_ops[i] = load_v(i, v_imm);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pre[i], qf[i], acc, 0, 0, 0);
      } else {
        const int j = i - NQK;
        nxt[j] = load_k(j, k_imm_next);
        o_acc[j % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pv_ops[j], p_in[j / DB], o_acc[j % DB], 0, 0, 0);
      }
      if (i == 0) {
        __builtin_amdgcn_sched_barrier(0);
        stage_a(0);
        stage_b(0);
        stage_a(1);
      }
      if (i + 1 < n_mfma) stage_b(i + 1);
      if (i + 2 < n_mfma) stage_a(i + 2);
      stage_c(i);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int h = 0; h < 2; h++) p_out[h] = __builtin_bit_cast(bf16x8, u32x4{pw[4 * h], pw[4 * h + 1], pw[4 * h + 2], pw[4 * h + 3]});
    float psum = ps0 + ps1;
    if (__builtin_expect(__any(!(psum <= kSumCap)), 0)) {
      float top = s_in[0];
#pragma unroll
      for (int i = 1; i < 16; i++) top = fmaxf(top, s_in[i]);
      top = halves_max(top);
      const float m_new = fmaxf(m_ref, top);
      const float f = m_new == m_ref ? 1.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c2);
      l_run *= f;
#pragma unroll
      for (int db = 0; db < DB; db++)
#pragma unroll
        for (int i = 0; i < 16; i++) o_acc[db][i] *= f;
      m_ref = m_new;
      mc = m_ref * c2;
      const float mc2 = m_ref == -INFINITY ? 0.f : mc;
      float q0s = 0.f, q1s = 0.f;
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s_in[i], c2, -mc2)), y = __builtin_amdgcn_exp2f(__builtin_fmaf(s_in[i + 1], c2, -mc2));
        p_out[i >> 3][i & 7] = (__bf16)x;
        p_out[i >> 3][(i & 7) + 1] = (__bf16)y;
        q0s += x;
        q1s += y;
      }
      psum = q0s + q1s;
    }
    l_run += psum;
    s_out = acc;
#pragma unroll
    for (int i = 0; i < NQK; i++) pre[i] = nxt[i];
  };

  // bf16: the lane's 32 bytes of V of tile u, which have landed
  auto look_at = [&](int u, int slot) __attribute__((always_inline)) {
    if constexpr (!F8) {
      if (u >= edge_tile && u <= last_tile) {
#pragma unroll
        for (int i = 0; i < IPW; i++) look(*reinterpret_cast<const u32x4*>(lds + (NS + slot) * TILE_BYTES + (wave * IPW + i) * 1024 + lane * 16));
      }
    }
  };
#pragma unroll
  for (int ks = 0; ks < KS; ks++) asm volatile("" ::"v"(qf[ks]));
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
  look_at(0, 0);
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();   // B_0
  asm volatile("" ::: "memory");

  f32x16 sA, sB;
  bf16x8 pA[2], pB[2];
  constexpr unsigned SUBB = SUB * RB;
  auto tile_step = [&](int u, auto su_c, auto kt_c, auto inner_c) __attribute__((always_inline)) {
    constexpr int su = decltype(su_c)::value, kt = decltype(kt_c)::value, sp = (su + NS - 1) % NS;
    constexpr bool INNER = decltype(inner_c)::value != 0, even = (NSW * su + kt) % 2 == 0;
    constexpr unsigned v_imm = kt == 0 ? sp * TILE_BYTES + (NSW - 1) * SUBB : su * TILE_BYTES + (kt - 1) * SUBB;
    constexpr unsigned k_imm = (su + (kt + 2) / NSW) % NS * TILE_BYTES + (kt + 2) % NSW * SUBB;
    const int j = NSW * u + kt;
    if (INNER ? !is_tree<P> || rows_here : j <= (kt == 0 ? jw_first : jw_in)) {
      if (even) step(j * SUB, IC<0>{}, IC<(int)v_imm>{}, IC<(int)k_imm>{}, sA, sB, pB, pA, inner_c);
      else step(j * SUB, IC<0>{}, IC<(int)v_imm>{}, IC<(int)k_imm>{}, sB, sA, pA, pB, inner_c);
    }
  };
  if (n_tiles > 0) {
    if constexpr (BEHIND == 1) pair(3, 2, IC<0>{});
    if (jw > 0) {
#pragma unroll
      for (int i = 0; i < 16; i++) sA[i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ks++) sA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(load_k(ks, 0), qf[ks], sA, 0, 0, 0);
#pragma unroll
      for (int ks = 0; ks < KS; ks++) pre[ks] = load_k(ks, SUBB);
    }
    if constexpr (BEHIND == 2) {   // (K_4 goes where K_0 was: all waves have read it)
      __builtin_amdgcn_s_waitcnt(0xC07F);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      pair(0, 2, IC<0>{});
    }
    if (jw > 0) {
      constexpr unsigned k_imm0 = 2 % NSW * SUBB + 2 / NSW * TILE_BYTES;
      step(0, IC<1>{}, IC<0>{}, IC<(int)k_imm0>{}, sA, sB, pB, pA, IC<0>{});
      if constexpr (NSW > 1) tile_step(0, IC<0>{}, IC<1>{}, IC<0>{});
      if constexpr (NSW > 2) {
        tile_step(0, IC<0>{}, IC<2>{}, IC<0>{});
        tile_step(0, IC<0>{}, IC<3>{}, IC<0>{});
      }
    }
  }
  // Tile u = 1 .. n_tiles (the last index folds the last sub-tile's product in): pair u + 3 goes out behind barrier B_u, into the slots of K_{u-1} and V_{u-2};
  // K_{u+2} and V_{u+1}, the newest pair in front of B_u, may still be on their way there.  (BEHIND 2: K_{u+4} in the slot of K_u, and K_{u+3} may be on its way.)
  auto tile_body = [&](int u, auto su_c, auto inner_c) __attribute__((always_inline)) {
    constexpr int su = decltype(su_c)::value;
    constexpr bool INNER = decltype(inner_c)::value != 0;
    if constexpr (F8) {
      __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): this wave's part of the tiles has been written
    } else {
      constexpr int none = 0x0F70;
      if (INNER || u + 1 + BEHIND <= last_tile) __builtin_amdgcn_s_waitcnt(none | 2 * IPW);
      else __builtin_amdgcn_s_waitcnt(none);
      asm volatile("" ::: "memory");
      if (!INNER) look_at(u, su);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    pair((su + 2 + BEHIND) % NS, (su + 2) % NS, inner_c);
    tile_step(u, su_c, IC<0>{}, inner_c);
    if constexpr (NSW > 1) tile_step(u, su_c, IC<1>{}, inner_c);
    if constexpr (NSW > 2) {
      tile_step(u, su_c, IC<2>{}, inner_c);
      tile_step(u, su_c, IC<3>{}, inner_c);
    }
  };
  // Inner tiles: every step runs in this wave without a mask, and what they send lies in front of the last tile.  Waves may disagree about where they
  // end: both bodies hold the same barrier and the same number of loads.
  // A tree's few rows may leave waves without any.  Those too send inner tiles as inner ones, or all wait for them: loads that may be left out are waited for at once (16 trees of 100 rows in
  // 8 bits 78 -> 69 us).
  const int j_inner = is_tree<P> && !rows_here ? kPosLimit : min(min(jw, NSW * n_tiles - 1), kmask_from >= 0 ? kmask_from / SUB : -1) - (NSW - 1);
  const int u_inner = uniform(min(min(j_inner < 0 ? -1 : j_inner / NSW, last_tile - (F8 ? 6 : 4 + BEHIND)), edge_tile - 3));
  if (1 <= n_tiles) tile_body(1, IC<1>{}, IC<0>{});
  if (2 <= n_tiles) tile_body(2, IC<2>{}, IC<0>{});
  if (3 <= n_tiles) tile_body(3, IC<3>{}, IC<0>{});
  int u0 = NS;
  for (; u0 + NS - 1 <= u_inner; u0 += NS) {
    tile_body(u0, IC<0>{}, IC<1>{});
    tile_body(u0 + 1, IC<1>{}, IC<1>{});
    tile_body(u0 + 2, IC<2>{}, IC<1>{});
    tile_body(u0 + 3, IC<3>{}, IC<1>{});
  }
  for (; u0 <= n_tiles; u0 += NS) {
    tile_body(u0, IC<0>{}, IC<0>{});
    if (u0 + 1 <= n_tiles) tile_body(u0 + 1, IC<1>{}, IC<0>{});
    if (u0 + 2 <= n_tiles) tile_body(u0 + 2, IC<2>{}, IC<0>{});
    if (u0 + 3 <= n_tiles) tile_body(u0 + 3, IC<3>{}, IC<0>{});
  }
  if (__any(bad != 0) && lane == 0) *reinterpret_cast<int*>(lds + T::FLAG) = 1;
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();   // every wave is done with the rings and none of its loads is still landing
  if (*reinterpret_cast<volatile int*>(lds + T::FLAG)) return false;

  // ---- epilogue: each wave turns its 32 x D results over in LDS and stores whole rows
  {
  const int lane = lane_anew(), ql = lane & 31, hf = lane >> 5;   // (not held over the loop)
  const float l_tot = halves_sum(l_run), inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  const float lse = l_tot > 0.f ? m_ref * p.scale + logf(l_tot) : l_tot == 0.f ? -INFINITY : __builtin_nanf("");
  char* const my = lds + wave * (32 * 4 * D);
  int64_t* const my_off = reinterpret_cast<int64_t*>(lds + T::OFF) + wave * 32;   // where the wave's rows go, counted once a row
  if (hf == 0 && qw0 + ql < n_rows) {
    if (w.n_parts > 1) {
      my_off[ql] = (int64_t)(slot_row + qw0 + ql) * D;
      p.part_lse[slot_row + qw0 + ql] = lse;
    } else {
      const int r = row0 + qw0 + ql, t = divide(p.by_gq, r), head = w.hk * p.gq + r - t * p.gq;
      my_off[ql] = (int64_t)head * p.o_sh + (int64_t)(w.q.start + t) * p.o_ss;
      p.lse[(int64_t)head * p.l_sh + (int64_t)(w.q.start + t) * p.l_ss] = lse != lse ? -INFINITY : lse;
    }
  }
#pragma unroll
  for (int db = 0; db < DB; db++)
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const int c = 8 * db + 2 * g + hf;
      f32x4 o;
#pragma unroll
      for (int r = 0; r < 4; r++) o[r] = o_acc[db][4 * g + r] * inv;
      *reinterpret_cast<f32x4*>(my + ql * (4 * D) + ((c ^ (ql & 15)) << 4)) = o;
    }
  __builtin_amdgcn_s_waitcnt(0xC07F);
  constexpr int CPRF = D / 4, RPO = 64 / CPRF;
  const bool whole = w.n_parts == 1;
  float* const to_f32 = whole ? reinterpret_cast<float*>(p.out) : p.part_out;
#pragma unroll
  for (int it = 0; it < 32 / RPO; it++) {
    const int r = it * RPO + lane / CPRF, c = lane % CPRF;
    if (qw0 + r >= n_rows) continue;
    const f32x4 o = *reinterpret_cast<const f32x4*>(my + r * (4 * D) + ((c ^ (r & 15)) << 4));
    const int64_t to = my_off[r] + 4 * c;
    if (OUT_F32 || !whole) {
      *reinterpret_cast<f32x4*>(to_f32 + to) = o;
    } else {
      bf16x4 ob;
#pragma unroll
      for (int k = 0; k < 4; k++) ob[k] = (__bf16)o[k];
      *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(p.out) + to) = ob;
    }
  }
  }
  return true;
}

template <int D, bool F8, bool OUT_F32, int WAVES, typename P>
__device__ __forceinline__ void many_rows(const P& p, char* lds) {
  constexpr int ROWS = Tile<D, WAVES>::ROWS;
  Item w;
  if (!find_item(p, make_plan(p), (int)blockIdx.x, w)) return;
  const int row0 = w.tile * ROWS, slot_row = w.slot * ROWS, n = min(ROWS, w.rows - row0);
  if (tile_rows<D, F8, OUT_F32, WAVES>(p, w, slot_row, lds)) return;
#pragma unroll 1
  for (int r = 0; r < n; r += 16) {
    __syncthreads();
    few_rows<D, F8, 1, WAVES, false, OUT_F32>(p, w, row0 + r, slot_row + r, lds);
  }
}
template <int D, bool F8, bool OUT_F32, typename P>
__global__ void __launch_bounds__(512, 2) paged_many_kernel(const P p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  many_rows<D, F8, OUT_F32, 8>(p, lds);
}
// Trees alone: 128 rows, two workgroups a compute unit, so that one's set-up and epilogue run beside the other's products.  A tile at D 128 is one sub-tile of 32 keys: in bf16 K is sent a tile
// earlier for that (64 trees of 25 tokens, 8 heads of 128 for 32, 1000 keys: 50 us, in bf16, 47 in 8 bits; with 256 rows, of which 100 are there, 61 and 56).
template <int D, bool F8, bool OUT_F32, typename P>
__global__ void __launch_bounds__(256, 2) paged_half_kernel(const P p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  many_rows<D, F8, OUT_F32, 4>(p, lds);
}

}  // namespace
}  // namespace tr
