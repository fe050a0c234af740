// Writing new keys into the pages of a cache and reading them back as dense tensors.
#include "paged.h"

namespace tr {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

// Sequence of token t: the last one that starts at or before it (those without tokens start where the next one does), -1: none.
__device__ __forceinline__ int sequence_of(const Sequences& s, int t) {
  int lo = -1, hi = s.n;   // q_start[lo] <= t < q_start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.q_start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

// A wave has 16 tokens (write) or keys (read) of one head, of K or of V: lane i finds the place of the i-th, and rows are 16 bytes of bf16 a lane, D / 8 lanes
// each.  What a wave touches of a page lies together, its 16 scales too: single bytes from different compute units would be merged in memory.  All its rows are
// on their way at once.  Bound: HBM: 52K tokens on 8 heads of 128, bf16 to e4m3, 67.5 us, 4.75 TB/s (row by row with the heads side by side 152); 32K keys read back 30.3 us, 6.7 TB/s.
template <int D>
struct Rows {
  static constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, TURNS = 16 / AT_ONCE;   // lanes a row, rows at once
};
__device__ __forceinline__ int64_t from(int64_t x, int lane) {
  return (int64_t)(((uint64_t)(unsigned)__shfl((int)(x >> 32), lane) << 32) | (unsigned)__shfl((int)x, lane));
}
// The first of the 16 rows of this wave, its head, and whether it has V's.
struct WaveRows { int rows, head, is_v; };

template <int D, bool F8>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const CacheCopyParams p) {
  typedef Rows<D> R;
  const int lane = threadIdx.x & 63, c = lane % R::LANES;
  WaveRows w;
  {
    const int g = divide(p.by_heads, (int)blockIdx.x), other = (int)blockIdx.x - g * 2 * p.heads;
    w.rows = (g * (kThreads / 64) + (int)(threadIdx.x >> 6)) * 16;
    w.is_v = other >= p.heads;
    w.head = w.is_v ? other - p.heads : other;
  }
  if (w.rows >= p.seq.tokens) return;
  // the places of its tokens, -1: nowhere
  int64_t to = -1, scale_to = -1;
  {
    const int t = w.rows + (lane & 15), b = t < p.seq.tokens ? sequence_of(p.seq, t) : -1;
    if (b >= 0) {
      const Sequence q = sequence(p.seq, b);
      const int key = q.pos + (t - q.start);
      if (t >= q.start && t < q.start + q.n && key >= 0 && key < q.len) {
        const Slot at = slot_of(p.seq, b, key);
        if (at.page >= 0) {
          to = (int64_t)at.page * p.page_b + (int64_t)w.head * p.head_b + (int64_t)at.slot * p.slot_b;
          scale_to = (int64_t)at.page * p.scale_sp + (int64_t)w.head * p.scale_sh + at.slot;
        }
      }
    }
  }
  const char* const src = (w.is_v ? p.v : p.k) + 2 * (int64_t)w.head * p.d_sh + 16 * c;
  char* const pages = w.is_v ? p.v_pages : p.k_pages;
  u32x4 x[R::TURNS];
#pragma unroll
  for (int i = 0; i < R::TURNS; i++)
    x[i] = *reinterpret_cast<const u32x4*>(src + 2 * (int64_t)min(w.rows + i * R::AT_ONCE + lane / R::LANES, p.seq.tokens - 1) * p.d_ss);
  int scale_here = 127;
#pragma unroll
  for (int i = 0; i < R::TURNS; i++) {
    const int64_t off = from(to, i * R::AT_ONCE + lane / R::LANES);
    if constexpr (!F8) {
      if (off >= 0) *reinterpret_cast<u32x4*>(pages + off + 16 * c) = x[i];
    } else {
      float f[8], top = 0.f;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        f[2 * j] = __builtin_bit_cast(float, x[i][j] << 16);
        f[2 * j + 1] = __builtin_bit_cast(float, x[i][j] & 0xffff0000u);
      }
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float a = fabsf(f[j]);
        if (a < INFINITY) top = fmaxf(top, a);
        else f[j] = __builtin_nanf("");
      }
#pragma unroll
      for (int d = 1; d < R::LANES; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
      // top = 1.m * 2^e: top / 2^(e - 8) lies in [256, 512) and is at most 448 = 1.75 * 2^8 if 1.m is at most 1.75.
      const unsigned bits = __builtin_bit_cast(unsigned, top);
      const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
      const int scale = top == 0.f ? 127 : max(e, 1);
      const float inv = __builtin_bit_cast(float, (unsigned)(254 - scale) << 23);   // (scale is 247 at most)
      int y[2];
#pragma unroll
      for (int j = 0; j < 2; j++) {
        y[j] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j] * inv, f[4 * j + 1] * inv, 0, false);
        y[j] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2] * inv, f[4 * j + 3] * inv, y[j], true);
      }
      if (off >= 0) *reinterpret_cast<u32x2*>(pages + off + 8 * c) = u32x2{(unsigned)y[0], (unsigned)y[1]};
      const int mine = __shfl(scale, (lane & (R::AT_ONCE - 1)) * R::LANES);   // of row lane mod AT_ONCE of this turn
      if ((lane & 15) / R::AT_ONCE == i) scale_here = mine;
    }
  }
  if (F8 && lane < 16 && scale_to >= 0) (w.is_v ? p.v_scales : p.k_scales)[scale_to] = (unsigned char)scale_here;
}

template <int D, bool F8>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const CacheCopyParams p) {
  typedef Rows<D> R;
  const int lane = threadIdx.x & 63, c = lane % R::LANES;
  WaveRows w;
  w.rows = ((int)blockIdx.x * (kThreads / 64) + (int)(threadIdx.x >> 6)) * 16;   // a workgroup has 64 keys of a head, which lie together in the result
  if (w.rows >= p.rows) return;
  for (int64_t y = blockIdx.y; y < (int64_t)p.seq.n * 2 * p.heads; y += gridDim.y) {
    const int b = divide(p.by_heads, (int)y), other = (int)y - b * 2 * p.heads;
    w.is_v = other >= p.heads;
    w.head = w.is_v ? other - p.heads : other;
    int64_t at = -1;
    unsigned scale = 127;
    const int64_t key = p.first + w.rows + (lane & 15);
    if (w.rows + (lane & 15) < p.rows && key < clamped(p.seq.kv_len[b], 0, p.seq.max_pages * p.seq.page_size)) {
      const Slot x = slot_of(p.seq, b, (int)key);
      if (x.page >= 0) {
        at = (int64_t)x.page * p.page_b + (int64_t)w.head * p.head_b + (int64_t)x.slot * p.slot_b;
        if (F8) scale = (w.is_v ? p.v_scales : p.k_scales)[(int64_t)x.page * p.scale_sp + (int64_t)w.head * p.scale_sh + x.slot];
      }
    }
    const char* const pages = w.is_v ? p.v_pages : p.k_pages;
    u32x4 x[R::TURNS];
    int64_t off[R::TURNS];
#pragma unroll
    for (int i = 0; i < R::TURNS; i++) {
      off[i] = from(at, i * R::AT_ONCE + lane / R::LANES);
      if (off[i] < 0) continue;
      if constexpr (F8) {
        const u32x2 y = *reinterpret_cast<const u32x2*>(pages + off[i] + 8 * c);
        x[i][0] = y[0];
        x[i][1] = y[1];
      } else {
        x[i] = *reinterpret_cast<const u32x4*>(pages + off[i] + 16 * c);
      }
    }
    char* const dst = (w.is_v ? p.v_out : p.k_out) + 2 * ((int64_t)b * p.d_sb + (int64_t)w.head * p.d_sh + (int64_t)w.rows * p.d_ss) + 16 * c;
#pragma unroll
    for (int i = 0; i < R::TURNS; i++) {
      const int r = i * R::AT_ONCE + lane / R::LANES;
      const unsigned s = F8 ? __shfl(scale, r) : 0;
      if (off[i] < 0) continue;
      u32x4 y = x[i];
      if constexpr (F8) y = u32x4{f8_pair(x[i][0], false, s), f8_pair(x[i][0], true, s), f8_pair(x[i][1], false, s), f8_pair(x[i][1], true, s)};
      __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(dst + 2 * (int64_t)r * p.d_ss));
    }
  }
}

}  // namespace

hipError_t launch_cache_write(const CacheCopyParams& p, int D, bool f8, hipStream_t stream) {
  const int64_t groups = ((int64_t)p.seq.tokens + kThreads / 4 - 1) / (kThreads / 4) * 2 * p.heads;
  const dim3 grid((unsigned)groups), block(kThreads);
  if (D == 128) return f8 ? launch_kernel(cache_write_kernel<128, true>, grid, block, 0, stream, p) : launch_kernel(cache_write_kernel<128, false>, grid, block, 0, stream, p);
  return f8 ? launch_kernel(cache_write_kernel<64, true>, grid, block, 0, stream, p) : launch_kernel(cache_write_kernel<64, false>, grid, block, 0, stream, p);
}

hipError_t launch_cache_read(const CacheCopyParams& p, int D, bool f8, hipStream_t stream) {
  const int64_t heads = (int64_t)p.seq.n * 2 * p.heads;
  const dim3 grid((unsigned)((p.rows + kThreads / 4 - 1) / (kThreads / 4)), (unsigned)(heads < 65535 ? heads : 65535)), block(kThreads);
  if (D == 128) return f8 ? launch_kernel(cache_read_kernel<128, true>, grid, block, 0, stream, p) : launch_kernel(cache_read_kernel<128, false>, grid, block, 0, stream, p);
  return f8 ? launch_kernel(cache_read_kernel<64, true>, grid, block, 0, stream, p) : launch_kernel(cache_read_kernel<64, false>, grid, block, 0, stream, p);
}

}  // namespace tr
