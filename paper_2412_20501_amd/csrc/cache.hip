// Writing new keys into the pages of a cache and reading them back as dense tensors.
#include "paged.h"

namespace tr {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

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

// A row of D values is D / 8 lanes' work, 16 bytes each.  Bound: HBM.
template <int D, bool F8>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const CacheCopyParams p) {
  constexpr int LANES = D / 8;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES;
  const int c = threadIdx.x % LANES;
  const int tk = divide(p.by_heads, (int)row), h = (int)row - tk * p.heads, t = tk >> 1;   // rows: token, K or V, head
  const bool is_v = tk & 1;
  if (t >= p.seq.tokens) return;
  const int b = sequence_of(p.seq, t);
  if (b < 0) return;
  const Sequence q = sequence(p.seq, b);
  const int key = q.pos + (t - q.start);
  if (t < q.start || t >= q.start + q.n || key < 0 || key >= q.len) return;
  const Slot at = slot_of(p.seq, b, key);
  if (at.page < 0) return;
  const u32x4 x = *reinterpret_cast<const u32x4*>((is_v ? p.v : p.k) + 2 * ((int64_t)h * p.d_sh + (int64_t)t * p.d_ss) + 16 * c);
  char* const dst = (is_v ? p.v_pages : p.k_pages) + (int64_t)at.page * p.page_b + (int64_t)h * p.head_b + (int64_t)at.slot * p.slot_b;
  if constexpr (!F8) {
    *reinterpret_cast<u32x4*>(dst + 16 * c) = x;
  } else {
    float f[8], top = 0.f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      f[2 * i] = __builtin_bit_cast(float, x[i] << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, x[i] & 0xffff0000u);
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float a = fabsf(f[i]);
      if (a < INFINITY) top = fmaxf(top, a);
      else f[i] = __builtin_nanf("");
    }
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    // top = 1.m * 2^e: top / 2^(e - 8) lies in [256, 512) and is at most 448 = 1.75 * 2^8 if m is at most 0.75.
    const unsigned bits = __builtin_bit_cast(unsigned, top);
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    const int scale = top == 0.f ? 127 : max(e, 1);
    const float inv = __builtin_bit_cast(float, (unsigned)(254 - scale) << 23);   // (scale is 247 at most)
    int w[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i] * inv, f[4 * i + 1] * inv, 0, false);
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2] * inv, f[4 * i + 3] * inv, w[i], true);
    }
    *reinterpret_cast<u32x2*>(dst + 8 * c) = u32x2{(unsigned)w[0], (unsigned)w[1]};
    if (c == 0) (is_v ? p.v_scales : p.k_scales)[(int64_t)at.page * p.scale_sp + (int64_t)h * p.scale_sh + at.slot] = (unsigned char)scale;
  }
}

template <int D, bool F8>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const CacheCopyParams p) {
  constexpr int LANES = D / 8;
  const int s = (int)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES, c = threadIdx.x % LANES;
  const bool is_v = blockIdx.z;
  if (s >= p.rows) return;
  for (int bh = blockIdx.y; bh < p.seq.n * p.heads; bh += gridDim.y) {
    const int b = divide(p.by_heads, bh), h = bh - b * p.heads;
    const int64_t key = p.first + s;
    if (key >= clamped(p.seq.kv_len[b], 0, p.seq.max_pages * p.seq.page_size)) continue;
    const Slot at = slot_of(p.seq, b, (int)key);
    if (at.page < 0) continue;
    const char* const src = (is_v ? p.v_pages : p.k_pages) + (int64_t)at.page * p.page_b + (int64_t)h * p.head_b + (int64_t)at.slot * p.slot_b;
    u32x4 x;
    if constexpr (!F8) {
      x = *reinterpret_cast<const u32x4*>(src + 16 * c);
    } else {
      const u32x2 y = *reinterpret_cast<const u32x2*>(src + 8 * c);
      const unsigned scale = (is_v ? p.v_scales : p.k_scales)[(int64_t)at.page * p.scale_sp + (int64_t)h * p.scale_sh + at.slot];
#pragma unroll
      for (int i = 0; i < 4; i++) x[i] = f8_pair(y[i >> 1], i & 1, scale);
    }
    *reinterpret_cast<u32x4*>((is_v ? p.v_out : p.k_out) + 2 * ((int64_t)b * p.d_sb + (int64_t)h * p.d_sh + (int64_t)s * p.d_ss) + 16 * c) = x;
  }
}

}  // namespace

hipError_t launch_cache_write(const CacheCopyParams& p, int D, bool f8, hipStream_t stream) {
  const int64_t rows = (int64_t)p.seq.tokens * 2 * p.heads;
  const dim3 grid((unsigned)((rows + kThreads * 8 / D - 1) / (kThreads * 8 / D)));
  if (D == 128) return f8 ? launch_kernel(cache_write_kernel<128, true>, grid, dim3(kThreads), 0, stream, p) : launch_kernel(cache_write_kernel<128, false>, grid, dim3(kThreads), 0, stream, p);
  return f8 ? launch_kernel(cache_write_kernel<64, true>, grid, dim3(kThreads), 0, stream, p) : launch_kernel(cache_write_kernel<64, false>, grid, dim3(kThreads), 0, stream, p);
}

hipError_t launch_cache_read(const CacheCopyParams& p, int D, bool f8, hipStream_t stream) {
  const int64_t heads = (int64_t)p.seq.n * p.heads;
  const dim3 grid((unsigned)((p.rows + kThreads * 8 / D - 1) / (kThreads * 8 / D)), (unsigned)(heads < 65535 ? heads : 65535), 2);
  if (D == 128) return f8 ? launch_kernel(cache_read_kernel<128, true>, grid, dim3(kThreads), 0, stream, p) : launch_kernel(cache_read_kernel<128, false>, grid, dim3(kThreads), 0, stream, p);
  return f8 ? launch_kernel(cache_read_kernel<64, true>, grid, dim3(kThreads), 0, stream, p) : launch_kernel(cache_read_kernel<64, false>, grid, dim3(kThreads), 0, stream, p);
}

}  // namespace tr
