// Internal declarations of the operators on a paged cache.
#pragma once
#include "paged_plan.h"
#include "tr_internal.h"

namespace tr {

// Arguments of the kernels that copy between dense tensors and pages.
struct CacheCopyParams {
  Sequences seq;
  const char* k;   // new tokens, bf16
  const char* v;
  char* k_out;     // dense result, bf16
  char* v_out;
  char* k_pages;
  char* v_pages;
  unsigned char* k_scales;
  unsigned char* v_scales;
  int64_t d_sb, d_sh, d_ss;         // of the dense tensors, in elements
  int64_t page_b, head_b, slot_b;   // of the pages, in bytes
  int64_t scale_sp, scale_sh;
  int heads;        // K/V heads
  Divisor by_heads;   // of 2 * heads
  int rows;         // read: rows of a sequence's result
  int64_t first;    // read: key of row 0
};
hipError_t launch_cache_write(const CacheCopyParams& p, int D, bool f8, hipStream_t stream);
hipError_t launch_cache_read(const CacheCopyParams& p, int D, bool f8, hipStream_t stream);

// Arguments of the attention kernel on pages and of its fold.
struct PagedParams {
  Sequences seq;
  const __bf16* q;
  void* out;     // bf16 or fp32
  float* lse;
  const char* k_pages;
  const char* v_pages;
  const unsigned char* k_scales;
  const unsigned char* v_scales;
  int64_t q_sh, q_ss, o_sh, o_ss, l_sh, l_ss;
  int64_t page_b, head_b;   // bytes
  int slot_b;               // bytes, at most 2^25
  int64_t scale_sp, scale_sh;
  int Hkv, gq;
  Divisor by_gq;
  int causal, out_f32;
  float scale;
  RowClass rows;   // of the launch
  Share share;     // of the keys among workgroups
  int slots;       // of the scratch
  float* part_out; // [slots][rows of a tile][D]
  float* part_lse; // [slots][rows of a tile]
};

// The same where new tokens see those of the others that their bits say.
struct TreeParams : PagedParams {
  const unsigned* tree;    // [tokens][words], rows tree_stride apart
  int64_t tree_stride;
  int words;
};

// p without what belongs to a launch (rows, share, scratch); workspace: null or the floats of all parts
hipError_t launch_paged_attn(PagedParams& p, const PagedLaunch& l, int D, bool f8, float* workspace, hipStream_t stream);
hipError_t launch_paged_attn(TreeParams& p, const PagedLaunch& l, int D, bool f8, float* workspace, hipStream_t stream);

#if defined(__HIPCC__)
// Two e4m3 values (the upper ones of x, if upper) times 2^(scale - 127), as two bf16: the conversion takes the scale as the exponent of a float.  It reads 0 as
// 2^-127 and 255 as NaN, like the type (all 65536 pairs of a code and a scale are tested).
__device__ __forceinline__ unsigned f8_pair(unsigned x, bool upper, unsigned scale) {
  const float s = __builtin_bit_cast(float, scale << 23);
  return __builtin_bit_cast(unsigned, upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, false));
}
#endif

}  // namespace tr
