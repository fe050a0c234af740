// Internal declarations of the operators that choose and move the keys of a paged cache.
#pragma once
#include "paged_plan.h"
#include "tr_internal.h"

namespace tr {

// Arguments of the kernels that weigh keys.
struct WeighParams {
  Sequences seq;
  const __bf16* q;
  const float* lse;
  const char* k_pages;
  const unsigned char* k_scales;
  float* weights;
  int64_t q_sh, q_ss, l_sh, l_ss;
  int64_t page_b, head_b;      // bytes
  int slot_b;                  // bytes, at most 2^25
  int64_t scale_sp, scale_sh, w_sp, w_sh;
  int Hkv, gq;
  Divisor by_gq;
  int causal, fresh;
  float scale;
};
hipError_t launch_cache_weigh(const WeighParams& p, int D, bool f8, hipStream_t stream);

struct SelectParams {
  Sequences seq;
  const float* weights;
  int64_t w_sp, w_sh;
  int heads, first, last, most;   // most: keys that stay, at most
  int* keys;
  int* count;
  int64_t k_sb, k_sh;             // of keys
};
hipError_t launch_cache_select(const SelectParams& p, hipStream_t stream);

struct KeepParams {
  Sequences seq;
  char* k_pages;
  char* v_pages;
  unsigned char* k_scales;   // or null
  unsigned char* v_scales;
  float* weights;            // or null
  int64_t page_b, head_b, slot_b;   // bytes
  int64_t scale_sp, scale_sh, w_sp, w_sh;
  int heads, row_bytes, most;
  const int* keys;
  const int* count;
  const int* start;          // or null
  int64_t k_sb, k_sh;        // of keys
};
hipError_t launch_cache_keep(const KeepParams& p, hipStream_t stream);

}  // namespace tr
