// Argument checks shared by the entry points on a paged cache (host code).
#pragma once
#include <string.h>

#include "checks.h"
#include "paged.h"

namespace tr {
namespace {

constexpr int64_t kMaxKeys = (int64_t)1 << 30;
// Sequences of an attention call.  Its workgroups each go through all of them, 64 at a time in about half a microsecond, so that the time for it grows with their square: tokens of as many sequences with
// 200 keys, on 8 K/V heads, 50 us for 256, 0.37 ms for 1024 (twice what the keys take), 3.6 for 4096, 53 for 16384.
constexpr int64_t kMaxAttended = (int64_t)1 << 16;
constexpr int64_t kMaxGroups = (int64_t)1 << 24;   // workgroups of 256 threads of a grid's dimension, which holds fewer than 2^32 threads

// A descriptor without the strides of dimensions of one element, which say nothing; null stays null.
struct View {
  tr_tensor t;
  const tr_tensor* at;
  explicit View(const tr_tensor* from) : at(from ? &t : nullptr) {
    if (!from) return;
    t = *from;
    if (t.B <= 1 && t.stride_b > 0) t.stride_b = 0;
    if (t.H <= 1 && t.stride_h > 0) t.stride_h = 0;
    if (t.S <= 1 && t.stride_s > 0) t.stride_s = 0;
  }
};

bool same_layout(const tr_tensor* a, const tr_tensor* b) {
  return a->dtype == b->dtype && a->B == b->B && a->H == b->H && a->S == b->S && a->D == b->D && a->stride_b == b->stride_b &&
         a->stride_h == b->stride_h && a->stride_s == b->stride_s;
}

// Whether two views of one shape and the same strides certainly share no element: apart as a whole, or side by side inside the step of one
// dimension (K and V as the two halves of each page, or of each row) that the steps of the dimensions outside it are multiples of.
bool apart(const tr_tensor* a, const tr_tensor* b) {
  if (!overlaps(a, b)) return true;
  const int64_t eb = elem_bytes(a->dtype), bytes = a->ptr > b->ptr ? (char*)a->ptr - (char*)b->ptr : (char*)b->ptr - (char*)a->ptr;
  if (bytes % eb) return false;
  const int64_t off = bytes / eb;
  int64_t size[3] = {a->B, a->H, a->S}, stride[3] = {a->stride_b, a->stride_h, a->stride_s};
  for (int i = 0; i < 3; i++)
    for (int j = i + 1; j < 3; j++)
      if (size[i] <= 1 ? size[j] > 1 : (size[j] > 1 && stride[j] > stride[i])) {   // from the outside in, dimensions of one element last
        const int64_t x = size[i], y = stride[i];
        size[i] = size[j]; stride[i] = stride[j];
        size[j] = x; stride[j] = y;
      }
  for (int i = 0; i < 3 && size[i] > 1; i++) {
    int64_t inner = a->D;
    for (int j = i + 1; j < 3; j++) inner += size[j] > 1 ? (size[j] - 1) * stride[j] : 0;
    const int64_t at = off % stride[i];
    if (at >= inner && at + inner <= stride[i]) return true;
    if (i + 1 < 3 && size[i + 1] > 1 && stride[i] % stride[i + 1]) return false;
  }
  return false;
}

// The device arrays of a tr_sequences as tensors, for overlap tests.
struct SeqViews {
  tr_tensor t[8];
  int n = 0;
  void add(const int32_t* ptr, int64_t elems) {
    if (!ptr || elems <= 0) return;
    memset(&t[n], 0, sizeof(t[n]));
    t[n].ptr = const_cast<int32_t*>(ptr);
    t[n].dtype = TR_F32;
    t[n].B = t[n].H = t[n].S = 1;
    t[n++].D = elems;
  }
};

tr_status check_cache(const tr_tensor* kp, const tr_tensor* vp, const tr_tensor* ks, const tr_tensor* vs, bool written) {
  tr_status st;
  if ((st = check_typed("k_pages", kp, kBf16 | kF8, 16)) != TR_OK) return st;
  if ((st = check_typed("v_pages", vp, kBf16 | kF8, 16)) != TR_OK) return st;
  if (kp->dtype != vp->dtype) return fail(TR_ERR_DTYPE, "k_pages and v_pages must have one dtype");
  if (kp->B != vp->B || kp->H != vp->H || kp->S != vp->S || kp->D != vp->D) return fail(TR_ERR_SHAPE, "k_pages and v_pages shapes differ");
  if (!same_layout(kp, vp)) return fail(TR_ERR_STRIDE, "k_pages and v_pages must share their strides");
  if (kp->D != 64 && kp->D != 128) return fail(TR_ERR_SHAPE, "head dim %lld not supported (64 or 128)", (long long)kp->D);
  if (kp->H < 1) return fail(TR_ERR_SHAPE, "a cache needs a K/V head");
  if (kp->S < 16 || kp->S % 16) return fail(TR_ERR_SHAPE, "page size %lld is not a multiple of 16", (long long)kp->S);
  if (kp->stride_s > ((int64_t)1 << 24)) return fail(TR_ERR_STRIDE, "stride_s of k_pages and v_pages must not exceed 2^24 elements");
  if (written) {
    if ((st = check_written("k_pages", kp)) != TR_OK) return st;
    if (!apart(kp, vp)) return fail(TR_ERR_ALIAS, "k_pages and v_pages overlap");
  }
  if (kp->dtype == TR_BF16) {
    if (ks || vs) return fail(TR_ERR_DTYPE, "bf16 pages have no scales");
    return TR_OK;
  }
  if (!ks || !vs) return fail(TR_ERR_NULL, "e4m3 pages need k_scales and v_scales");
  if ((st = check_typed("k_scales", ks, kE8m0, 1)) != TR_OK) return st;
  if ((st = check_typed("v_scales", vs, kE8m0, 1)) != TR_OK) return st;
  if (ks->B != kp->B || ks->H != kp->H || ks->S != kp->S || ks->D != 1) return fail(TR_ERR_SHAPE, "k_scales shape does not match k_pages");
  if (vs->B != kp->B || vs->H != kp->H || vs->S != kp->S || vs->D != 1) return fail(TR_ERR_SHAPE, "v_scales shape does not match v_pages");
  if (!same_layout(ks, vs)) return fail(TR_ERR_STRIDE, "k_scales and v_scales must share their strides");
  if (ks->stride_s != 1 || ks->stride_b % 16 || ks->stride_h % 16 || (uintptr_t)ks->ptr % 16 || (uintptr_t)vs->ptr % 16)
    return fail(TR_ERR_STRIDE, "scales: stride_s must be 1, pointer and other strides multiples of 16");
  if (written) {
    if ((st = check_written("k_scales", ks)) != TR_OK) return st;
    if (!apart(ks, vs)) return fail(TR_ERR_ALIAS, "k_scales and v_scales overlap");
    for (const tr_tensor* s : {ks, vs})
      if (overlaps(s, kp) || overlaps(s, vp)) return fail(TR_ERR_ALIAS, "scales overlap pages");
  }
  return TR_OK;
}

// tokens: S of the call's tensors, -1: q_start is not used.
tr_status take_sequences(const tr_sequences* seqs, const tr_tensor* pages, int64_t tokens, Sequences& s, SeqViews& views) {
  if (!seqs) return fail(TR_ERR_NULL, "the sequences are NULL");
  if (seqs->n_seqs < 0 || seqs->n_seqs > (1 << 24)) return fail(TR_ERR_SHAPE, "%lld sequences out of range [0, 2^24]", (long long)seqs->n_seqs);
  if (seqs->max_pages < 0 || seqs->max_pages > kMaxKeys / pages->S) return fail(TR_ERR_SHAPE, "max_pages %lld out of range: at most 2^30 keys a sequence", (long long)seqs->max_pages);
  if (seqs->n_seqs > 0) {
    if (!seqs->kv_len || (tokens >= 0 && !seqs->q_start) || (seqs->max_pages > 0 && !seqs->page_table)) return fail(TR_ERR_NULL, "an array of the sequences is NULL");
    if (seqs->table_stride < 0 || (seqs->n_seqs > 1 && seqs->table_stride < seqs->max_pages))
      return fail(TR_ERR_STRIDE, "table_stride %lld smaller than max_pages %lld", (long long)seqs->table_stride, (long long)seqs->max_pages);
    if (((uintptr_t)seqs->page_table | (uintptr_t)seqs->kv_len | (uintptr_t)(tokens >= 0 ? seqs->q_start : nullptr) | (uintptr_t)(tokens >= 0 ? seqs->q_pos : nullptr)) % 4)
      return fail(TR_ERR_STRIDE, "an array of the sequences is not 4-byte aligned");
  }
  s.table = seqs->page_table; s.kv_len = seqs->kv_len; s.q_start = seqs->q_start; s.q_pos = seqs->q_pos;
  s.table_stride = seqs->table_stride;
  s.n = (int)seqs->n_seqs; s.max_pages = pages->B > 0 ? (int)seqs->max_pages : 0;   // (no pages: no keys)
  s.tokens = (int)(tokens < 0 ? 0 : tokens);
  s.n_pages = (int)pages->B; s.page_size = (int)pages->S;
  s.by_page = make_divisor((unsigned)pages->S);
  views.add(seqs->page_table, seqs->max_pages > 0 && seqs->n_seqs > 0 ? (seqs->n_seqs - 1) * seqs->table_stride + seqs->max_pages : 0);
  views.add(seqs->kv_len, seqs->n_seqs);
  if (tokens >= 0) {
    views.add(seqs->q_start, seqs->n_seqs > 0 ? seqs->n_seqs + 1 : 0);
    views.add(seqs->q_pos, seqs->n_seqs);
  }
  return TR_OK;
}

// No tensor that a call writes shares memory with one that it reads, or with another that it writes.
tr_status check_apart(const tr_tensor* const* written, int n_written, const tr_tensor* const* read, int n_read, const SeqViews& views) {
  for (int i = 0; i < n_written; i++) {
    if (!written[i]) continue;
    for (int j = 0; j < n_read; j++)
      if (read[j] && overlaps(written[i], read[j])) return fail(TR_ERR_ALIAS, "outputs overlap inputs");
    for (int j = 0; j < views.n; j++)
      if (overlaps(written[i], &views.t[j])) return fail(TR_ERR_ALIAS, "outputs overlap the arrays of the sequences");
  }
  return TR_OK;
}

}  // namespace
}  // namespace tr
