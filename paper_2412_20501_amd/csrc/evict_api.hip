// C ABI of the operators that choose and move the keys of a paged cache: argument validation, descriptor -> kernel-parameter marshalling.
#include <math.h>
#include <string.h>

#include "evict.h"
#include "paged_checks.h"

using tr::check_apart;
using tr::check_cache;
using tr::check_tensor;
using tr::check_typed;
using tr::check_written;
using tr::elem_bytes;
using tr::fail;
using tr::overlaps;
using tr::SeqViews;
using tr::take_sequences;
using tr::View;

namespace {

// Weights of the keys on pages; `pages`: of what shape, or null.
tr_status check_weights(const tr_tensor* w, const tr_tensor* pages, bool written) {
  tr_status st;
  if ((st = check_typed("weights", w, tr::kF32, 4)) != TR_OK) return st;
  if (w->D != 1) return fail(TR_ERR_SHAPE, "weights must be [n_pages, Hkv, page_size]");
  if (pages && (w->B != pages->B || w->H != pages->H || w->S != pages->S)) return fail(TR_ERR_SHAPE, "weights shape does not match the pages");
  if (w->H < 1) return fail(TR_ERR_SHAPE, "a cache needs a K/V head");
  if (w->S < 16 || w->S % 16) return fail(TR_ERR_SHAPE, "page size %lld is not a multiple of 16", (long long)w->S);
  if (w->stride_s != 1 || w->stride_b % 4 || w->stride_h % 4 || (uintptr_t)w->ptr % 16) return fail(TR_ERR_STRIDE, "weights: stride_s must be 1, pointer and other strides multiples of 16 bytes");
  return written ? check_written("weights", w) : TR_OK;
}

// An int32 array as a tensor, for overlap tests.
tr_tensor ints(const int32_t* ptr, int64_t elems) {
  tr_tensor t;
  memset(&t, 0, sizeof(t));
  t.ptr = const_cast<int32_t*>(ptr);
  t.dtype = TR_F32;
  t.B = t.H = t.S = 1;
  t.D = ptr ? elems : 0;
  return t;
}

// keys: as a tensor [n_seqs, heads, 1, max_keys]
tr_status check_kept(const tr_kept* kept, int64_t n_seqs, int64_t heads, bool written, tr_tensor& keys, tr_tensor& count) {
  if (!kept) return fail(TR_ERR_NULL, "the kept keys are NULL");
  if (kept->heads != heads && (written || kept->heads != 1)) return fail(TR_ERR_SHAPE, "kept keys of %lld heads, the pages have %lld", (long long)kept->heads, (long long)heads);
  if (kept->max_keys < 0 || kept->max_keys > tr::kMaxKeys) return fail(TR_ERR_SHAPE, "max_keys %lld out of range [0, 2^30]", (long long)kept->max_keys);
  if (kept->stride_b < 0 || kept->stride_h < 0) return fail(TR_ERR_STRIDE, "kept keys: negative stride");
  memset(&keys, 0, sizeof(keys));
  keys.ptr = kept->keys; keys.dtype = TR_F32;
  keys.B = n_seqs; keys.H = kept->heads; keys.S = 1; keys.D = kept->max_keys;
  keys.stride_b = n_seqs > 1 ? kept->stride_b : 0; keys.stride_h = kept->heads > 1 ? kept->stride_h : 0;
  count = ints(kept->count, n_seqs);
  if (n_seqs > 0 && (!kept->count || (kept->max_keys > 0 && !kept->keys))) return fail(TR_ERR_NULL, "an array of the kept keys is NULL");
  if (((uintptr_t)kept->keys | (uintptr_t)kept->count) % 4) return fail(TR_ERR_STRIDE, "an array of the kept keys is not 4-byte aligned");
  tr_status st;
  if (written && (st = check_written("keys", &keys)) != TR_OK) return st;
  return TR_OK;
}

}  // namespace

extern "C" {

tr_status tr_cache_weigh(const tr_tensor* q_, const tr_tensor* lse_, const tr_tensor* k_pages_, const tr_tensor* k_scales_, const tr_sequences* seqs,
                         int causal, float scale, int fresh, const tr_tensor* weights_, void* hip_stream) {
  tr::clear_error();
  const View q_view(q_), lse_view(lse_), k_pages_view(k_pages_), k_scales_view(k_scales_), weights_view(weights_);
  const tr_tensor * const q = q_view.at, * const lse = lse_view.at, * const k_pages = k_pages_view.at, * const k_scales = k_scales_view.at, * const weights = weights_view.at;
  tr_status st;
  if ((st = check_tensor("q", q, true, false, 16)) != TR_OK || (st = check_tensor("lse", lse, false, true, 4)) != TR_OK) return st;
  if ((st = check_cache(k_pages, k_pages, k_scales, k_scales, false)) != TR_OK) return st;
  if ((st = check_weights(weights, k_pages, true)) != TR_OK) return st;
  if (q->B != 1 || lse->B != 1) return fail(TR_ERR_SHAPE, "q and lse hold the tokens of all sequences along S: B must be 1");
  if (q->D != k_pages->D) return fail(TR_ERR_SHAPE, "head dims of q and the pages differ");
  if (lse->H != q->H || lse->S != q->S || lse->D != 1) return fail(TR_ERR_SHAPE, "lse shape does not match q");
  if (q->H < 1) return fail(TR_ERR_SHAPE, "weighing needs a query head");
  if (q->H % k_pages->H) return fail(TR_ERR_SHAPE, "query heads %lld not a multiple of K/V heads %lld", (long long)q->H, (long long)k_pages->H);
  if (!(scale > 0.f) || !isfinite(scale)) return fail(TR_ERR_UNSUPPORTED, "scale must be finite and > 0");
  if (q->S * q->H >= tr::kMaxKeys) return fail(TR_ERR_SHAPE, "too many rows for one call (S * Hq must stay below 2^30)");
  tr::WeighParams p;
  memset(&p, 0, sizeof(p));
  SeqViews views;
  if ((st = take_sequences(seqs, k_pages, q->S, p.seq, views)) != TR_OK) return st;
  if (seqs->n_seqs > tr::kMaxAttended) return fail(TR_ERR_SHAPE, "%lld sequences, one call weighs for 2^16 at most", (long long)seqs->n_seqs);
  // (the kernels round the number of stretches of keys up to a multiple of 8)
  if ((double)seqs->n_seqs * (double)k_pages->H * (double)((seqs->max_pages * k_pages->S + 63) / 64) >= 0x1p31 - 8) return fail(TR_ERR_SHAPE, "too many keys for one call (sequences * Hkv * keys / 64 must stay below 2^31 - 8)");
  const tr_tensor* const written[] = {weights};
  const tr_tensor* const read[] = {q, lse, k_pages, k_scales};
  if ((st = check_apart(written, 1, read, 4, views)) != TR_OK) return st;
  if (q->S == 0 || p.seq.n == 0 || p.seq.max_pages == 0) return TR_OK;
  const int64_t eb = elem_bytes(k_pages->dtype);
  p.q = (const __bf16*)q->ptr; p.lse = (const float*)lse->ptr; p.weights = (float*)weights->ptr;
  p.q_sh = q->stride_h; p.q_ss = q->stride_s;
  p.l_sh = lse->stride_h; p.l_ss = lse->stride_s;
  p.k_pages = (const char*)k_pages->ptr;
  p.page_b = k_pages->stride_b * eb; p.head_b = k_pages->stride_h * eb; p.slot_b = (int)(k_pages->stride_s * eb);
  if (k_scales) {
    p.k_scales = (const unsigned char*)k_scales->ptr;
    p.scale_sp = k_scales->stride_b; p.scale_sh = k_scales->stride_h;
  }
  p.w_sp = weights->stride_b; p.w_sh = weights->stride_h;
  p.Hkv = (int)k_pages->H; p.gq = (int)(q->H / k_pages->H);
  p.by_gq = tr::make_divisor((unsigned)p.gq);
  p.causal = causal != 0; p.fresh = fresh != 0;
  p.scale = scale;
  const hipError_t e = tr::launch_cache_weigh(p, (int)q->D, k_scales != nullptr, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(TR_ERR_HIP, "cache weigh launch failed: %s", hipGetErrorString(e));
  return TR_OK;
}

tr_status tr_cache_select(const tr_tensor* weights_, const tr_sequences* seqs, int64_t first, int64_t last, const tr_kept* kept, void* hip_stream) {
  tr::clear_error();
  const View weights_view(weights_);
  const tr_tensor* const weights = weights_view.at;
  tr_status st;
  if ((st = check_weights(weights, nullptr, false)) != TR_OK) return st;
  tr::SelectParams p;
  memset(&p, 0, sizeof(p));
  SeqViews views;
  if ((st = take_sequences(seqs, weights, -1, p.seq, views)) != TR_OK) return st;
  tr_tensor keys, count;
  if ((st = check_kept(kept, seqs->n_seqs, weights->H, true, keys, count)) != TR_OK) return st;
  if (first < 0 || last < 0 || first > kept->max_keys || last > kept->max_keys - first)
    return fail(TR_ERR_SHAPE, "first %lld and last %lld keys do not fit among %lld", (long long)first, (long long)last, (long long)kept->max_keys);
  const tr_tensor* const written[] = {&keys, &count};
  const tr_tensor* const read[] = {weights};
  if ((st = check_apart(written, 2, read, 1, views)) != TR_OK) return st;
  if (overlaps(&keys, &count)) return fail(TR_ERR_ALIAS, "keys and count overlap");
  if (p.seq.n == 0) return TR_OK;
  p.weights = (const float*)weights->ptr;
  p.w_sp = weights->stride_b; p.w_sh = weights->stride_h;
  p.heads = (int)weights->H; p.first = (int)first; p.last = (int)last; p.most = (int)kept->max_keys;
  p.keys = kept->keys; p.count = kept->count;
  p.k_sb = keys.stride_b; p.k_sh = keys.stride_h;
  const hipError_t e = tr::launch_cache_select(p, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(TR_ERR_HIP, "cache select launch failed: %s", hipGetErrorString(e));
  return TR_OK;
}

tr_status tr_cache_keep(const tr_tensor* k_pages_, const tr_tensor* v_pages_, const tr_tensor* k_scales_, const tr_tensor* v_scales_, const tr_tensor* weights_,
                        const tr_sequences* seqs, const tr_kept* kept, const int32_t* start, void* hip_stream) {
  tr::clear_error();
  const View k_pages_view(k_pages_), v_pages_view(v_pages_), k_scales_view(k_scales_), v_scales_view(v_scales_), weights_view(weights_);
  const tr_tensor * const k_pages = k_pages_view.at, * const v_pages = v_pages_view.at, * const k_scales = k_scales_view.at, * const v_scales = v_scales_view.at, * const weights = weights_view.at;
  tr_status st;
  if ((st = check_cache(k_pages, v_pages, k_scales, v_scales, true)) != TR_OK) return st;
  if (weights && (st = check_weights(weights, k_pages, true)) != TR_OK) return st;
  tr::KeepParams p;
  memset(&p, 0, sizeof(p));
  SeqViews views;
  if ((st = take_sequences(seqs, k_pages, -1, p.seq, views)) != TR_OK) return st;
  tr_tensor keys, count;
  if ((st = check_kept(kept, seqs->n_seqs, k_pages->H, false, keys, count)) != TR_OK) return st;
  if ((uintptr_t)start % 4) return fail(TR_ERR_STRIDE, "start is not 4-byte aligned");
  const tr_tensor starts = ints(start, seqs->n_seqs);
  const tr_tensor* const written[] = {k_pages, v_pages, k_scales, v_scales, weights};
  const tr_tensor* const read[] = {&keys, &count, &starts};
  if ((st = check_apart(written, 5, read, 3, views)) != TR_OK) return st;
  if (weights)
    for (int i = 0; i < 4; i++)
      if (written[i] && overlaps(weights, written[i])) return fail(TR_ERR_ALIAS, "weights overlap pages or scales");
  if (p.seq.n == 0 || p.seq.max_pages == 0 || kept->max_keys == 0) return TR_OK;
  const int64_t eb = elem_bytes(k_pages->dtype);
  p.k_pages = (char*)k_pages->ptr; p.v_pages = (char*)v_pages->ptr;
  p.page_b = k_pages->stride_b * eb; p.head_b = k_pages->stride_h * eb; p.slot_b = k_pages->stride_s * eb;
  if (k_scales) {
    p.k_scales = (unsigned char*)k_scales->ptr; p.v_scales = (unsigned char*)v_scales->ptr;
    p.scale_sp = k_scales->stride_b; p.scale_sh = k_scales->stride_h;
  }
  if (weights) {
    p.weights = (float*)weights->ptr;
    p.w_sp = weights->stride_b; p.w_sh = weights->stride_h;
  }
  p.heads = (int)k_pages->H; p.row_bytes = (int)(k_pages->D * eb); p.most = (int)kept->max_keys;
  p.keys = kept->keys; p.count = kept->count; p.start = start;
  p.k_sb = keys.stride_b; p.k_sh = keys.stride_h;
  const hipError_t e = tr::launch_cache_keep(p, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(TR_ERR_HIP, "cache keep launch failed: %s", hipGetErrorString(e));
  return TR_OK;
}

}  // extern "C"
