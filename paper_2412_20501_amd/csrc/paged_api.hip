// C ABI of the operators on a paged cache: argument validation, descriptor -> kernel-parameter marshalling.
#include <math.h>
#include <string.h>

#include "checks.h"
#include "paged.h"

using tr::check_tensor;
using tr::check_typed;
using tr::check_written;
using tr::elem_bytes;
using tr::fail;
using tr::overlaps;

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
  tr_tensor t[4];
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
  if ((st = check_typed("k_pages", kp, tr::kBf16 | tr::kF8, 16)) != TR_OK) return st;
  if ((st = check_typed("v_pages", vp, tr::kBf16 | tr::kF8, 16)) != TR_OK) return st;
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
  if ((st = check_typed("k_scales", ks, tr::kE8m0, 1)) != TR_OK) return st;
  if ((st = check_typed("v_scales", vs, tr::kE8m0, 1)) != TR_OK) return st;
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
tr_status take_sequences(const tr_sequences* seqs, const tr_tensor* pages, int64_t tokens, tr::Sequences& s, SeqViews& views) {
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
  s.by_page = tr::make_divisor((unsigned)pages->S);
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

void set_pages(tr::CacheCopyParams& p, const tr_tensor* kp, const tr_tensor* vp, const tr_tensor* ks, const tr_tensor* vs) {
  const int64_t eb = elem_bytes(kp->dtype);
  p.k_pages = (char*)kp->ptr; p.v_pages = (char*)vp->ptr;
  p.page_b = kp->stride_b * eb; p.head_b = kp->stride_h * eb; p.slot_b = kp->stride_s * eb;
  if (ks) {
    p.k_scales = (unsigned char*)ks->ptr; p.v_scales = (unsigned char*)vs->ptr;
    p.scale_sp = ks->stride_b; p.scale_sh = ks->stride_h;
  }
  p.heads = (int)kp->H;
  p.by_heads = tr::make_divisor((unsigned)kp->H * 2);
}

}  // namespace

extern "C" {

tr_status tr_cache_write(const tr_tensor* k_, const tr_tensor* v_, const tr_tensor* k_pages_, const tr_tensor* v_pages_,
                         const tr_tensor* k_scales_, const tr_tensor* v_scales_, const tr_sequences* seqs, void* hip_stream) {
  tr::clear_error();
  const View k_view(k_);
  const View v_view(v_);
  const View k_pages_view(k_pages_);
  const View v_pages_view(v_pages_);
  const View k_scales_view(k_scales_);
  const View v_scales_view(v_scales_);
  const tr_tensor * const k = k_view.at, * const v = v_view.at, * const k_pages = k_pages_view.at, * const v_pages = v_pages_view.at, * const k_scales = k_scales_view.at, * const v_scales = v_scales_view.at;
  tr_status st;
  if ((st = check_tensor("k", k, true, false, 16)) != TR_OK || (st = check_tensor("v", v, true, false, 16)) != TR_OK) return st;
  if ((st = check_cache(k_pages, v_pages, k_scales, v_scales, true)) != TR_OK) return st;
  if (k->B != 1 || v->B != 1) return fail(TR_ERR_SHAPE, "k and v hold the tokens of all sequences along S: B must be 1");
  if (k->H != k_pages->H || k->D != k_pages->D) return fail(TR_ERR_SHAPE, "k does not match the pages' heads or head dim");
  if (v->H != k->H || v->S != k->S || v->D != k->D) return fail(TR_ERR_SHAPE, "k and v shapes differ");
  if (k->stride_h != v->stride_h || k->stride_s != v->stride_s) return fail(TR_ERR_STRIDE, "k and v must share their strides");
  if ((k->S + 63) / 64 * k->H * 2 >= kMaxGroups) return fail(TR_ERR_SHAPE, "too many rows for one call (2 * ceil(S / 64) * Hkv must stay below 2^24)");
  tr::CacheCopyParams p;
  memset(&p, 0, sizeof(p));
  SeqViews views;
  if ((st = take_sequences(seqs, k_pages, k->S, p.seq, views)) != TR_OK) return st;
  const tr_tensor* const written[] = {k_pages, v_pages, k_scales, v_scales};
  const tr_tensor* const read[] = {k, v};
  if ((st = check_apart(written, 4, read, 2, views)) != TR_OK) return st;
  set_pages(p, k_pages, v_pages, k_scales, v_scales);
  p.k = (const char*)k->ptr; p.v = (const char*)v->ptr;
  p.d_sh = k->stride_h; p.d_ss = k->stride_s;
  if (p.seq.tokens == 0 || p.seq.n == 0 || p.seq.max_pages == 0 || p.seq.n_pages == 0) return TR_OK;
  const hipError_t e = tr::launch_cache_write(p, (int)k->D, k_scales != nullptr, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(TR_ERR_HIP, "cache write launch failed: %s", hipGetErrorString(e));
  return TR_OK;
}

tr_status tr_cache_read(const tr_tensor* k_pages_, const tr_tensor* v_pages_, const tr_tensor* k_scales_, const tr_tensor* v_scales_,
                        const tr_sequences* seqs, int64_t first, const tr_tensor* k_, const tr_tensor* v_, void* hip_stream) {
  tr::clear_error();
  const View k_pages_view(k_pages_);
  const View v_pages_view(v_pages_);
  const View k_scales_view(k_scales_);
  const View v_scales_view(v_scales_);
  const View k_view(k_);
  const View v_view(v_);
  const tr_tensor * const k_pages = k_pages_view.at, * const v_pages = v_pages_view.at, * const k_scales = k_scales_view.at, * const v_scales = v_scales_view.at, * const k = k_view.at, * const v = v_view.at;
  tr_status st;
  if ((st = check_cache(k_pages, v_pages, k_scales, v_scales, false)) != TR_OK) return st;
  if ((st = check_tensor("k", k, true, false, 16)) != TR_OK || (st = check_tensor("v", v, true, false, 16)) != TR_OK) return st;
  if ((st = check_written("k", k)) != TR_OK || (st = check_written("v", v)) != TR_OK) return st;
  if (first < 0) return fail(TR_ERR_SHAPE, "first must be >= 0");
  if (k->H != k_pages->H || k->D != k_pages->D) return fail(TR_ERR_SHAPE, "k does not match the pages' heads or head dim");
  if (v->B != k->B || v->H != k->H || v->S != k->S || v->D != k->D) return fail(TR_ERR_SHAPE, "k and v shapes differ");
  if (k->stride_b != v->stride_b || k->stride_h != v->stride_h || k->stride_s != v->stride_s) return fail(TR_ERR_STRIDE, "k and v must share their strides");
  tr::CacheCopyParams p;
  memset(&p, 0, sizeof(p));
  SeqViews views;
  if ((st = take_sequences(seqs, k_pages, -1, p.seq, views)) != TR_OK) return st;
  if (k->B != seqs->n_seqs) return fail(TR_ERR_SHAPE, "k has %lld batch entries for %lld sequences", (long long)k->B, (long long)seqs->n_seqs);
  if ((k->S + 63) / 64 * k->H * 2 >= kMaxGroups) return fail(TR_ERR_SHAPE, "too many rows for one call (2 * ceil(S / 64) * Hkv must stay below 2^24)");
  if (2 * k->B * k->H >= ((int64_t)1 << 31)) return fail(TR_ERR_SHAPE, "too many heads for one call (2 * sequences * Hkv must stay below 2^31)");
  const tr_tensor* const written[] = {k, v};
  const tr_tensor* const read[] = {k_pages, v_pages, k_scales, v_scales};
  if ((st = check_apart(written, 2, read, 4, views)) != TR_OK) return st;
  if (!apart(k, v)) return fail(TR_ERR_ALIAS, "k and v overlap");
  set_pages(p, k_pages, v_pages, k_scales, v_scales);
  p.k_out = (char*)k->ptr; p.v_out = (char*)v->ptr;
  p.d_sb = k->stride_b; p.d_sh = k->stride_h; p.d_ss = k->stride_s;
  p.rows = (int)k->S;
  p.first = first < kMaxKeys ? first : kMaxKeys;
  if (p.rows == 0 || p.seq.n == 0 || p.seq.max_pages == 0 || p.seq.n_pages == 0) return TR_OK;
  const hipError_t e = tr::launch_cache_read(p, (int)k->D, k_scales != nullptr, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(TR_ERR_HIP, "cache read launch failed: %s", hipGetErrorString(e));
  return TR_OK;
}

size_t tr_paged_attn_workspace_bytes(const tr_tensor* q, const tr_tensor* k_pages, int64_t n_seqs, int64_t max_pages) {
  if (!q || !k_pages || q->dtype != TR_BF16 || q->B != 1 || q->S < 0 || q->S > kMaxKeys || q->H < 0 || q->H > INT32_MAX || (q->D != 64 && q->D != 128)) return 0;
  if ((k_pages->dtype != TR_BF16 && k_pages->dtype != TR_F8E4M3) || k_pages->B < 0 || k_pages->H < 1 || q->H % k_pages->H || k_pages->D != q->D || k_pages->S < 16 || k_pages->S % 16) return 0;
  if (n_seqs < 0 || n_seqs > kMaxAttended || max_pages < 0 || max_pages > kMaxKeys / k_pages->S || q->S * q->H >= ((int64_t)1 << 31)) return 0;
  if (q->S == 0 || q->H == 0 || n_seqs == 0) return 0;
  const tr::PagedLaunch l = tr::paged_launch(q->S, n_seqs, max_pages * k_pages->S, (int)k_pages->H, (int)(q->H / k_pages->H), (int)q->D, k_pages->dtype == TR_F8E4M3);
  int64_t floats = 0;
  for (int i = 0; i < l.n; i++) floats += l.part[i].floats((int)q->D);
  return (size_t)floats * 4;
}

tr_status tr_paged_attn(const tr_tensor* q_, const tr_tensor* k_pages_, const tr_tensor* v_pages_, const tr_tensor* k_scales_,
                        const tr_tensor* v_scales_, const tr_sequences* seqs, int causal, float scale, const tr_tensor* out_,
                        const tr_tensor* lse_, void* workspace, size_t workspace_bytes, void* hip_stream) {
  tr::clear_error();
  const View q_view(q_);
  const View k_pages_view(k_pages_);
  const View v_pages_view(v_pages_);
  const View k_scales_view(k_scales_);
  const View v_scales_view(v_scales_);
  const View out_view(out_);
  const View lse_view(lse_);
  const tr_tensor * const q = q_view.at, * const k_pages = k_pages_view.at, * const v_pages = v_pages_view.at, * const k_scales = k_scales_view.at, * const v_scales = v_scales_view.at, * const out = out_view.at, * const lse = lse_view.at;
  tr_status st;
  if ((st = check_tensor("q", q, true, false, 16)) != TR_OK) return st;
  if ((st = check_cache(k_pages, v_pages, k_scales, v_scales, false)) != TR_OK) return st;
  if ((st = check_tensor("out", out, true, true, 16)) != TR_OK) return st;
  if ((st = check_tensor("lse", lse, false, true, 4)) != TR_OK) return st;
  if ((st = check_written("out", out)) != TR_OK || (st = check_written("lse", lse)) != TR_OK) return st;
  if (q->B != 1 || out->B != 1 || lse->B != 1) return fail(TR_ERR_SHAPE, "q, out and lse hold the tokens of all sequences along S: B must be 1");
  if (q->D != k_pages->D) return fail(TR_ERR_SHAPE, "head dims of q and the pages differ");
  if (out->H != q->H || out->S != q->S || out->D != q->D || lse->H != q->H || lse->S != q->S || lse->D != 1) return fail(TR_ERR_SHAPE, "out/lse shape does not match q");
  if (q->H % k_pages->H) return fail(TR_ERR_SHAPE, "query heads %lld not a multiple of K/V heads %lld", (long long)q->H, (long long)k_pages->H);
  if (!(scale > 0.f) || !isfinite(scale)) return fail(TR_ERR_UNSUPPORTED, "scale must be finite and > 0");
  if (q->S * q->H >= ((int64_t)1 << 31)) return fail(TR_ERR_SHAPE, "too many rows for one call (S * Hq must stay below 2^31)");
  tr::PagedParams p;
  memset(&p, 0, sizeof(p));
  SeqViews views;
  if ((st = take_sequences(seqs, k_pages, q->S, p.seq, views)) != TR_OK) return st;
  if (seqs->n_seqs > kMaxAttended) return fail(TR_ERR_SHAPE, "%lld sequences, one call attends for 2^16 at most", (long long)seqs->n_seqs);
  const tr_tensor* const written[] = {out, lse};
  const tr_tensor* const read[] = {q, k_pages, v_pages, k_scales, v_scales};
  if ((st = check_apart(written, 2, read, 5, views)) != TR_OK) return st;
  if (overlaps(out, lse)) return fail(TR_ERR_ALIAS, "out and lse overlap");
  if (q->H == 0 || q->S == 0 || p.seq.n == 0) return TR_OK;

  const int gq = (int)(q->H / k_pages->H), D = (int)q->D;
  const tr::PagedLaunch l = tr::paged_launch(q->S, p.seq.n, (int64_t)p.seq.max_pages * p.seq.page_size, (int)k_pages->H, gq, D, k_scales != nullptr);
  for (int i = 0; i < l.n; i++)
    if (l.part[i].tiles + l.part[i].share.most() >= ((int64_t)1 << 23) - 8) return fail(TR_ERR_SHAPE, "too many workgroups for one launch");   // (of 512 threads, fewer than 2^32 in all)
  const size_t need = tr_paged_attn_workspace_bytes(q, k_pages, seqs->n_seqs, seqs->max_pages);
  if (workspace && need > 0) {
    if ((uintptr_t)workspace % 256) return fail(TR_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(TR_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    tr_tensor all;
    memset(&all, 0, sizeof(all));
    all.ptr = workspace; all.dtype = TR_F32;
    all.B = all.H = all.S = 1;
    all.D = (int64_t)(need / 4);
    const tr_tensor* const ws[] = {&all};
    const tr_tensor* const others[] = {q, k_pages, v_pages, k_scales, v_scales, out, lse};
    if (check_apart(ws, 1, others, 7, views) != TR_OK) return fail(TR_ERR_ALIAS, "workspace overlaps a tensor argument");
  }
  p.q = (const __bf16*)q->ptr; p.out = out->ptr; p.lse = (float*)lse->ptr;
  p.q_sh = q->stride_h; p.q_ss = q->stride_s;
  p.o_sh = out->stride_h; p.o_ss = out->stride_s;
  p.l_sh = lse->stride_h; p.l_ss = lse->stride_s;
  const int64_t eb = elem_bytes(k_pages->dtype);
  p.k_pages = (const char*)k_pages->ptr; p.v_pages = (const char*)v_pages->ptr;
  p.page_b = k_pages->stride_b * eb; p.head_b = k_pages->stride_h * eb; p.slot_b = (int)(k_pages->stride_s * eb);
  if (k_scales) {
    p.k_scales = (const unsigned char*)k_scales->ptr; p.v_scales = (const unsigned char*)v_scales->ptr;
    p.scale_sp = k_scales->stride_b; p.scale_sh = k_scales->stride_h;
  }
  p.Hkv = (int)k_pages->H; p.gq = gq;
  p.by_gq = tr::make_divisor((unsigned)gq);
  p.causal = causal != 0; p.out_f32 = out->dtype == TR_F32;
  p.scale = scale;
  const hipError_t e = tr::launch_paged_attn(p, l, D, k_scales != nullptr, need > 0 ? (float*)workspace : nullptr, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(TR_ERR_HIP, "paged attention launch failed: %s", hipGetErrorString(e));
  return TR_OK;
}

}  // extern "C"
