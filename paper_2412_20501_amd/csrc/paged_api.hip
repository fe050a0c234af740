// C ABI of the operators on a paged cache: argument validation, descriptor -> kernel-parameter marshalling.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "paged_checks.h"

using tr::check_apart;
using tr::check_cache;
using tr::check_tensor;
using tr::check_written;
using tr::elem_bytes;
using tr::fail;
using tr::kMaxAttended;
using tr::kMaxGroups;
using tr::kMaxKeys;
using tr::overlaps;
using tr::SeqViews;
using tr::take_sequences;
using tr::View;

namespace {

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

tr_status take_tree(const tr_tree& tree, int64_t tokens, tr::TreeParams& p, SeqViews& views) {
  if (tree.tokens != tokens) return fail(TR_ERR_SHAPE, "a tree of %lld tokens for %lld", (long long)tree.tokens, (long long)tokens);
  if (tree.words < 1 || tree.words > (1 << 15)) return fail(TR_ERR_SHAPE, "%lld words a row of the tree out of range [1, 2^15]", (long long)tree.words);
  if (tokens > 0 && !tree.bits) return fail(TR_ERR_NULL, "the tree's bits are NULL");
  if (tree.stride != 0 && tree.stride < tree.words && tokens > 1) return fail(TR_ERR_STRIDE, "rows of %lld words of the tree lie %lld apart", (long long)tree.words, (long long)tree.stride);
  if (tree.stride < 0 || (uintptr_t)tree.bits % 4) return fail(TR_ERR_STRIDE, "the tree's stride is negative, or its bits are not 4-byte aligned");
  p.tree = reinterpret_cast<const unsigned*>(tree.bits);
  p.tree_stride = tokens > 1 ? tree.stride : 0;
  p.words = (int)tree.words;
  if (tokens > 0) views.add(tree.bits, (tokens - 1) * p.tree_stride + tree.words);
  return TR_OK;
}

size_t workspace_bytes_of(const tr_tensor* q, const tr_tensor* k_pages, int64_t n_seqs, int64_t max_pages, bool tree) {
  if (!q || !k_pages || q->dtype != TR_BF16 || q->B != 1 || q->S < 0 || q->S > kMaxKeys || q->H < 0 || q->H > INT32_MAX || (q->D != 64 && q->D != 128)) return 0;
  if ((k_pages->dtype != TR_BF16 && k_pages->dtype != TR_F8E4M3) || k_pages->B < 0 || k_pages->H < 1 || q->H % k_pages->H || k_pages->D != q->D || k_pages->S < 16 || k_pages->S % 16) return 0;
  if (n_seqs < 0 || n_seqs > kMaxAttended || max_pages < 0 || max_pages > kMaxKeys / k_pages->S || q->S * q->H >= ((int64_t)1 << 31)) return 0;
  if (q->S == 0 || q->H == 0 || n_seqs == 0) return 0;
  const tr::PagedLaunch l = tr::paged_launch(q->S, n_seqs, max_pages * k_pages->S, (int)k_pages->H, (int)(q->H / k_pages->H), (int)q->D, k_pages->dtype == TR_F8E4M3, tree);
  int64_t floats = 0;
  for (int i = 0; i < l.n; i++) floats += l.part[i].floats((int)q->D);
  return (size_t)floats * 4;
}

// tr_paged_attn (P = PagedParams, tree = null) and tr_paged_attn_tree (TreeParams).
template <typename P>
__attribute__((always_inline)) inline tr_status attend(const tr_tensor* q_, const tr_tensor* k_pages_, const tr_tensor* v_pages_, const tr_tensor* k_scales_,
                 const tr_tensor* v_scales_, const tr_sequences* seqs, const tr_tree* tree, int causal, float scale, const tr_tensor* out_,
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
  P p;
  memset(&p, 0, sizeof(p));
  SeqViews views;
  if ((st = take_sequences(seqs, k_pages, q->S, p.seq, views)) != TR_OK) return st;
  if (seqs->n_seqs > kMaxAttended) return fail(TR_ERR_SHAPE, "%lld sequences, one call attends for 2^16 at most", (long long)seqs->n_seqs);
  constexpr bool TREE = std::is_same<P, tr::TreeParams>::value;
  if constexpr (TREE) {
    if ((st = take_tree(*tree, q->S, p, views)) != TR_OK) return st;
  }
  const tr_tensor* const written[] = {out, lse};
  const tr_tensor* const read[] = {q, k_pages, v_pages, k_scales, v_scales};
  if ((st = check_apart(written, 2, read, 5, views)) != TR_OK) return st;
  if (overlaps(out, lse)) return fail(TR_ERR_ALIAS, "out and lse overlap");
  if (q->H == 0 || q->S == 0 || p.seq.n == 0) return TR_OK;

  const int gq = (int)(q->H / k_pages->H), D = (int)q->D;
  const tr::PagedLaunch l = tr::paged_launch(q->S, p.seq.n, (int64_t)p.seq.max_pages * p.seq.page_size, (int)k_pages->H, gq, D, k_scales != nullptr, TREE);
  for (int i = 0; i < l.n; i++)
    if (l.part[i].tiles + l.part[i].share.most() >= ((int64_t)1 << 23) - 8) return fail(TR_ERR_SHAPE, "too many workgroups for one launch");   // (of 512 threads, fewer than 2^32 in all)
  const size_t need = workspace_bytes_of(q, k_pages, seqs->n_seqs, seqs->max_pages, TREE);
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
  if (!tr::apart(k, v)) return fail(TR_ERR_ALIAS, "k and v overlap");
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
  return workspace_bytes_of(q, k_pages, n_seqs, max_pages, false);
}
size_t tr_paged_attn_tree_workspace_bytes(const tr_tensor* q, const tr_tensor* k_pages, int64_t n_seqs, int64_t max_pages) {
  return workspace_bytes_of(q, k_pages, n_seqs, max_pages, true);
}

tr_status tr_paged_attn(const tr_tensor* q, const tr_tensor* k_pages, const tr_tensor* v_pages, const tr_tensor* k_scales, const tr_tensor* v_scales,
                        const tr_sequences* seqs, int causal, float scale, const tr_tensor* out, const tr_tensor* lse, void* workspace,
                        size_t workspace_bytes, void* hip_stream) {
  return attend<tr::PagedParams>(q, k_pages, v_pages, k_scales, v_scales, seqs, nullptr, causal, scale, out, lse, workspace, workspace_bytes, hip_stream);
}

tr_status tr_paged_attn_tree(const tr_tensor* q, const tr_tensor* k_pages, const tr_tensor* v_pages, const tr_tensor* k_scales, const tr_tensor* v_scales,
                             const tr_sequences* seqs, const tr_tree* tree, float scale, const tr_tensor* out, const tr_tensor* lse, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
  if (!tree) {
    tr::clear_error();
    return fail(TR_ERR_NULL, "the tree is NULL");
  }
  return attend<tr::TreeParams>(q, k_pages, v_pages, k_scales, v_scales, seqs, tree, 1, scale, out, lse, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
