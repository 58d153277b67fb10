// Host side of the operators with a key/value cache (include/sparsed.h): argument validation and dispatch.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "cache.hpp"
#include "host.hpp"

using namespace sparsed;

namespace {

// Tokens of a packed array or a sequence: positions and the ends of their blocks are worked out in 32 bits.
constexpr int64_t kMaxTokens = (int64_t)1 << 30;
// Sequences of an attention call: each work-group looks for its place among all of them, so a call's time grows with their square (1024 sequences
// of one token, 32 heads of 64: 0.2 ms, 16384 106, 65536 1670; a million would be minutes).
constexpr int32_t kMaxAttendedSeqs = 1 << 16;
// Rows of a packed array that a kernel addresses with 32-bit byte offsets from a 64-bit base.
constexpr int64_t kRowsPerBase = 128;

hipStream_t stream_of(const sparsed_exec* ex) { return ex ? static_cast<hipStream_t>(ex->stream) : nullptr; }
int element_bytes(const sparsed_tensor* t) { return t->dtype == SPARSED_BF16 ? 2 : 4; }

sparsed_status check_common(const sparsed_tensor* t, const char* name) {
  if (t->dtype != SPARSED_BF16 && t->dtype != SPARSED_F32) return fail(SPARSED_ERR_DTYPE, "%s: unknown dtype %d", name, t->dtype);
  if (t->H <= 0 || t->D <= 0) return fail(SPARSED_ERR_SHAPE, "%s: non-positive dimension [%d,%d,%d,%d]", name, t->B, t->H, t->L, t->D);
  if (t->D != 64 && t->D != 128) return fail(SPARSED_ERR_UNSUPPORTED, "%s: head dim %d not in {64,128}", name, t->D);
  if (reinterpret_cast<uintptr_t>(t->data) % 16 != 0) return fail(SPARSED_ERR_STRIDE, "%s.data is not 16-byte aligned", name);
  return SPARSED_OK;
}

// Whether rows of D elements share memory in an array that is written: strides are taken as nested, the smallest first, which every view
// of an array in some order of its dimensions has. (A layout in which dimensions mesh without meeting counts as sharing.)
struct Dim {
  int64_t n, stride;
};
template <int N>
bool rows_overlap(int D, Dim (&dims)[N]) {
  std::sort(dims, dims + N, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  __int128 extent = D;
  for (const Dim& d : dims) {
    if (d.n <= 1) continue;
    if (d.stride < extent) return true;
    extent += (__int128)d.stride * (d.n - 1);
  }
  return false;
}

// A packed array [1, H, T, D]. Strides of dimensions with one entry are not looked at.
sparsed_status check_packed(const sparsed_tensor* t, const char* name) {
  if (!t) return fail(SPARSED_ERR_NULL, "%s is NULL", name);
  if (t->L > 0 && !t->data) return fail(SPARSED_ERR_NULL, "%s.data is NULL", name);
  const sparsed_status st = check_common(t, name);
  if (st != SPARSED_OK) return st;
  if (t->B != 1 || t->L < 0) return fail(SPARSED_ERR_SHAPE, "%s: [%d,%d,%d,%d] is not a packed array (B = 1, L tokens)", name, t->B, t->H, t->L, t->D);
  if (t->L > kMaxTokens) return fail(SPARSED_ERR_UNSUPPORTED, "%s: %d tokens, the limit is 2^30", name, t->L);
  const int al = 16 / element_bytes(t);
  if ((t->L > 1 && (t->stride_l < t->D || t->stride_l % al)) || (t->H > 1 && (t->stride_h < 0 || t->stride_h % al)))
    return fail(SPARSED_ERR_STRIDE, "%s: strides (%lld,%lld) must be multiples of %d elements and stride_l >= D", name, (long long)t->stride_h,
                (long long)t->stride_l, al);
  if (t->L > 1 && t->stride_l * kRowsPerBase * element_bytes(t) >= ((int64_t)1 << 31))
    return fail(SPARSED_ERR_STRIDE, "%s: %lld rows span %lld bytes, the limit is 2^31", name, (long long)kRowsPerBase,
                (long long)(t->stride_l * kRowsPerBase * element_bytes(t)));
  return SPARSED_OK;
}

sparsed_status check_pages(const sparsed_tensor* t, const char* name) {
  if (!t->data) return fail(SPARSED_ERR_NULL, "%s.data is NULL", name);
  const sparsed_status st = check_common(t, name);
  if (st != SPARSED_OK) return st;
  if (t->B <= 0) return fail(SPARSED_ERR_SHAPE, "%s: %d pages", name, t->B);
  if (t->L != 16 && t->L != 32 && t->L != 64 && t->L != 128 && t->L != 256)
    return fail(SPARSED_ERR_UNSUPPORTED, "%s: page size %d not in {16,32,64,128,256}", name, t->L);
  const int al = 16 / element_bytes(t);
  if (t->stride_l < t->D || t->stride_l % al || (t->H > 1 && (t->stride_h < 0 || t->stride_h % al)) ||
      (t->B > 1 && (t->stride_b < 0 || t->stride_b % al)))
    return fail(SPARSED_ERR_STRIDE, "%s: strides (%lld,%lld,%lld) must be multiples of %d elements and stride_l >= D", name,
                (long long)t->stride_b, (long long)t->stride_h, (long long)t->stride_l, al);
  if (t->stride_l * t->L * element_bytes(t) >= ((int64_t)1 << 31))
    return fail(SPARSED_ERR_STRIDE, "%s: a page of one head spans %lld bytes, the limit is 2^31", name,
                (long long)(t->stride_l * t->L * element_bytes(t)));
  return SPARSED_OK;
}

sparsed_status check_cache(const sparsed_paged_cache* c) {
  if (!c) return fail(SPARSED_ERR_NULL, "cache is NULL");
  sparsed_status st;
  if ((st = check_pages(&c->k, "cache k")) || (st = check_pages(&c->v, "cache v"))) return st;
  if (c->k.dtype != c->v.dtype) return fail(SPARSED_ERR_DTYPE, "cache k and v have different dtypes");
  if (c->k.B != c->v.B || c->k.H != c->v.H || c->k.L != c->v.L || c->k.D != c->v.D)
    return fail(SPARSED_ERR_SHAPE, "cache k [%d,%d,%d,%d] and v [%d,%d,%d,%d] disagree", c->k.B, c->k.H, c->k.L, c->k.D, c->v.B, c->v.H, c->v.L,
                c->v.D);
  if (c->n_seqs < 0 || c->max_pages < 0) return fail(SPARSED_ERR_RANGE, "cache: %d sequences of at most %d pages", c->n_seqs, c->max_pages);
  if (c->n_seqs > kMaxTokens) return fail(SPARSED_ERR_UNSUPPORTED, "cache: %d sequences, the limit is 2^30", c->n_seqs);
  if (c->n_seqs > 0 && !c->seq_lens) return fail(SPARSED_ERR_NULL, "cache seq_lens is NULL");
  if (c->n_seqs > 0 && c->max_pages > 0 && !c->page_table) return fail(SPARSED_ERR_NULL, "cache page_table is NULL");
  if (c->n_seqs > 1 && c->table_stride < c->max_pages)
    return fail(SPARSED_ERR_STRIDE, "cache: rows of the page table are %lld entries apart and have %d", (long long)c->table_stride, c->max_pages);
  if ((int64_t)c->max_pages * c->k.L > kMaxTokens)
    return fail(SPARSED_ERR_UNSUPPORTED, "cache: %d pages of %d tokens a sequence, the limit is 2^30 tokens", c->max_pages, c->k.L);
  return SPARSED_OK;
}

sparsed_status check_mask_block(int32_t* mask_block) {
  if (*mask_block < 1) return fail(SPARSED_ERR_RANGE, "mask_block %d < 1", *mask_block);
  if (*mask_block > kMaxTokens) *mask_block = (int32_t)kMaxTokens;  // no sequence is longer: hides nothing either way
  return SPARSED_OK;
}

sparsed_status check_attended(int32_t n_seqs) {
  return n_seqs > kMaxAttendedSeqs ? fail(SPARSED_ERR_UNSUPPORTED, "%d sequences, the limit of an attention call is 2^16", n_seqs) : SPARSED_OK;
}

// q against the heads of k and against out
sparsed_status check_heads(const sparsed_tensor* q, const sparsed_tensor* k, const sparsed_tensor* out, const char* kname) {
  if (q->dtype != k->dtype) return fail(SPARSED_ERR_DTYPE, "q and %s have different dtypes", kname);
  if (q->D != k->D) return fail(SPARSED_ERR_SHAPE, "q has head dim %d, %s %d", q->D, kname, k->D);
  if (q->H % k->H != 0) return fail(SPARSED_ERR_SHAPE, "query heads %d not a multiple of %s heads %d", q->H, kname, k->H);
  if (!out) return SPARSED_OK;
  if (out->dtype != q->dtype) return fail(SPARSED_ERR_DTYPE, "out and q have different dtypes");
  Dim dims[] = {{out->L > 0 ? out->H : 0, out->stride_h}, {out->L, out->stride_l}};
  if (rows_overlap(out->D, dims))
    return fail(SPARSED_ERR_STRIDE, "out: rows overlap, heads %lld and tokens %lld elements apart", (long long)out->stride_h, (long long)out->stride_l);
  if (out->H != q->H || out->L != q->L || out->D != q->D) return fail(SPARSED_ERR_SHAPE, "out shape differs from q");
  return SPARSED_OK;
}

PackedArg packed(const sparsed_tensor* t, int unit = 1) {
  return PackedArg{t->data, t->H > 1 ? t->stride_h * unit : 0, t->L > 1 ? t->stride_l * unit : (int64_t)t->D * unit};
}
PagesArg pages(const sparsed_tensor* t, int unit = 1) {
  return PagesArg{t->data, t->B > 1 ? t->stride_b * unit : 0, t->H > 1 ? t->stride_h * unit : 0, t->stride_l * unit};
}
int page_shift(int page_size) { return __builtin_ctz((unsigned)page_size); }
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Where the parts of split rows lie in the workspace of a paged call.
struct PagedSpace {
  PagedShape shape;
  size_t stat, o, bytes;
};
PagedSpace paged_space(const sparsed_tensor* q, const sparsed_paged_cache* c, bool one_each) {
  PagedSpace w{};
  w.shape = paged_shape(q->dtype == SPARSED_BF16, q->L, c->n_seqs, q->H, c->k.H, one_each, (int64_t)c->max_pages * c->k.L);
  w.bytes = 256;
  if (w.shape.splits && q->L > 0) {
    w.stat = align256((size_t)q->L * q->H * 8);
    w.o = w.stat + align256((size_t)w.shape.parts * 8);
    w.bytes = w.o + align256((size_t)w.shape.parts * q->D * 4);
  }
  return w;
}

float scale_log2(int D) { return (float)(1.4426950408889634 / std::sqrt((double)D)); }

}  // namespace

extern "C" {

sparsed_status sparsed_cache_append(const sparsed_paged_cache* cache, const sparsed_tensor* k, const sparsed_tensor* v, const int32_t* cu,
                                    const sparsed_exec* ex) {
  sparsed_status st;
  if ((st = check_cache(cache)) || (st = check_packed(k, "k")) || (st = check_packed(v, "v"))) return st;
  if (k->dtype != cache->k.dtype || v->dtype != cache->k.dtype) return fail(SPARSED_ERR_DTYPE, "k, v and the cache have different dtypes");
  if (k->H != cache->k.H || v->H != cache->k.H || k->D != cache->k.D || v->D != cache->k.D || k->L != v->L)
    return fail(SPARSED_ERR_SHAPE, "k [%d,%d,%d], v [%d,%d,%d] and the cache (%d heads of %d) disagree", k->H, k->L, k->D, v->H, v->L, v->D,
                cache->k.H, cache->k.D);
  if (!cu && k->L != cache->n_seqs)
    return fail(SPARSED_ERR_SHAPE, "%d tokens for %d sequences: more or fewer than one each need cu", k->L, cache->n_seqs);
  for (const sparsed_tensor* t : {&cache->k, &cache->v}) {
    Dim dims[] = {{t->B, t->stride_b}, {t->H, t->stride_h}, {t->L, t->stride_l}};
    if (rows_overlap(t->D, dims))
      return fail(SPARSED_ERR_STRIDE, "cache %s: places overlap, pages %lld, heads %lld and tokens %lld elements apart", t == &cache->k ? "k" : "v",
                  (long long)t->stride_b, (long long)t->stride_h, (long long)t->stride_l);
  }
  if (k->L == 0 || cache->n_seqs == 0 || cache->max_pages == 0) return SPARSED_OK;
  AppendArgs a{};
  const int es = element_bytes(k);
  a.k = packed(k, es);
  a.v = packed(v, es);
  a.cu = cu;
  a.ck = pages(&cache->k, es);
  a.cv = pages(&cache->v, es);
  a.page_table = cache->page_table;
  a.seq_lens = cache->seq_lens;
  a.table_stride = cache->table_stride;
  a.n_seqs = cache->n_seqs;
  a.max_pages = cache->max_pages;
  a.n_pages = cache->k.B;
  a.page_shift = page_shift(cache->k.L);
  a.T = k->L;
  a.Hkv = k->H;
  a.row_bytes = k->D * es;
  const hipError_t e = launch_cache_append(a, stream_of(ex));
  if (e != hipSuccess) return hip_fail(e, "cache append launch");
  return SPARSED_OK;
}

sparsed_status sparsed_attn_prompt(const sparsed_tensor* q, const sparsed_tensor* k, const sparsed_tensor* v, sparsed_tensor* out,
                                   const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs, int32_t mask_block, const sparsed_exec* ex) {
  sparsed_status st;
  if ((st = check_packed(q, "q")) || (st = check_packed(k, "k")) || (st = check_packed(v, "v")) || (st = check_packed(out, "out"))) return st;
  if ((st = check_heads(q, k, out, "k")) || (st = check_heads(q, v, nullptr, "v"))) return st;
  if (k->H != v->H || k->L != v->L) return fail(SPARSED_ERR_SHAPE, "k [%d,%d,%d] and v [%d,%d,%d] disagree", k->H, k->L, k->D, v->H, v->L, v->D);
  if (n_seqs < 0) return fail(SPARSED_ERR_RANGE, "%d sequences", n_seqs);
  if ((st = check_attended(n_seqs))) return st;
  if ((st = check_mask_block(&mask_block))) return st;
  if (n_seqs > 0 && !cu_q) return fail(SPARSED_ERR_NULL, "cu_q is NULL");
  if (!cu_k && k->L != q->L) return fail(SPARSED_ERR_SHAPE, "q has %d tokens, k %d: different offsets need cu_k", q->L, k->L);
  if (q->L == 0 || n_seqs == 0) return SPARSED_OK;
  PromptArgs a{};
  a.q = packed(q);
  a.k = packed(k);
  a.v = packed(v);
  const PackedArg o = packed(out);
  a.o = out->data;
  a.o_sh = o.sh;
  a.o_sl = o.sl;
  a.lse = ex ? ex->lse_out : nullptr;
  a.cu_q = cu_q;
  a.cu_k = cu_k ? cu_k : cu_q;
  a.n_seqs = n_seqs;
  a.Tq = q->L;
  a.Tk = k->L;
  a.Hq = q->H;
  a.group = q->H / k->H;
  a.mask_block = mask_block;
  a.scale_log2 = scale_log2(q->D);
  const hipError_t e = q->dtype == SPARSED_BF16 ? launch_prompt_bf16(q->D, a, stream_of(ex)) : launch_prompt_f32(q->D, a, stream_of(ex));
  if (e == hipErrorInvalidConfiguration)
    return fail(SPARSED_ERR_UNSUPPORTED, "prompt attention: %d tokens of %d heads in %d sequences in one call", q->L, q->H, n_seqs);
  if (e != hipSuccess) return hip_fail(e, "prompt attention launch");
  return SPARSED_OK;
}

sparsed_status sparsed_attn_paged(const sparsed_tensor* q, const sparsed_paged_cache* cache, const int32_t* cu_q, int32_t mask_block,
                                  sparsed_tensor* out, const sparsed_exec* ex) {
  sparsed_status st;
  if ((st = check_packed(q, "q")) || (st = check_cache(cache)) || (st = check_packed(out, "out"))) return st;
  if ((st = check_heads(q, &cache->k, out, "cache")) || (st = check_attended(cache->n_seqs))) return st;
  if ((st = check_mask_block(&mask_block))) return st;
  if (!cu_q && q->L != cache->n_seqs)
    return fail(SPARSED_ERR_SHAPE, "%d tokens for %d sequences: more or fewer than one each need cu_q", q->L, cache->n_seqs);
  if (q->L == 0 || cache->n_seqs == 0) return SPARSED_OK;
  char* ws = nullptr;
  const PagedSpace space = paged_space(q, cache, cu_q == nullptr);
  if ((st = caller_workspace(ex, space.bytes, "paged attention", &ws))) return st;
  if (!grid_fits((int64_t)q->L * q->H, 256) || !grid_fits(space.shape.groups, 256) || space.shape.parts > 0x7fffffff)
    return fail(SPARSED_ERR_UNSUPPORTED, "paged attention: %d tokens of %d heads in one call", q->L, q->H);
  PagedArgs a{};
  a.q = packed(q);
  const PackedArg o = packed(out);
  a.o = out->data;
  a.o_sh = o.sh;
  a.o_sl = o.sl;
  a.lse = ex ? ex->lse_out : nullptr;
  a.cu_q = cu_q;
  a.k = pages(&cache->k);
  a.v = pages(&cache->v);
  a.page_table = cache->page_table;
  a.seq_lens = cache->seq_lens;
  a.table_stride = cache->table_stride;
  a.n_seqs = cache->n_seqs;
  a.max_pages = cache->max_pages;
  a.n_pages = cache->k.B;
  a.page_shift = page_shift(cache->k.L);
  a.Tq = q->L;
  a.Hq = q->H;
  a.group = q->H / cache->k.H;
  a.mask_block = mask_block;
  a.scale_log2 = scale_log2(q->D);
  if (space.shape.splits) {
    a.ws_desc = ws;
    a.ws_stat = ws + space.stat;
    a.ws_o = ws + space.o;
    a.ws_rows = space.shape.part_rows;
    a.ws_parts = space.shape.parts;
  }
  const hipError_t e = launch_attn_paged(q->dtype == SPARSED_BF16, q->D, a, space.shape, stream_of(ex));
  if (e != hipSuccess) return hip_fail(e, "paged attention launch");
  return SPARSED_OK;
}

size_t sparsed_paged_workspace_bytes(const sparsed_tensor* q, const sparsed_paged_cache* cache) {
  if (check_packed(q, "q") != SPARSED_OK || check_cache(cache) != SPARSED_OK || check_heads(q, &cache->k, nullptr, "cache") != SPARSED_OK ||
      check_attended(cache->n_seqs) != SPARSED_OK)
    return 0;
  // either way of the call: with offsets, and without where there is a token for every sequence
  const size_t with = paged_space(q, cache, false).bytes;
  const size_t without = q->L == cache->n_seqs ? paged_space(q, cache, true).bytes : 0;
  return with > without ? with : without;
}

sparsed_status sparsed_cache_validate(const sparsed_paged_cache* cache, const sparsed_exec* ex) {
  sparsed_status st;
  if ((st = check_cache(cache))) return st;
  char* ws = nullptr;
  if ((st = caller_workspace(ex, 256, "cache validation", &ws))) return st;
  if (cache->n_seqs == 0) return SPARSED_OK;
  hipStream_t s = stream_of(ex);
  int32_t* bad = reinterpret_cast<int32_t*>(ws);
  int32_t host_bad = 0;
  hipError_t e = hipMemsetAsync(bad, 0, sizeof(int32_t), s);
  if (e == hipSuccess) {
    CacheCheckArgs a{cache->page_table, cache->seq_lens, cache->table_stride, cache->n_seqs, cache->max_pages, cache->k.B, page_shift(cache->k.L), bad};
    e = launch_cache_check(a, s);
  }
  if (e == hipSuccess) e = hipMemcpyAsync(&host_bad, bad, sizeof(int32_t), hipMemcpyDeviceToHost, s);
  if (e == hipSuccess) e = hipStreamSynchronize(s);
  if (e != hipSuccess) return hip_fail(e, "cache validation");
  if (host_bad != 0) return fail(SPARSED_ERR_INDEX, "%d lengths or page numbers of the cache out of range", host_bad);
  return SPARSED_OK;
}

}  // extern "C"
