// Internal interface of the operators with a key/value cache: arguments of their kernels, what a kernel reads of a
// sequence, and the launchers. The host side is api_cache.hip; include/sparsed.h is the public boundary.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sparsed {

// A packed [T, H, D] array: element strides of head and token (stride of D is 1).
struct PackedArg {
  const void* ptr;
  int64_t sh, sl;
};
// Pages of tokens: element strides of page, head and token within a page.
struct PagesArg {
  const void* ptr;
  int64_t sp, sh, sl;
};

struct PromptArgs {
  PackedArg q, k, v;
  void* o;
  int64_t o_sh, o_sl;
  float* lse;              // optional [Hq, Tq], natural logarithm
  const int32_t *cu_q, *cu_k;
  int32_t n_seqs, Tq, Tk, Hq, group;
  int32_t mask_block;
  float scale_log2;        // log2(e) / sqrt(D)
};

struct PagedArgs {
  PackedArg q;
  void* o;
  int64_t o_sh, o_sl;
  float* lse;              // optional [Hq, Tq], natural logarithm
  const int32_t* cu_q;     // null: one token for every sequence
  PagesArg k, v;
  const int32_t* page_table;
  const int32_t* seq_lens;
  int64_t table_stride;
  int32_t n_seqs, max_pages, n_pages, page_shift;  // tokens per page = 1 << page_shift
  int32_t Tq, Hq, group;
  int32_t mask_block;
  float scale_log2;
  // parts of rows whose keys are split (PagedShape::splits, else null)
  void *ws_desc, *ws_stat, *ws_o;
  int32_t ws_rows;         // PagedShape::part_rows
  int64_t ws_parts;        // PagedShape::parts
};

// Launch of a paged call, from what the host knows.
struct PagedShape {
  int tile_rows;           // query rows of a work-group
  bool splits;             // whether keys may be split (some sequence may be long enough)
  int64_t groups;          // work-groups: at least the runs there can be
  int part_rows;           // rows of a run that parts are kept of
  int64_t parts;           // row parts there can be
};
PagedShape paged_shape(bool bf16, int64_t Tq, int64_t n_seqs, int64_t Hq, int64_t heads, bool one_each, int64_t max_tokens);

struct AppendArgs {
  PackedArg k, v;          // strides in BYTES here and in the pages
  const int32_t* cu;       // null: one token for every sequence
  PagesArg ck, cv;
  const int32_t* page_table;
  const int32_t* seq_lens;
  int64_t table_stride;
  int32_t n_seqs, max_pages, n_pages, page_shift;
  int32_t T, Hkv;
  int32_t row_bytes;       // of one head of one token
};

struct CacheCheckArgs {
  const int32_t* page_table;
  const int32_t* seq_lens;
  int64_t table_stride;
  int32_t n_seqs, max_pages, n_pages, page_shift;
  int32_t* bad;            // device counter of lengths and page numbers out of range
};

// Rows [begin, end) of sequence s of a packed array of T rows, offsets cut to it.
struct SeqRows {
  int begin, end;
};
__device__ __forceinline__ SeqRows cut_rows(int b, int e, int T) {
  b = b < 0 ? 0 : b > T ? T : b;
  e = e < b ? b : e > T ? T : e;
  return SeqRows{b, e};
}
__device__ __forceinline__ SeqRows seq_rows(const int32_t* cu, int s, int T) { return cut_rows(cu[s], cu[s + 1], T); }

// The sequence that holds row t: the last one whose first row is not behind it (offsets ascend), n_seqs if t is behind all.
__device__ __forceinline__ int seq_of_row(const int32_t* cu, int n_seqs, int t) {
  int lo = 0, hi = n_seqs;  // first s with cu[s + 1] > t
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Tokens of a sequence that count, cut to what its row of the page table can name.
__device__ __forceinline__ int cached_tokens(const int32_t* seq_lens, int s, int max_pages, int page_shift) {
  const int m = seq_lens[s], most = max_pages << page_shift;
  return m < 0 ? 0 : m > most ? most : m;
}

// Keys that the query at position p of a sequence of m tokens sees (m <= 2^30, mask_block <= 2^30: no overflow in 32 bits).
__device__ __forceinline__ int keys_seen(int p, int m, int mask_block) {
  if (p < 0) return 0;
  if (mask_block == 1) return p < m ? p + 1 : m;
  const uint32_t end = ((uint32_t)p / (uint32_t)mask_block + 1u) * (uint32_t)mask_block;
  return end < (uint32_t)m ? (int)end : m;
}

// A launch has fewer than 2^32 threads.
constexpr bool grid_fits(int64_t groups, int threads) { return groups > 0 && groups * threads < ((int64_t)1 << 32); }

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_cache_check(const CacheCheckArgs& a, hipStream_t s);
// Prompt calls of few rows (tokens times heads) leave the chip partly idle for the time of the longest row; those of very short
// sequences leave the tiles of the other forms mostly empty (the launchers below, with both sides measured).
inline bool few_rows(bool bf16, int D, const PromptArgs& a) {
  const int64_t rows = (int64_t)a.Tq * a.Hq, few = bf16 && D == 64 ? 28672 : 16384;
  return rows <= few || (rows <= (D == 64 ? 131072 : 65536) && a.Tq <= (int64_t)a.n_seqs * 8);
}

// Prompts: hipErrorInvalidConfiguration, and nothing is launched, where the grid would not fit.
hipError_t launch_prompt_bf16(int D, const PromptArgs& a, hipStream_t s);
hipError_t launch_prompt_few_rows_bf16(int D, const PromptArgs& a, hipStream_t s);  // attn_paged.hip
hipError_t launch_prompt_few_rows_f32(int D, const PromptArgs& a, hipStream_t s);   // attn_paged.hip
hipError_t launch_prompt_f32(int D, const PromptArgs& a, hipStream_t s);
hipError_t launch_attn_paged(bool bf16, int D, const PagedArgs& a, const PagedShape& shape, hipStream_t s);

}  // namespace sparsed
