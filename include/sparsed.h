/*
 * sparsed.h - C ABI of the MI355X (gfx950) SparseD attention library.
 *
 * SparseD (arXiv 2509.24014) runs full bidirectional attention for the early
 * denoising steps of a diffusion language model, selects one block-sparse
 * pattern per head at a switch step, and reuses it for every later step
 * (Section 3.3, Algorithm 1). The three calls of that algorithm are the three
 * compute entry points below. Beside them: attention of prompts and of newest
 * tokens with a paged key/value cache, for models that generate block by block.
 * Plain C11: no C++ or framework types cross this boundary.
 *
 * Conventions for every entry point
 *  - All tensor, index and workspace pointers are DEVICE pointers owned by the
 *    caller. The library never frees them and keeps no reference after a call
 *    returns. Descriptor structs themselves live in HOST memory.
 *  - Work is enqueued on `ex->stream` (a hipStream_t; NULL or ex == NULL means
 *    the default stream) and the call returns without synchronising, except
 *    where a function says it synchronises. The library allocates no device
 *    memory and keeps no state between calls except the thread-local error
 *    message: scratch memory is the caller's (`ex->workspace`), and a call that
 *    needs one and is given none returns SPARSED_ERR_WORKSPACE.
 *    sparsed_attn_dense, sparsed_attn_sparse and the selection entry points
 *    only launch kernels (no allocation, no memset, no copy), so they may be
 *    recorded into a HIP graph on a capturing stream.
 *  - Errors are returned as a sparsed_status; nothing throws or aborts. Every
 *    argument check happens before the first launch: on a status other than
 *    SPARSED_OK and SPARSED_ERR_HIP no kernel was launched and outputs are
 *    untouched. SPARSED_ERR_HIP reports a failed launch; the selection entry
 *    points launch several kernels in a row, so earlier ones of the same call
 *    may already be enqueued (they write only the workspace, pooled_out and
 *    the index). sparsed_last_error() gives a thread-local message.
 *  - Tensors are [B, H, L, D] views with arbitrary element strides for B, H, L
 *    and unit stride for D. `data` must be 16-byte aligned and every stride a
 *    multiple of 8 elements (bf16) or 4 elements (fp32), so that every row is
 *    16-byte aligned. One (batch, head) slab, (L-1)*stride_l + D elements, must
 *    span less than 2^31 bytes.
 *  - Grouped-query attention: q has Hq heads, k and v have Hkv heads with
 *    Hq % Hkv == 0; query head h reads key/value head h / (Hq / Hkv).
 *  - Supported shapes: D in {64, 128}; any L >= 1; block_q in {32, 64, 128};
 *    block_k in {32, 64, 128}; the paper's square settings 32 x 32 and 128 x 128
 *    are among them. L need not be a
 *    multiple of the block sizes: there are nqb = ceil(L / block_q) query blocks
 *    and nkb = ceil(L / block_k) key blocks, the last of each possibly partial
 *    (the paper pools with L // block_size and is silent on a remainder).
 *  - Arithmetic: bf16 tensors are multiplied on the bf16 matrix cores with
 *    fp32 accumulation, softmax in fp32, probabilities rounded to bf16 before
 *    the product with V. fp32 tensors: fp32 accumulation, fp32 softmax, products as
 *    good as fp32 ones; they run on the bf16 matrix cores with every operand as the sum
 *    of three bf16 parts, or on the fp32 matrix cores where the parts would not do
 *    (infinities, NaN, values beyond 3.3e38 or so small that their low parts would be
 *    cut off, about 2^-108).
 *    Pooled scores for selection are fp32 from the logits on, for either dtype.
 *  - A call repeated with the same arguments gives the same bits. How a row's keys are
 *    divided over the chip follows from B, H, L and the capacity of the index, and the
 *    order of its sums with it: a sample of a batch, or a head of several, may differ in
 *    rounding from the same sample or head alone.
 */
#ifndef SPARSED_H
#define SPARSED_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum sparsed_status {
  SPARSED_OK = 0,
  SPARSED_ERR_NULL = 1,        /* a required pointer is NULL */
  SPARSED_ERR_SHAPE = 2,       /* dimensions disagree or are not block multiples */
  SPARSED_ERR_DTYPE = 3,       /* unknown dtype or dtypes differ between tensors */
  SPARSED_ERR_STRIDE = 4,      /* misaligned pointer or stride */
  SPARSED_ERR_RANGE = 5,       /* rho outside (0, 1], negative size, ... */
  SPARSED_ERR_UNSUPPORTED = 6, /* head dim / block size the kernels do not cover */
  SPARSED_ERR_WORKSPACE = 7,   /* workspace missing or too small */
  SPARSED_ERR_INDEX = 8,       /* malformed block index or page table */
  SPARSED_ERR_HIP = 9          /* a HIP runtime call failed; see sparsed_last_error() */
} sparsed_status;

typedef enum sparsed_dtype { SPARSED_BF16 = 0, SPARSED_F32 = 1 } sparsed_dtype;

/* A [B, H, L, D] view of device memory. Strides are in elements. */
typedef struct sparsed_tensor {
  void* data;
  int32_t dtype; /* sparsed_dtype */
  int32_t B, H, L, D;
  int64_t stride_b, stride_h, stride_l;
} sparsed_tensor;

/*
 * The sparse pattern M_S of Eq. 4 stored as a per-head CSR over key blocks:
 * query block I of head (b, h) attends to key blocks
 *   col_idx[(b*H + h)*cap_per_head + t],  t in [row_ptr[(b*H+h)*(nqb+1) + I],
 *                                               row_ptr[(b*H+h)*(nqb+1) + I + 1])
 * i.e. offsets in row_ptr are local to the head's slab and row_ptr[.., 0] == 0.
 * Each row is strictly ascending. H is the number of QUERY heads. Rows may have
 * different lengths; an empty row makes that query block's output all zeros.
 */
typedef struct sparsed_block_index {
  int32_t B, H, nqb, nkb;
  int32_t block_q, block_k;
  int32_t cap_per_head; /* entries of col_idx reserved per (b, h) */
  int32_t* row_ptr;     /* device, [B, H, nqb + 1] */
  int32_t* col_idx;     /* device, [B, H, cap_per_head] */
} sparsed_block_index;

/* Optional execution context. A NULL context means: default stream, no extras. */
typedef struct sparsed_exec {
  void* stream;           /* hipStream_t */
  void* workspace;        /* device scratch for the selection calls, sparsed_attn_paged and the validation calls, 256-byte aligned */
  size_t workspace_bytes; /* its size */
  float* lse_out;         /* attn_dense: optional [B, Hq, L] fp32, log-sum-exp of each row's scaled logits (attn_prompt, attn_paged: [Hq, T]) */
  const float* lse_in;    /* select_pattern: optional [B, Hq, L] fp32 from attn_dense on the SAME q, k */
  float* pooled_out;      /* select_pattern: optional [B, Hq, nqb, nkb] fp32 copy of the pooled scores A' */
  const int32_t* seq_lens; /* optional DEVICE array [B]: per-sample lengths, see below */
} sparsed_exec;

/*
 * Per-sample lengths (not in the paper, whose runs use one length per call): with ex->seq_lens set,
 * batch element b has min(seq_lens[b], L) tokens; its rows and keys at or past that do not exist.
 *  - attn_dense / attn_sparse: those query rows are neither computed nor stored (out and lse_out keep
 *    what they held); keys past the length are masked.
 *  - select_pattern: sample b pools and ranks its own ceil(len / block_k) key blocks and keeps
 *    sparsed_kept_blocks(rho, that many) per query block: row_ptr[I] = I * k_b for its ceil(len / block_q)
 *    query blocks, and the query blocks it does not have get empty rows. pooled_out entries of blocks a
 *    sample does not have are not written. nqb, nkb and cap_per_head are still those of L.
 *  - select_pattern_isolated: the same with two ranges per sample, [0, min(prefill_blocks, its blocks)) and
 *    the rest of its blocks, each with its own count; a sample no longer than the prefill has one range.
 *  - select_pattern_isolated_tokens: the same with the boundary at a key token p; a sample longer than p
 *    splits the key block that holds p as described at that call (its generation part ends at the sample's
 *    length), a sample no longer than p has one range over its own blocks.
 *  - A length <= 0 makes the whole sample a no-op.
 */

/*
 * Full attention of the early denoising steps (Section 3.1, Eq. 1; Algorithm 1,
 * the "Skipping Sparse" branch):
 *     out[b,h,i,:] = sum_j softmax_j(q[b,h,i,:] . k[b,g,j,:] / sqrt(D)) * v[b,g,j,:]
 * over all j in [0, L), no causal mask. q, out: [B, Hq, L, D]; k, v: [B, Hkv, L, D].
 * If ex->lse_out is set it also receives log(sum_j exp(logit_ij)) per row.
 */
sparsed_status sparsed_attn_dense(const sparsed_tensor* q, const sparsed_tensor* k,
                                  const sparsed_tensor* v, sparsed_tensor* out,
                                  const sparsed_exec* ex);

/*
 * Pattern selection at the switch step (Section 3.3 "Isolated Selection" with a
 * single key range, Eq. 6; Algorithm 1, the per-query-block loop):
 *   1. A' = average of the softmax probabilities A of Eq. 1 over each
 *      block_q x block_k rectangle (each row of A normalised over all L keys;
 *      a partial last block is averaged over the entries that exist);
 *   2. for every query block keep the k = sparsed_kept_blocks(rho, nkb) key
 *      blocks with the largest A' (ties: lower block index), listed ascending.
 * The L x L matrix A is never formed. Fills out_block_index->row_ptr / col_idx
 * (every row has exactly k entries, row_ptr[I] = I*k); its B, H, nqb, nkb,
 * block_q, block_k must already describe q and the blocks and cap_per_head must
 * be >= nqb*k, else SPARSED_ERR_INDEX. Needs ex->workspace of at least
 * sparsed_select_workspace_min_bytes() bytes (SPARSED_ERR_WORKSPACE otherwise;
 * sparsed_select_workspace_bytes() lets it pool in one pass over the keys); the
 * workspace holds the row statistics and the pooled scores while the call's
 * kernels run, so calls that may overlap on the GPU need a workspace each.
 */
sparsed_status sparsed_select_pattern(const sparsed_tensor* q, const sparsed_tensor* k,
                                      int32_t block_q, int32_t block_k, double rho,
                                      sparsed_block_index* out_block_index,
                                      const sparsed_exec* ex);

/*
 * The switch step in one call (Algorithm 1 nests the selection under the full-attention branch): the dense
 * attention of sparsed_attn_dense and, from the same q and k, the pattern of sparsed_select_pattern. The attention
 * kernel leaves the pooled scores itself (its softmax already forms every block's row sums), so that Q K^T and the
 * exponentials are computed once instead of twice, but where two kernels are the quicker: bf16 calls with few query rows,
 * fp32 calls whose block sums do not fit the LDS or whose query blocks fill the chip badly. Same outputs
 * as the two calls up to fp32 summation order. Arguments and limits are those of the two calls; ex->lse_out and
 * ex->pooled_out are optional, ex->lse_in is ignored. Needs ex->workspace; sparsed_select_workspace_bytes()
 * always suffices.
 */
sparsed_status sparsed_attn_dense_select(const sparsed_tensor* q, const sparsed_tensor* k,
                                         const sparsed_tensor* v, sparsed_tensor* out,
                                         int32_t block_q, int32_t block_k, double rho,
                                         sparsed_block_index* out_block_index,
                                         const sparsed_exec* ex);

/*
 * sparsed_select_pattern for callers that cannot allocate device memory or bring a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * selection, same kernels and results, with the scratch (row statistics + pooled scores) in a
 * fixed array of SPARSED_STATIC_SCRATCH_BYTES that is part of the library's code object; each GPU
 * the library runs on holds its own copy until the process ends. ex->workspace is ignored;
 * ex->stream, lse_in, pooled_out and seq_lens work as in sparsed_select_pattern. The call
 * allocates and frees nothing (its first call on a device looks the array's device address up
 * once). Returns SPARSED_ERR_WORKSPACE when sparsed_select_workspace_min_bytes() for these arguments
 * (the _min_ form) exceeds SPARSED_STATIC_SCRATCH_BYTES (e.g. 32 heads of 65536 tokens with 128 x 64 blocks need
 * 75 MB; 32 heads of 16384 tokens with 64 x 64 blocks need 10 MB and fit). All calls on one GPU
 * share that GPU's array, which keeps the previous call's contents (every entry a call reads it
 * has written first): calls that may overlap on one GPU race, so keep them on one stream or
 * order them with events.
 */
#define SPARSED_STATIC_SCRATCH_BYTES ((size_t)32 << 20)
sparsed_status sparsed_select_pattern_static(const sparsed_tensor* q, const sparsed_tensor* k,
                                             int32_t block_q, int32_t block_k, double rho,
                                             sparsed_block_index* out_block_index,
                                             const sparsed_exec* ex);

/*
 * Sparse attention of the later steps ("Sparse Reusing"; Eq. 3 with the mask of
 * Eq. 4): rows of query block I attend only to the keys of the key blocks
 * listed for I (those below L, for a partial last block); the softmax is
 * normalised over those keys only. The index
 * contents are trusted (check them with sparsed_index_validate); its shape
 * fields are checked against q.
 */
sparsed_status sparsed_attn_sparse(const sparsed_tensor* q, const sparsed_tensor* k,
                                   const sparsed_tensor* v, const sparsed_block_index* block_index,
                                   sparsed_tensor* out, const sparsed_exec* ex);

/*
 * Isolated selection proper (Section 3.3, Eq. 5 and Eq. 6): key blocks
 * [0, prefill_blocks) and [prefill_blocks, nkb) are ranked separately, each
 * keeping sparsed_kept_blocks(rho, size of its range) blocks (none for an empty
 * range); a row is the ascending union. prefill_blocks == nkb or 0 gives the
 * same result as sparsed_select_pattern. cap_per_head must be >= nqb * (sum of
 * the two counts).
 */
sparsed_status sparsed_select_pattern_isolated(const sparsed_tensor* q, const sparsed_tensor* k,
                                               int32_t block_q, int32_t block_k, double rho,
                                               int32_t prefill_blocks,
                                               sparsed_block_index* out_block_index,
                                               const sparsed_exec* ex);

/*
 * Isolated selection with the boundary given as a key TOKEN (Eq. 5 splits the keys
 * into prefill tokens [0, prefill_tokens) and generation tokens [prefill_tokens, L)).
 * On a block edge this is sparsed_select_pattern_isolated. Otherwise the paper is
 * silent; reading: the key block that holds the boundary is pooled twice, over its
 * prefill keys and over its generation keys (each a mean over the entries that
 * exist), competes in both ranges with those scores, and is listed once if either
 * range keeps it. With n_pre = ceil(prefill_tokens / block_k) and n_gen = nkb -
 * floor(prefill_tokens / block_k), the ranges keep sparsed_kept_blocks(rho, n_pre)
 * and sparsed_kept_blocks(rho, n_gen) entries; a row has their sum or one fewer, so
 * row_ptr is not I*k here. cap_per_head must be >= nqb * (the sum). Workspace:
 * sparsed_select_tokens_workspace_bytes().
 */
sparsed_status sparsed_select_pattern_isolated_tokens(const sparsed_tensor* q, const sparsed_tensor* k,
                                                      int32_t block_q, int32_t block_k, double rho,
                                                      int32_t prefill_tokens,
                                                      sparsed_block_index* out_block_index,
                                                      const sparsed_exec* ex);

/*
 * Fixed pattern of the paper's sparse baselines (Section 4.1: sliding window, and
 * StreamingLLM = window + leading "sink" keys) written as a block index, so the
 * same sparse kernel runs them: query block I keeps every key block holding a
 * key j with |i - j| <= window_tokens/2 for one of its queries i (the window is
 * taken symmetric because attention here is bidirectional), plus the key blocks
 * that overlap the first sink_tokens keys. The same rows for every head; rows
 * have different lengths. idx->B, H, nqb, nkb, block_q, block_k must describe a
 * sequence of seq_len tokens (block counts rounded up); cap_per_head must be >=
 * sparsed_index_window_entries(...), else SPARSED_ERR_INDEX.
 */
sparsed_status sparsed_index_fill_window(sparsed_block_index* idx, int32_t seq_len, int32_t window_tokens,
                                         int32_t sink_tokens, const sparsed_exec* ex);

/* col_idx entries per head that sparsed_index_fill_window writes (-1 on bad arguments). Host only. */
int64_t sparsed_index_window_entries(int32_t seq_len, int32_t block_q, int32_t block_k, int32_t window_tokens,
                                     int32_t sink_tokens);

/* "Top rho%" of n blocks: ceil(rho*n - 1e-9) clamped to [1, n]; 0 if n <= 0. Host only. */
int32_t sparsed_kept_blocks(double rho, int32_t n);

/*
 * Number of full-attention steps of a T-step schedule with skip fraction `skip`
 * (Section 3.3 "Skipping Sparse"): clamp(ceil(T*skip - 1e-9), 1, T). Steps
 * 0 .. n-1 are dense, the pattern is selected at step n-1, steps n .. T-1 are
 * sparse. Host only.
 */
int32_t sparsed_n_dense_steps(int32_t T, double skip);

/*
 * Bytes of workspace the selection calls want for this q and these blocks (0 on bad arguments): the row statistics,
 * the pooled scores and, for bf16 inputs, the slabs of the one-pass pooled-score kernel that is used when no
 * ex->lse_in is handed over (128 x nkb floats for each of up to 1024 resident work-groups: 537 MB for 32
 * heads of 65536 tokens in 128 x 64 blocks). sparsed_select_workspace_min_bytes() is the part every call needs
 * (statistics + pooled scores, 75 MB in that example); with a workspace between the two, or with ex->lse_in set,
 * selection runs as row statistics (unless handed over) followed by pooled scores, two passes over the keys, with
 * the same results up to fp32 summation order.
 */
size_t sparsed_select_workspace_bytes(const sparsed_tensor* q, int32_t block_q, int32_t block_k);
size_t sparsed_select_workspace_min_bytes(const sparsed_tensor* q, int32_t block_q, int32_t block_k);

/* The same for sparsed_select_pattern_isolated_tokens (a little more: two extra pooled columns and row staging). */
size_t sparsed_select_tokens_workspace_bytes(const sparsed_tensor* q, int32_t block_q, int32_t block_k);

/*
 * Checks on the device that every row of the index is in range, strictly
 * ascending and within cap_per_head. SYNCHRONISES the stream. Returns
 * SPARSED_ERR_INDEX if any row is malformed. Needs ex->workspace of at least
 * 256 bytes (its first word counts the malformed rows).
 */
sparsed_status sparsed_index_validate(const sparsed_block_index* idx, const sparsed_exec* ex);

/*
 * ---- Attention with a key/value cache ------------------------------------------------------------
 *
 * Generation block by block (or token by token) keeps the keys and values of finished tokens: the prompt is attended to
 * once, its keys and values go into a cache, and every later step computes the newest tokens only. Sequences of different
 * length lie packed one behind the other, so none is padded.
 *
 * Packed tensors: a sparsed_tensor with B == 1 and L = all tokens, i.e. a [T, H, D] array with any strides for token
 * (stride_l) and head (stride_h); stride_b is not looked at, L may be 0, and the limit of 2^31 bytes per head does not
 * apply: (L - 1) * stride_l may be anything that fits 63 bits, 128 * stride_l elements must span less than 2^31 bytes.
 * Rows of an output, and places of a cache that sparsed_cache_append fills, must not share memory (strides are taken as nested, in
 * any order: SPARSED_ERR_STRIDE otherwise); what is only read may be expanded with strides of 0.
 * Sequence b has the rows cu[b] .. cu[b+1] - 1, cu being a DEVICE array of n_seqs + 1 ascending offsets from 0. Rows
 * at and behind cu[n_seqs] belong to no sequence: they are not read, and in outputs they keep what they held. Offsets below 0 or
 * beyond L count as 0 or L. Offsets have to ascend (equal ones are empty sequences): with one below its predecessor every access
 * stays within the tensors, but which rows of an output are written, and with what, is not specified.
 * An attention call takes up to 65536 sequences (SPARSED_ERR_UNSUPPORTED beyond): with many thousands its time is that of every
 * work-group looking for its own.
 *
 * Visibility: a sequence has m tokens, and a query at position p (0-based) of it sees the keys
 *     j < min(m, (p / mask_block + 1) * mask_block)
 * i.e. everything before the end of its own block of mask_block tokens. mask_block == 1 is causal attention, 32 that of
 * a model that denoises blocks of 32 tokens (each block in both directions, and all blocks before it), and any
 * mask_block >= m hides nothing. The n queries of a sequence are its last n tokens, at positions m - n .. m - 1;
 * a query at a negative position (n > m) sees nothing. A row that sees nothing is stored as zeros, its log-sum-exp as
 * -inf. Keys a row does not see have no influence on it, whatever K and V hold there (infinities and NaN included).
 *
 * Arithmetic is that of the other attention calls; fp32 products run on the fp32 matrix cores, and sparsed_attn_paged takes bf16
 * probabilities as the sum of two parts where T * Hq / Hkv <= 16 * n_seqs (one token each, and groups of up to 16 heads). A call
 * repeated with the same arguments and contents gives the same bits; how the keys of a row are divided, and the order of its sums with it, follows
 * from all lengths of the batch.
 */

/*
 * The cache of a batch of sequences: pages of page_size tokens, handed out by the caller. k and v describe the pages as
 * [B = number of pages, H = key/value heads, L = page_size, D] with strides stride_b (page), stride_h and stride_l, so
 * both [pages, page_size, H, D] and [pages, H, page_size, D] arrays are views; page_size is 16, 32, 64, 128 or 256.
 * Token i of sequence s is token i % page_size of page page_table[s * table_stride + i / page_size]. seq_lens[s] tokens
 * of it count, the newest of a step among them; lengths are cut to [0, max_pages * page_size]. A page number
 * outside [0, number of pages) is read as the nearest valid page and never written (sparsed_cache_validate finds it).
 */
typedef struct sparsed_paged_cache {
  sparsed_tensor k, v;
  const int32_t* page_table; /* device, n_seqs rows of at least max_pages entries */
  const int32_t* seq_lens;   /* device, [n_seqs] */
  int32_t n_seqs, max_pages;
  int64_t table_stride;      /* entries between the rows of page_table */
} sparsed_paged_cache;

/*
 * Puts the keys and values of new tokens into the cache. k, v: packed [1, Hkv, T, D]; the rows of sequence s are its
 * last tokens: row cu[s] + i goes to position seq_lens[s] - (cu[s+1] - cu[s]) + i (seq_lens already counts
 * them). cu == NULL: one token for every sequence (T == n_seqs). Tokens at negative positions are dropped, and so are those
 * that a length beyond max_pages * page_size puts behind the last page (lengths are not cut here). Two tokens for one place of
 * the cache (pages that sequences share) leave one of them. Only launches a kernel.
 */
sparsed_status sparsed_cache_append(const sparsed_paged_cache* cache, const sparsed_tensor* k, const sparsed_tensor* v,
                                    const int32_t* cu, const sparsed_exec* ex);

/*
 * Attention of packed prompts: q, out packed [1, Hq, T, D]; k, v packed [1, Hkv, Tk, D]. Sequence s has the queries
 * cu_q[s] .. cu_q[s+1] - 1 and the keys cu_k[s] .. cu_k[s+1] - 1 (cu_k == NULL: cu_q, and Tk == T); its queries are the
 * last tokens of its keys (see Visibility). ex->lse_out, optional, [Hq, T] fp32, receives each row's log-sum-exp. The keys of a
 * row are not divided over the chip: a few queries over many keys (one of 28/4 heads over 65536: 571 us) are work for
 * sparsed_attn_paged (29 us), for which packed keys whose sequences begin at multiples of a page size are pages as they lie.
 * Only launches a kernel.
 */
sparsed_status sparsed_attn_prompt(const sparsed_tensor* q, const sparsed_tensor* k, const sparsed_tensor* v,
                                   sparsed_tensor* out, const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs,
                                   int32_t mask_block, const sparsed_exec* ex);

/*
 * Attention of the newest tokens of every sequence over its cache (which holds their own keys and values already:
 * sparsed_cache_append). q, out packed [1, Hq, T, D]; cu_q as above, cu_q == NULL: one token for every sequence
 * (T == n_seqs). Made for one to a few dozen tokens a sequence; any number is computed. Long caches are split over the
 * chip and the parts joined (T * Hq < 2^24): needs ex->workspace of sparsed_paged_workspace_bytes() (held while the call's kernels run, so
 * calls that may overlap need one each). ex->lse_out as for prompts. Only launches kernels.
 */
sparsed_status sparsed_attn_paged(const sparsed_tensor* q, const sparsed_paged_cache* cache, const int32_t* cu_q,
                                  int32_t mask_block, sparsed_tensor* out, const sparsed_exec* ex);

/* Bytes of workspace sparsed_attn_paged needs for this q and cache (0 on bad arguments). Host only. */
size_t sparsed_paged_workspace_bytes(const sparsed_tensor* q, const sparsed_paged_cache* cache);

/*
 * Checks on the device that every length is within [0, max_pages * page_size] and every page that a length needs within
 * the cache. SYNCHRONISES the stream. Returns SPARSED_ERR_INDEX if one is not. Needs ex->workspace of at least 256 bytes.
 */
sparsed_status sparsed_cache_validate(const sparsed_paged_cache* cache, const sparsed_exec* ex);

const char* sparsed_status_string(sparsed_status s);
const char* sparsed_last_error(void); /* thread-local, never NULL */
int32_t sparsed_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SPARSED_H */
