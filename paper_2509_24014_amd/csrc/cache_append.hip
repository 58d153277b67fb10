// Keys and values of new tokens into the pages of their sequences, and the check of a page table.
#include "cache.hpp"

namespace sparsed {

typedef __attribute__((ext_vector_type(4))) uint32_t Piece;

// STREAM: past the caches, for calls whose keys and values would not stay in them (launch_cache_append).
template <bool STREAM>
__device__ __forceinline__ void copy_piece(const void* from, void* to) {
  if constexpr (STREAM) __builtin_nontemporal_store(__builtin_nontemporal_load(static_cast<const Piece*>(from)), static_cast<Piece*>(to));
  else *static_cast<Piece*>(to) = *static_cast<const Piece*>(from);
}

// One thread moves 16 bytes; a work-group takes whole tokens (K and V, every head), one behind the other.
// Nothing is computed: the bound is memory, every byte read once and written once. 393 us for the K and V of 57000 tokens of 32 heads of
// 128 in bf16 = 4.7 TB/s both ways, as a copy of 4 GiB. With one token each of a few sequences the call is its launch.
template <bool STREAM>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendArgs a) {
  const int per_row = a.row_bytes >> 4;                  // 16-byte pieces of one head of one token: 8, 16 or 32
  const int per_token = a.Hkv * per_row;
  const int64_t total = (int64_t)a.T * per_token;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int t = (int)(i / per_token), rest = (int)(i % per_token), h = rest / per_row, c = rest % per_row;
    int s = t, behind = 1;          // tokens of the sequence from this one on
    if (a.cu != nullptr) {
      s = seq_of_row(a.cu, a.n_seqs, t);
      if (s >= a.n_seqs) continue;  // behind the last sequence
      const SeqRows r = seq_rows(a.cu, s, a.T);
      if (t < r.begin) continue;    // before the first
      behind = r.end - t;
    }
    // by the length as it is: cut to the table first, tokens that have no place would take those of older ones
    const int64_t at = (int64_t)a.seq_lens[s] - behind;
    if (at < 0 || at >= (int64_t)a.max_pages << a.page_shift) continue;
    const int pos = (int)at;
    const int page = a.page_table[s * a.table_stride + (pos >> a.page_shift)];
    if (page < 0 || page >= a.n_pages) continue;
    const int slot = pos & ((1 << a.page_shift) - 1);
    const char* from_k = static_cast<const char*>(a.k.ptr) + t * a.k.sl + h * a.k.sh + 16 * c;
    const char* from_v = static_cast<const char*>(a.v.ptr) + t * a.v.sl + h * a.v.sh + 16 * c;
    char* to_k = static_cast<char*>(const_cast<void*>(a.ck.ptr)) + page * a.ck.sp + h * a.ck.sh + slot * a.ck.sl + 16 * c;
    char* to_v = static_cast<char*>(const_cast<void*>(a.cv.ptr)) + page * a.cv.sp + h * a.cv.sh + slot * a.cv.sl + 16 * c;
    copy_piece<STREAM>(from_k, to_k);
    copy_piece<STREAM>(from_v, to_v);
  }
}

// From 64 MB of keys and values on, what is read and written takes half and more of the 256 MB behind the L2 caches. us,
// through the caches -> past them, bf16, 8 heads of 128: 6000 tokens (25 MB) 10.3 -> 11.7, 10000 (41 MB) 14.6 -> 17.7, 16000 (66 MB)
// 28.3 -> 26.2, 28000 46.1 -> 43.2; 56851 tokens of 32 heads (1.9 GB in all) 407 -> 393.
hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s) {
  const int64_t total = (int64_t)a.T * a.Hkv * (a.row_bytes >> 4);
  const int64_t groups = (total + 255) / 256;
  const dim3 grid((unsigned)(groups < 65536 ? groups : 65536)), block(256);
  if (total * 32 >= ((int64_t)64 << 20)) hipLaunchKernelGGL(cache_append_kernel<true>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(cache_append_kernel<false>, grid, block, 0, s, a);
  return hipGetLastError();
}

// A work-group per sequence, and as many further ones as there are: any number of sequences is a launch that fits.
__global__ __launch_bounds__(256) void cache_check_kernel(const CacheCheckArgs a) {
  int bad = 0;
  for (int64_t s = blockIdx.x; s < a.n_seqs; s += gridDim.x) {
    const int m = a.seq_lens[s];
    if (m < 0 || m > (int64_t)a.max_pages << a.page_shift) {
      bad += threadIdx.x == 0;
    } else {
      const int pages = (int)(((int64_t)m + (1 << a.page_shift) - 1) >> a.page_shift);
      for (int i = threadIdx.x; i < pages; i += 256) {
        const int p = a.page_table[s * a.table_stride + i];
        bad += p < 0 || p >= a.n_pages;
      }
    }
  }
  if (bad) atomicAdd(a.bad, bad);
}

hipError_t launch_cache_check(const CacheCheckArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(cache_check_kernel, dim3((unsigned)(a.n_seqs < 65536 ? a.n_seqs : 65536)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace sparsed
