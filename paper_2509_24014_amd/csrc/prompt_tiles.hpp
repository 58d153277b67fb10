// Which query rows a work-group of a prompt call takes. The host knows how many rows there are in all but not how they are
// divided among the sequences: it launches as many work-groups as there can be tiles, and each finds its own.
#pragma once
#include "cache.hpp"

namespace sparsed {

struct PromptTile {
  int s;      // sequence, or -1: none
  int tile;   // of its rows
  SeqRows q, k;
};

template <int QT>
__device__ __forceinline__ int tiles_in(const SeqRows& r) {
  return (r.end - r.begin + QT - 1) / QT;
}
template <int QT, typename Args>
__device__ __forceinline__ int tiles_of(Args& a, int s) {
  return s < a.n_seqs ? tiles_in<QT>(seq_rows(a.cu_q, s, a.Tq)) : 0;
}
__device__ __forceinline__ int wave_sum_int(int x) {
#define SPARSED_SUM_STEP(CTRL, ROWS) x += __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
  SPARSED_SUM_STEP(0x111, 0xf)  // row_shr:1
  SPARSED_SUM_STEP(0x112, 0xf)
  SPARSED_SUM_STEP(0x114, 0xf)
  SPARSED_SUM_STEP(0x118, 0xf)
  SPARSED_SUM_STEP(0x142, 0xa)  // row_bcast:15
  SPARSED_SUM_STEP(0x143, 0xc)  // row_bcast:31
#undef SPARSED_SUM_STEP
  return __builtin_amdgcn_readlane(x, 63);
}

// Place `pos` in the order: tiles with the highest number first, sequences in their order among equals.
template <int QT, typename Args>
__device__ __forceinline__ PromptTile find_tile(Args& a, int pos, int lane) {
  // the first 64 sequences, a lane each: their offsets are read once
  SeqRows q = {0, 0}, k = {0, 0};
  if (lane < a.n_seqs) {
    q = seq_rows(a.cu_q, lane, a.Tq);
    k = seq_rows(a.cu_k, lane, a.Tk);
  }
  const int first = tiles_in<QT>(q);
  auto place = [&](int s, int tile) {
    if (s < 64) {
      auto at = [&](int v) { return __builtin_amdgcn_readlane(v, s); };
      return PromptTile{s, tile, {at(q.begin), at(q.end)}, {at(k.begin), at(k.end)}};
    }
    return PromptTile{s, tile, seq_rows(a.cu_q, s, a.Tq), seq_rows(a.cu_k, s, a.Tk)};
  };
  const PromptTile none = {-1, 0, {0, 0}, {0, 0}};
  // tiles whose number is at least j
  auto at_least = [&](int j) -> int {
    int sum = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
      const int n = s0 == 0 ? first : tiles_of<QT>(a, s0 + lane);
      sum += wave_sum_int(n > j ? n - j : 0);
    }
    return sum;
  };
  const int all = at_least(0);
  if (pos >= all) return none;
  if (a.n_seqs == 1) return place(0, all - 1 - pos);
  int lo = 0, hi = (a.Tq + QT - 1) / QT;  // at_least(lo) > pos >= at_least(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at_least(mid) > pos) lo = mid;
    else hi = mid;
  }
  int rank = pos - at_least(hi);          // among the sequences that have a tile number lo
  for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
    const int n = s0 == 0 ? first : tiles_of<QT>(a, s0 + lane);
    const uint64_t has = __builtin_amdgcn_ballot_w64(n > lo);
    const int count = __builtin_popcountll(has);
    if (rank < count) {
      const int before = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0));
      return place(s0 + __builtin_ctzll(__builtin_amdgcn_ballot_w64(n > lo && before == rank)), lo);
    }
    rank -= count;
  }
  return none;
}

}  // namespace sparsed
