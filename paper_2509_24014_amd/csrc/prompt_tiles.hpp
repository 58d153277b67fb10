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
__device__ __forceinline__ int wave_max_int(int x) {  // of values from 0 on
#define SPARSED_MAX_STEP(CTRL, ROWS) { const int y = __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); x = x > y ? x : y; }
  SPARSED_MAX_STEP(0x111, 0xf)
  SPARSED_MAX_STEP(0x112, 0xf)
  SPARSED_MAX_STEP(0x114, 0xf)
  SPARSED_MAX_STEP(0x118, 0xf)
  SPARSED_MAX_STEP(0x142, 0xa)
  SPARSED_MAX_STEP(0x143, 0xc)
#undef SPARSED_MAX_STEP
  return __builtin_amdgcn_readlane(x, 63);
}

// Place `pos` in the order: tiles with the highest number first, sequences in their order among equals.
//
// The tiles of the first 512 sequences are held in registers, 64 a register: the search below sums them once a step. Sequences of one
// tile need no step. (256 sequences of 64 tokens, 32 heads of 128, 256 rows a tile, us: 395 with the offsets read again in each of
// as many steps as all tokens would need, 247 like this.)
template <int QT, typename Args>
__device__ __forceinline__ PromptTile find_tile(Args& a, int pos, int lane) {
  constexpr int kHeld = 8;
  // the first 64 sequences, a lane each: their offsets are read once
  SeqRows q = {0, 0}, k = {0, 0};
  if (lane < a.n_seqs) {
    q = seq_rows(a.cu_q, lane, a.Tq);
    k = seq_rows(a.cu_k, lane, a.Tk);
  }
  auto place = [&](int s, int tile) {
    if (s < 64) {
      auto at = [&](int v) { return __builtin_amdgcn_readlane(v, s); };
      return PromptTile{s, tile, {at(q.begin), at(q.end)}, {at(k.begin), at(k.end)}};
    }
    return PromptTile{s, tile, seq_rows(a.cu_q, s, a.Tq), seq_rows(a.cu_k, s, a.Tk)};
  };
  const PromptTile none = {-1, 0, {0, 0}, {0, 0}};
  int held[kHeld];
  held[0] = tiles_in<QT>(q);
  if (a.n_seqs == 1) {
    const int all = __builtin_amdgcn_readfirstlane(held[0]);
    return pos < all ? place(0, all - 1 - pos) : none;
  }
  const bool many = a.n_seqs > 64;
#pragma unroll
  for (int c = 1; c < kHeld; ++c) held[c] = 0;
  if (many) {
    int cu[2][kHeld];                     // loads that wait for none of the others; behind the last sequence its end, twice
#pragma unroll
    for (int c = 1; c < kHeld; ++c) {
      const int s = 64 * c + lane;
      cu[0][c] = a.cu_q[s < a.n_seqs ? s : a.n_seqs];
      cu[1][c] = a.cu_q[s < a.n_seqs ? s + 1 : a.n_seqs];
    }
#pragma unroll
    for (int c = 1; c < kHeld; ++c) held[c] = tiles_in<QT>(cut_rows(cu[0][c], cu[1][c], a.Tq));
  }
  auto each = [&](auto&& f) {             // f of every lane's tiles, 64 sequences after the other
    f(held[0]);
    if (many) {
#pragma unroll
      for (int c = 1; c < kHeld; ++c) f(held[c]);
      for (int s = 64 * kHeld + lane; s - lane < a.n_seqs; s += 64) f(tiles_of<QT>(a, s));
    }
  };
  int sum = 0, most = 0;
  each([&](int n) {
    sum += n;
    most = most > n ? most : n;
  });
  if (pos >= wave_sum_int(sum)) return none;
  // tiles whose number is at least j: more than pos for j = lo; for j = hi `behind`, not more
  int lo = 0, hi = wave_max_int(most), behind = 0;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    sum = 0;
    each([&](int n) { sum += n > mid ? n - mid : 0; });
    sum = wave_sum_int(sum);
    if (sum > pos) {
      lo = mid;
    } else {
      hi = mid;
      behind = sum;
    }
  }
  // the sequence: number `rank` among those that have a tile number lo
  int rank = pos - behind, s0 = 0, found = -1;
  each([&](int n) {
    const uint64_t has = __builtin_amdgcn_ballot_w64(n > lo);
    const int count = __builtin_popcountll(has);
    if (found < 0 && rank < count) {
      const int before = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0));
      found = s0 + __builtin_ctzll(__builtin_amdgcn_ballot_w64(n > lo && before == rank));
    }
    rank -= count;
    s0 += 64;
  });
  return found < 0 ? none : place(found, lo);
}

}  // namespace sparsed
