// Attention of the newest tokens of every sequence over its paged cache (gfx950).
//
// The rows that share keys, `group` query heads of a sequence's new tokens for one key/value head, are few: the work is to
// read K and V once, as fast as memory gives them. A work-group of four waves takes one run of keys of one row tile (16 or 32
// rows); its waves take sub-tiles of 32 (fp32: 16) keys in turn and share nothing until the run ends, so the loop has no
// barrier. A wave asks for the next sub-tile's K when it has formed the logits of this one, and for its V when it has added
// this one's: 16 KB a wave (two heads' rows of 128 columns, bf16), 64 KB a work-group, two of which share a compute unit (of 64 columns,
// four). Measured, with the join, one token a sequence, heads of 128: 32 sequences of 500-8000, 32/32 heads, pages of 16: 327 us = 5.6 TB/s of
// cache; one of 65536, 28/4 heads: 31.6 us (24 the runs, 4.7 the join, the rest between them); 32 new tokens each of four
// sequences, 32/32 heads: 79.5 us; in fp32, 32/8 heads, one of 65536: 101 us = 5.3 TB/s, 32 of 4000: 175 us = 6.0.
//
// Prompts of few rows take the same kernels (launch_prompt_few_rows_*): a run is a row tile, K and V lie packed.
//
// Formulation, as in the dense kernels: logits transposed, S^T = K Q^T with 16 x 16 matrix tiles, so a lane holds one query
// (column lane % 16) and four keys of each 16-key half; O^T += V^T P^T takes these as they are as its B operand, which fixes
// the order in which keys enter the product (slot 8 g + 4 half + r of lane group g is key 16 half + 4 g + r).
//
// Softmax is online. The reference M of a query moves only when a logit exceeds it by more than 8 octaves, so that no
// exchange between lanes and no rescaling happens in most steps: probabilities are at most 2^8 times a sum that holds them.
//
// Hidden keys. Their logits become -inf, their probabilities 0; but 0 times what V holds there (an unused place of a page, a later
// token's infinity) is 0 only if that is finite. Places that no row of the tile sees are zeroed (bf16: in LDS), and
// where infinities or NaN lie among the keys that some rows see and others do not, the product is formed for every bound
// among the rows, from V zeroed behind that bound, and taken by the rows that have it.
//
// Long runs are split over the chip and joined by a second kernel. Runs are worked out on the device from the
// lengths there (the host does not know them): total work gives the run length (run_units), each work-group finds its own.
#include "cache.hpp"
#include "kernels.hpp"
#include "tile_bf16.hpp"

namespace sparsed {

typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kUnit = 128;          // keys a run is a multiple of: a sub-tile of every wave, or two
// Units of a run, for `work` units of all row tiles. Up to 8 by one run a compute unit: a unit is a trip to memory for its waves,
// 0.95 us, while a work-group has about that much of its own to do beside it; and from there on up to 4096 runs, which even out what
// the lengths of a batch leave. One token, us, by least units of a run (1, 2, 4, 8): 28/4 heads of 128 over 1024 tokens 9.7, 11.1,
// 13.1, 15.3; 8192 11.5, 12.8, 14.2, 18.2; 16384 14.5, 14.0, 15.2, 19.1; 65536 (2, 4, 8) 34.5, 32.3, 31.3; 32/32 heads over 4096
// tokens 19.2, 18.4, 18.2, 18.9. 32 sequences of 500-8000, by most runs (512, 1024, 2048, 4096): 367, 360, 341, 340.
constexpr int kMaxRuns = 4096;
__device__ __forceinline__ int run_units(float work) {
  const int few = (int)((work + 255.f) * (1.f / 256)), many = (int)(work * (1.f / kMaxRuns)) + 1;
  return few > 8 ? (many > 8 ? many : 8) : few > 1 ? few : 1;
}
// Sequences up to so many units are not split: joining takes 2.5 us (28/4 heads over 300 tokens: 7.6 us whole, 9.7 in three runs).
constexpr int kWholeUnits = 4;
constexpr float kNoReference = -3e38f;
constexpr float kSlack = 8.f;       // octaves a logit may lie above its reference

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// ---- which run of which row tile -----------------------------------------------------------------

struct SeqWork {  // one sequence, one key/value head
  int q0, n;      // its first row of q, its rows
  int k0, m;      // its first row of packed keys, its keys
  int tiles;      // row tiles
  int units;      // of keys
};

__device__ __forceinline__ int wave_scan(int x) {  // inclusive sum over the lanes up to this one
#define SPARSED_SCAN_STEP(CTRL, ROWS) x += __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
  SPARSED_SCAN_STEP(0x111, 0xf)  // row_shr:1
  SPARSED_SCAN_STEP(0x112, 0xf)
  SPARSED_SCAN_STEP(0x114, 0xf)
  SPARSED_SCAN_STEP(0x118, 0xf)
  SPARSED_SCAN_STEP(0x142, 0xa)  // row_bcast:15
  SPARSED_SCAN_STEP(0x143, 0xc)  // row_bcast:31
#undef SPARSED_SCAN_STEP
  return x;
}

// Rows of q and keys of a sequence, in pages or packed.
template <typename Args>
constexpr bool in_pages = __is_same(Args, PagedArgs);
template <int ROWS, typename Args>
__device__ __forceinline__ SeqWork seq_work(const Args& a, int number) {
  SeqWork w = {0, 0, 0, 0, 0, 0};
  const int s = number < a.n_seqs ? number : a.n_seqs - 1;  // (no branch: loads of several calls wait for none of the others)
  w.q0 = s;
  w.n = 1;
  if (!in_pages<Args> || a.cu_q != nullptr) {
    const SeqRows r = seq_rows(a.cu_q, s, a.Tq);
    w.q0 = r.begin;
    w.n = r.end - r.begin;
  }
  if constexpr (in_pages<Args>) {
    w.m = cached_tokens(a.seq_lens, s, a.max_pages, a.page_shift);
  } else {
    const SeqRows r = seq_rows(a.cu_k, s, a.Tk);
    w.k0 = r.begin;
    w.m = r.end - r.begin;
  }
  w.tiles = number < a.n_seqs ? (w.n * a.group + ROWS - 1) / ROWS : 0;
  w.units = (w.m + kUnit - 1) / kUnit;
  return w;
}

struct Run {
  int s;              // sequence, or -1: none
  int q0, n, k0, m;   // of it, as in SeqWork
  int tile;           // row tile
  int part, parts;    // which of how many runs
  int begin, end;     // units of keys
  int slot;           // of part 0 of this tile (parts > 1), in runs of one head
};

// Run number i of the launch. Every wave works it out for itself, a lane a sequence: 64 at a time, the first 256 of them read once.
// Prompts are not split: a run is a row tile. (One token each of 256 sequences of 100-300, 28/4 heads: 26.9 us, 29.5 with the lengths read 64 by
// 64; of 600, 68 and 80.)
template <int ROWS, typename Args>
__device__ __forceinline__ Run find_run(const Args& a, int i, int lane) {
  constexpr int kHeld = 4;
  const bool many = a.n_seqs > 64;
  SeqWork held[kHeld];
  held[0] = seq_work<ROWS>(a, lane);
#pragma unroll
  for (int c = 1; c < kHeld; ++c) held[c] = SeqWork{0, 0, 0, 0, 0, 0};
  if (many) {
#pragma unroll
    for (int c = 1; c < kHeld; ++c) held[c] = seq_work<ROWS>(a, 64 * c + lane);
  }
  int run = 0x40000000;
  if constexpr (in_pages<Args>) {
    auto of = [](const SeqWork& w) { return (float)w.tiles * (float)w.units; };
    float work = of(held[0]);  // in units: a float is exact enough to choose a run length by, and the same in every wave
    if (many) {
#pragma unroll
      for (int c = 1; c < kHeld; ++c) work += of(held[c]);
      for (int s0 = 64 * kHeld; s0 < a.n_seqs; s0 += 64) work += of(seq_work<ROWS>(a, s0 + lane));
    }
    run = __builtin_amdgcn_readfirstlane(run_units(wave_sum(work) * (float)(a.Hq / a.group)));
  }
  Run r = {-1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  int base = 0, slots = 0;
  auto look = [&](const SeqWork& w, int s0) -> bool {  // whether it is one of a sequence from s0 on
    const int parts = in_pages<Args> && w.units > kWholeUnits ? (int)(((unsigned)w.units + run - 1) / (unsigned)run) : 1;
    const int count = w.tiles * parts, mine = parts > 1 ? count : 0;
    const int upto = wave_scan(count), slots_upto = wave_scan(mine);
    const uint64_t behind = __builtin_amdgcn_ballot_w64(base + upto > i);
    if (behind != 0) {
      const int l = __builtin_ctzll(behind);
      auto at = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      const int tiles = at(w.tiles), n_parts = at(parts), units = at(w.units), in = i - (base + at(upto - count));
      if ((unsigned)in >= (unsigned)at(count)) return true;  // (sums that wrapped: offsets that overlap name more rows than there are)
      // (wave-uniform, but divided in vector registers)
      const int part = __builtin_amdgcn_readfirstlane(in / tiles), tile = in - part * tiles;
      const int each = __builtin_amdgcn_readfirstlane((units + n_parts - 1) / n_parts);
      const int end = (part + 1) * each;
      r = Run{s0 + l, at(w.q0), at(w.n), at(w.k0), at(w.m), tile, part, n_parts, part * each, end < units ? end : units,
              slots + at(slots_upto - mine) + tile * n_parts};
      return true;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
    slots += __builtin_amdgcn_readlane(slots_upto, 63);
    return false;
  };
  if (look(held[0], 0) || !many) return r;
#pragma unroll
  for (int c = 1; c < kHeld; ++c)
    if (look(held[c], 64 * c)) return r;
  for (int s0 = 64 * kHeld; s0 < a.n_seqs; s0 += 64)
    if (look(seq_work<ROWS>(a, s0 + lane), s0)) return r;
  return r;
}

// ---- the rows of a tile ----------------------------------------------------------------------------

struct TileRows {
  int q0, n, m;        // first row of the sequence in q, its new tokens, its tokens
  int R, r0;           // rows of this key/value head, first one of the tile
  int least, most;     // keys that the first and the last row of the tile see
};

template <int ROWS, typename Args>
__device__ __forceinline__ TileRows tile_rows(const Args& a, const Run& run) {
  TileRows t;
  t.q0 = run.q0;
  t.n = run.n;
  t.m = run.m;
  t.R = t.n * a.group;
  t.r0 = run.tile * ROWS;
  const int last = t.r0 + ROWS < t.R ? t.r0 + ROWS - 1 : t.R - 1;
  t.least = __builtin_amdgcn_readfirstlane(keys_seen(t.m - t.n + t.r0 / a.group, t.m, a.mask_block));
  t.most = __builtin_amdgcn_readfirstlane(keys_seen(t.m - t.n + last / a.group, t.m, a.mask_block));
  return t;
}

// The page of a key of sequence s.
__device__ __forceinline__ int page_of(const PagedArgs& a, int s, int key) {
  const int page = a.page_table[s * a.table_stride + (key >> a.page_shift)];
  return page < 0 ? 0 : page >= a.n_pages ? a.n_pages - 1 : page;
}

// Four lanes, one of each group of 16, share a query.
__device__ __forceinline__ float quad_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// ---- the end of a run: the waves' parts merged, the result or the run's part stored ----------------

struct PartsOut {  // in the workspace
  int2* desc;      // [Tq * Hq]: first element (below) of a row's parts, and their number
  float2* stat;    // per element: reference, sum
  float* o;        // per element: D unnormalised columns
  int rows;        // elements of a run of one head
};
__device__ __forceinline__ PartsOut parts_out(const PagedArgs& a) {
  return PartsOut{static_cast<int2*>(a.ws_desc), static_cast<float2*>(a.ws_stat), static_cast<float*>(a.ws_o), a.ws_rows};
}

template <typename T>
__device__ __forceinline__ void store_four(T* to, f32x4 x) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(to) = x;
  } else {
    const f32x2 lo = {x[0], x[1]}, hi = {x[2], x[3]};
    u32x2 w;
    w[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2));
    *reinterpret_cast<u32x2*>(to) = w;
  }
}

// 16 rows of the tile, those from row r on: `stage` holds 16 x D floats of every wave, 16-byte slot c of row n at c ^ n;
// ref, sum: [4][16] of the waves. Thread x of row n (16 threads a row) takes the slots x, x + 16, ...
template <typename T, int D, typename Args>
__device__ __forceinline__ void merge_rows(const Args& a, const Run& run, const TileRows& t, int hk, int r, const char* stage, const float* ref,
                                           const float* sum) {
  const int n = threadIdx.x >> 4, x = threadIdx.x & 15;
  if (r + n >= t.R) return;
  float M = ref[n];
#pragma unroll
  for (int w = 1; w < 4; ++w) M = fmaxf(M, ref[16 * w + n]);
  float l = 0.f, f[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = __builtin_amdgcn_exp2f(ref[16 * w + n] - M);
    l += sum[16 * w + n] * f[w];
  }
  f32x4 o[D / 64];
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w)
      o[c] += *reinterpret_cast<const f32x4*>(stage + w * (16 * D * 4) + n * (D * 4) + (((16 * c + x) ^ n) << 4)) * f[w];
  }
  const int token = (r + n) / a.group, h = hk * a.group + (r + n) % a.group;
  const int64_t row = t.q0 + token;
  if (!in_pages<Args> || run.parts == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* const to = static_cast<T*>(a.o) + row * a.o_sl + h * a.o_sh;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) store_four(to + 64 * c + 4 * x, o[c] * inv);
    if (a.lse != nullptr && x == 0)
      a.lse[(int64_t)h * a.Tq + row] = l == 0.f ? -__builtin_inff() : (M + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    if constexpr (in_pages<Args>) {
      if (a.ws_desc != nullptr && x == 0) parts_out(a).desc[row * a.Hq + h] = int2{0, 1};
    }
  } else if constexpr (in_pages<Args>) {
    const PartsOut p = parts_out(a);
    const int heads = a.Hq / a.group;
    const int64_t first = ((int64_t)run.slot * heads + hk) * p.rows + (r + n - t.r0);
    const int64_t at = first + (int64_t)run.part * heads * p.rows;
    if ((uint64_t)at >= (uint64_t)a.ws_parts) return;  // (as in find_run)
#pragma unroll
    for (int c = 0; c < D / 64; ++c) *reinterpret_cast<f32x4*>(p.o + at * D + 64 * c + 4 * x) = o[c];
    if (x == 0) {
      p.stat[at] = float2{M, l};
      if (run.part == 0) p.desc[row * a.Hq + h] = int2{(int)first, run.parts};
    }
  }
}

// ---- bf16 ------------------------------------------------------------------------------------------

// Sub-tiles of a wave in LDS: 32 rows of K, 32 of V, each copied in whole rows (global -> LDS directly, 1 KB a copy: a lane that
// loaded 16 bytes of its own key row, as the first product wants them, would touch 16 rows with every load, and the address path
// takes about four times as long for that).
//   V: 32-byte unit u of row r at position u ^ (r % 8) (D = 64, two rows in 256 bytes: u ^ (r / 2 % 4)), so that the eight
//      rows of a transpose read's 32 lanes lie in different banks;
//   K: 16-byte chunk c of row r at position c ^ (r % 16) (D = 64: c ^ (r / 2 % 8)), so that the sixteen rows that 16 lanes read the
//      same chunk of do.
template <int D>
struct SubTile {
  static constexpr int kBytes = 32 * 2 * D;
  static constexpr int kRowsPerLoad = 512 / D;                  // of a 1 KB copy
  static constexpr int kLoads = 16 / kRowsPerLoad;              // of one half
  __device__ static __forceinline__ int v_swz(int r) { return D == 128 ? r & 7 : (r >> 1) & 3; }
  __device__ static __forceinline__ int k_swz(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  // byte within its row that lane `lane` of copy u of a half fetches; the row is lane / (D / 8) of the copy's
  __device__ static __forceinline__ int v_column(int u, int lane) {
    const int r = u * kRowsPerLoad + lane / (D / 8), p = lane % (D / 8);
    return 32 * ((p >> 1) ^ v_swz(r)) + 16 * (p & 1);
  }
  __device__ static __forceinline__ int k_column(int u, int lane) {
    const int r = u * kRowsPerLoad + lane / (D / 8), p = lane % (D / 8);
    return 16 * (p ^ k_swz(r));
  }
  // where a lane reads 4 keys 16 half + 4 g .. of column 16 dt + lane % 16 of V: at v_at ^ 32 dt, 16 rows further for half 1
  __device__ static __forceinline__ uint32_t v_at(int lane) {
    const int r = 4 * (lane >> 4) + ((lane >> 2) & 3);
    return r * 2 * D + (v_swz(r) << 5) + 8 * (lane & 3);
  }
  __device__ static __forceinline__ u32x2 read_v(const char* buf, uint32_t at, int half, int dt) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((SPARSED_LDS s16x4*)(buf + (at ^ (dt << 5)) + half * 16 * 2 * D)));
  }
  // columns 32 c + 8 g .. + 7 of key 16 half + n: at k_at ^ 64 c
  __device__ static __forceinline__ uint32_t k_at(int n, int g) { return n * 2 * D + ((g ^ k_swz(n)) << 4); }
  __device__ static __forceinline__ bf16x8 read_k(const char* buf, uint32_t at, int half, int c) {
    return *reinterpret_cast<const bf16x8*>(buf + (at ^ (c << 6)) + half * 16 * 2 * D);
  }
};

// All copies of this wave but the newest N have arrived.
template <int N>
__device__ __forceinline__ void copies_done_but() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <int D, int NQ, typename Args>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : NQ == 1 ? 4 : 3, 4))) void few_rows_bf16_kernel(const Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kRows = 16 * NQ, kSteps = D / 32, kCols = D / 16;
  using Tile = SubTile<D>;
  constexpr int kCopies = 2 * Tile::kLoads;                     // of K or V of a sub-tile
  // Probabilities go into the product with V as so many bf16 parts. One rounds them to half a step of 2^-8, which over many keys is most of a
  // result's error (65536 keys, one token: 0.0023 of the result's size, 0.0017 with two, of which all is the result's own rounding). A second part
  // costs little where 16 rows share a key and memory is the bound: 32 sequences of 500-8000, 32/32 heads 327.2 -> 327.4 us, 65536 tokens, 28/4
  // heads 31.6 -> 31.7, 256 sequences of 100-300 26.6 -> 27.0, one of 300 7.3 -> 7.6 (the look at the result, below). With 32 rows the products
  // show: 128 new tokens over 16000, 28/4 heads 75.5 -> 80.7. Prompts, where products are the bound, have one part as the dense kernels do.
  constexpr int kParts = in_pages<Args> && NQ == 1 ? 2 : 1;
  __shared__ __attribute__((aligned(1024))) char kbuf[4 * Tile::kBytes];
  __shared__ __attribute__((aligned(1024))) char vbuf[4 * Tile::kBytes];
  __shared__ bf16x8 q_lds[NQ][kSteps][64];                       // fragments in the order of their use: registers are scarcer
  __shared__ float refs[NQ][4][16], sums[NQ][4][16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, g = lane >> 4;
  const int heads = a.Hq / a.group;
  const int hk = __builtin_amdgcn_readfirstlane(blockIdx.x % heads), number = __builtin_amdgcn_readfirstlane(blockIdx.x / heads);
  const Run run = find_run<kRows>(a, number, lane);
  if (run.s < 0) return;
  const TileRows t = tile_rows<kRows>(a, run);

  const int begin = run.begin * kUnit;
  const int end = run.end * kUnit < t.most ? run.end * kUnit : t.most;
  const int subs = end > begin ? (end - begin + 31) >> 5 : 0;   // of the run; this wave's are wave, wave + 4, ...
  const int total = subs > wave ? (subs - wave + 3) >> 2 : 0;

  // In pages: 32 sub-tiles of this wave at a time, lane 2 i + half holds the page of that half of sub-tile i. The first pages are asked
  // for before Q, and the first keys with them before Q is waited for: one trip to memory instead of three.
  constexpr int kSegment = in_pages<Args> ? 32 : 0x7fffffff;
  auto pages_at = [&](int seg) -> int {
    const int key = begin + 32 * (wave + 4 * seg) + 128 * (lane >> 1) + 16 * (lane & 1);
    if constexpr (in_pages<Args>) return page_of(a, run.s, key < end ? key : end - 1);
    else return 0;
  };
  int pages = total > 0 ? pages_at(0) : 0;
  int bound[NQ];                                                // keys this lane's query sees
  bf16x8 q_mine[NQ];
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    int r = t.r0 + 16 * x + n;
    r = r < t.R ? r : t.R - 1;                                  // rows that are not there repeat the last one
    const int token = r / a.group, h = hk * a.group + r % a.group;
    bound[x] = keys_seen(t.m - t.n + token, t.m, a.mask_block);
    const __bf16* from = static_cast<const __bf16*>(a.q.ptr) + (t.q0 + token) * a.q.sl + h * a.q.sh + 8 * g;
    q_mine[x] = *reinterpret_cast<const bf16x8*>(from + 32 * (wave % kSteps));
  }

  float M[NQ], l[NQ];
  f32x4 o[NQ][kCols];
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    M[x] = kNoReference;
    l[x] = 0.f;
#pragma unroll
    for (int dt = 0; dt < kCols; ++dt) o[x][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c2 = a.scale_log2;
  const char* const kbase = static_cast<const char*>(a.k.ptr) + (hk * a.k.sh + run.k0 * a.k.sl) * 2;
  const char* const vbase = static_cast<const char*>(a.v.ptr) + (hk * a.v.sh + run.k0 * a.v.sl) * 2;
  char* const k = kbuf + wave * Tile::kBytes;
  char* const v = vbuf + wave * Tile::kBytes;
  const uint32_t kread = wave * Tile::kBytes + Tile::k_at(n, g), vread = wave * Tile::kBytes + Tile::v_at(lane);

  // One half of a sub-tile: 16 keys from `key` on. In pages: in page `page`, all of them (a key behind the end has the last page
  // that is named). Packed: those of the sequence; the descriptor ends with it, and what lies behind reads as zeros.
  struct Halves {
    int page[2], key;
  };
  auto half_rsrc = [&](const char* base, const auto& p, const Halves& f, int half) {
    const int key = f.key + 16 * half;
    if constexpr (in_pages<Args>) {
      return make_rsrc(base + (f.page[half] * p.sp + (key & ((1 << a.page_shift) - 1)) * p.sl) * 2, 0x7fffffff);
    } else {
      const int64_t left = t.m - key;
      return make_rsrc(base + key * p.sl * 2, left > 0 ? ((left - 1) * p.sl + D) * 2 : 0);
    }
  };
  auto row_at = [&](const char* base, const auto& p, int key) -> const char* {
    if constexpr (in_pages<Args>) return base + (page_of(a, run.s, key) * p.sp + (key & ((1 << a.page_shift) - 1)) * p.sl) * 2;
    else return base + key * p.sl * 2;
  };
  auto copy = [&](const char* base, const auto& p, const Halves& f, char* to, auto column) {
    const int row = lane / (D / 8) * (int)p.sl * 2, step = Tile::kRowsPerLoad * (int)p.sl * 2;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const __amdgpu_buffer_rsrc_t from = half_rsrc(base, p, f, half);
#pragma unroll
      for (int u = 0; u < Tile::kLoads; ++u) {
        // (the bound of a descriptor is checked against the lane's offset, not the scalar one)
        const int at = row + column(u, lane) + (in_pages<Args> ? 0 : u * step);
        lds_load_16(from, to + (half * Tile::kLoads + u) * 1024, at, in_pages<Args> ? u * step : 0);
      }
    }
  };
  auto copy_k = [&](const Halves& f) { copy(kbase, a.k, f, k, [](int u, int ln) { return Tile::k_column(u, ln); }); };
  auto copy_v = [&](const Halves& f) { copy(vbase, a.v, f, v, [](int u, int ln) { return Tile::v_column(u, ln); }); };
  auto logits = [&](f32x4 (&s)[NQ][2]) {
    uint32_t at = kread;
    asm volatile("" : "+v"(at));  // (the addresses of a sub-tile's reads are an instruction each: not kept across the loop)
#pragma unroll
    for (int x = 0; x < NQ; ++x)
#pragma unroll
      for (int half = 0; half < 2; ++half) s[x][half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
      bf16x8 q[NQ];
#pragma unroll
      for (int x = 0; x < NQ; ++x) q[x] = q_lds[x][c][lane];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8 kf = Tile::read_k(kbuf, at, half, c);
#pragma unroll
        for (int x = 0; x < NQ; ++x) s[x][half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[x], s[x][half], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // logits to probabilities; reference, sum and output with them
  auto softmax = [&](f32x4 (&s)[NQ][2], bf16x8 (&p)[NQ][kParts], int k0) {
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      const int left = bound[x] - k0 - 4 * g;                   // keys 16 half + r (+ 4 g) below it are seen
      float top = -__builtin_inff();
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[x][half][r] = 16 * half + r < left ? s[x][half][r] * c2 : -__builtin_inff();
          top = fmaxf(top, s[x][half][r]);
        }
      if (__builtin_amdgcn_ballot_w64(top > M[x] + kSlack) != 0) {
        const float Mn = fmaxf(M[x], quad_max(top)), alpha = __builtin_amdgcn_exp2f(M[x] - Mn);
        M[x] = Mn;
        l[x] *= alpha;
#pragma unroll
        for (int dt = 0; dt < kCols; ++dt) o[x][dt] *= alpha;
      }
      u32x4 w[kParts];
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          f32x2 two = {__builtin_amdgcn_exp2f(s[x][half][r] - M[x]), __builtin_amdgcn_exp2f(s[x][half][r + 1] - M[x])};
          l[x] += two[0];
          l[x] += two[1];
#pragma unroll
          for (int part = 0; part < kParts; ++part) {  // (the sum takes them as they are)
            const uint32_t both = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2));
            w[part][2 * half + r / 2] = both;
            two[0] -= __uint_as_float(both << 16);
            two[1] -= __uint_as_float(both & 0xffff0000u);
          }
        }
#pragma unroll
      for (int part = 0; part < kParts; ++part) p[x][part] = __builtin_bit_cast(bf16x8, w[part]);
    }
  };
  auto v_frag = [&](uint32_t at, int dt) -> u32x4 {             // V of column 16 dt + n
    const u32x2 lo = Tile::read_v(vbuf, at, 0, dt), hi = Tile::read_v(vbuf, at, 1, dt);
    u32x4 w;
    w[0] = lo[0];
    w[1] = lo[1];
    w[2] = hi[0];
    w[3] = hi[1];
    return w;
  };

  // halves of sub-tile i of the segment whose first key (of this wave) is key0
  auto halves = [&](int key0, int i) {
    Halves f = {{0, 0}, key0 + 128 * i};
    if constexpr (in_pages<Args>) {
      f.page[0] = __builtin_amdgcn_readlane(pages, 2 * i);
      f.page[1] = __builtin_amdgcn_readlane(pages, 2 * i + 1);
    }
    return f;
  };
  auto copy_first = [&](int key0) {
    __builtin_amdgcn_sched_barrier(0);
    copy_k(halves(key0, 0));
    __builtin_amdgcn_sched_barrier(0);
    copy_v(halves(key0, 0));
    __builtin_amdgcn_sched_barrier(0);
  };
  if (total > 0) copy_first(begin + 32 * wave);
  if (wave < kSteps) {
#pragma unroll
    for (int x = 0; x < NQ; ++x) q_lds[x][wave][lane] = q_mine[x];
  }
  __syncthreads();

  for (int seg = 0; seg < total;) {
    const int mine = total - seg < kSegment ? total - seg : kSegment;
    const int key0 = begin + 32 * (wave + 4 * seg);             // of the wave's first sub-tile here
    // Loads complete in order. On entry the copies of K and then those of V are under way; each wait leaves those that were issued after
    // what it waits for. (Written out: the compiler does not see that a transpose read needs a copy.)
    auto step = [&](auto more, int i) {
      constexpr bool kMore = decltype(more)::value;
      const int k0 = key0 + 128 * i;
      f32x4 s[NQ][2];
      bf16x8 p[NQ][kParts];
      copies_done_but<kCopies>();
      logits(s);
      if constexpr (kMore) copy_k(halves(key0, i + 1));
      __builtin_amdgcn_sched_barrier(0);
      softmax(s, p, k0);
      copies_done_but<kMore ? kCopies : 0>();
      if (k0 + 32 > t.most) {                                   // places that no row of the tile sees: zeros
        for (int x = (t.most - k0) * (D / 8) + lane; x < 32 * (D / 8); x += 64) *reinterpret_cast<u32x4*>(v + 16 * x) = u32x4{0, 0, 0, 0};
      }
      uint32_t at = vread;
      asm volatile("" : "+v"(at));
#pragma unroll
      for (int dt = 0; dt < kCols; ++dt) {
        const bf16x8 w = __builtin_bit_cast(bf16x8, v_frag(at, dt));
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int x = 0; x < NQ; ++x) o[x][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, p[x][part], o[x][dt], 0, 0, 0);
        if (dt % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (kMore) copy_v(halves(key0, i + 1));
      __builtin_amdgcn_sched_barrier(0);
    };
    for (int i = 0; i < mine - 1; ++i) step(Yes{}, i);
    step(No{}, mine - 1);
    seg += mine;
    if (seg < total) {
      pages = pages_at(seg);
      copy_first(begin + 32 * (wave + 4 * seg));
    }
  }

  // A wave whose part is not finite looks for such a value of V among the keys that only some rows see (with two parts, whose second may be
  // zero or below, among all), and with one does its share again, slowly and with one part: a sub-tile's product is formed for every bound among
  // the rows, from V zeroed behind it, and taken by the rows that have it.
  const int odd_from = kParts == 1 && begin < t.least ? t.least : begin;
  if ((kParts > 1 || t.least < t.most) && end > odd_from) {
    f32x4 worst = {0.f, 0.f, 0.f, 0.f};  // not a number where a value is infinite or none; four sums, for the length of the chain
#pragma unroll
    for (int x = 0; x < NQ; ++x)
#pragma unroll
      for (int dt = 0; dt < kCols; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) worst[r] = __builtin_fmaf(o[x][dt][r], 0.f, worst[r]);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!((worst[0] + worst[1]) + (worst[2] + worst[3]) == 0.f)) != 0, 0)) {
      bool odd = false;
      for (int key = odd_from + (lane >> 3); key < end; key += 8) {
        const char* row = row_at(vbase, a.v, key);
        for (int x = lane & 7; x < D / 2; x += 8)  // an exponent of all ones carries
          odd = odd || (((reinterpret_cast<const uint32_t*>(row)[x] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0;
      }
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
          M[x] = kNoReference;
          l[x] = 0.f;
#pragma unroll
          for (int dt = 0; dt < kCols; ++dt) o[x][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll 1
        for (int i = 0; i < total; ++i) {
          const int k0 = begin + 32 * (wave + 4 * i);
          Halves f = {{0, 0}, k0};
          if constexpr (in_pages<Args>) {
            f.page[0] = __builtin_amdgcn_readfirstlane(page_of(a, run.s, k0));
            f.page[1] = __builtin_amdgcn_readfirstlane(page_of(a, run.s, k0 + 16 < end ? k0 + 16 : end - 1));
          }
          f32x4 s[NQ][2];
          bf16x8 p[NQ][kParts];
          copy_k(f);
          copy_v(f);
          copies_done_but<0>();
          logits(s);
          softmax(s, p, k0);
#pragma unroll 1
          for (int b = k0 + 32 <= t.least ? 32 : 1; b <= 32; ++b) {
            bool has[NQ], any = false;
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
              has[x] = (bound[x] - k0 < 32 ? bound[x] - k0 : 32) == b;
              any = any || has[x];
            }
            if (__builtin_amdgcn_ballot_w64(any) == 0) continue;
            uint32_t keep[4];                                   // of key pairs 16 (j / 2) + 2 (j % 2) + 4 g: those below b
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int left = b - 4 * g - 16 * (j >> 1) - 2 * (j & 1);
              keep[j] = left > 1 ? ~0u : left > 0 ? 0xffffu : 0u;
            }
#pragma unroll
            for (int dt = 0; dt < kCols; ++dt) {
              u32x4 w = v_frag(vread, dt);
#pragma unroll
              for (int j = 0; j < 4; ++j) w[j] &= keep[j];
#pragma unroll
              for (int x = 0; x < NQ; ++x) {
                const f32x4 add = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), p[x][0], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[x][dt][r] += has[x] ? add[r] : 0.f;
              }
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        }
      }
    }
  }

  // each wave's part, 16 rows at a time, to its own piece of the V buffer, which it has done with
  static_assert(16 * D * 4 == Tile::kBytes, "16 rows of fp32 output take a wave's V tile");
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    const float sum = quad_sum(l[x]);
    if (g == 0) {
      refs[x][wave][n] = M[x];
      sums[x][wave][n] = sum;
    }
    if (x > 0) __syncthreads();
#pragma unroll
    for (int dt = 0; dt < kCols; ++dt) *reinterpret_cast<f32x4*>(v + n * (D * 4) + (((4 * dt + g) ^ n) << 4)) = o[x][dt];
    __syncthreads();
    merge_rows<__bf16, D>(a, run, t, hk, t.r0 + 16 * x, vbuf, &refs[x][0][0], &sums[x][0][0]);
  }
#endif
}

// ---- fp32 ------------------------------------------------------------------------------------------
//
// Products on the fp32 matrix instruction (16 x 16, 4 columns a step), K and V from global memory straight into the registers
// that feed it: a lane loads 16 bytes of a row and uses them in four steps. First product: lane (i, g) holds columns
// 16 c + 4 g .. + 3 of key i, step e of c contracts the columns 16 c + 4 g' + e. Second: step s contracts the keys 4 g' + s, which
// is what accumulator register s of the first product holds; lane (i, g) loads columns 64 b + 4 i .. + 3 of key 4 g + s,
// element e of them makes output tile (b, e), whose row i is column 64 b + 4 i + e.
template <int D, typename Args>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 4))) void few_rows_f32_kernel(const Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kSteps = D / 16, kCols = D / 64;
  __shared__ __attribute__((aligned(1024))) char stage[4 * 16 * D * 4];
  __shared__ float refs[4][16], sums[4][16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, g = lane >> 4;
  const int heads = a.Hq / a.group;
  const int hk = __builtin_amdgcn_readfirstlane(blockIdx.x % heads), number = __builtin_amdgcn_readfirstlane(blockIdx.x / heads);
  const Run run = find_run<16>(a, number, lane);
  if (run.s < 0) return;
  const TileRows t = tile_rows<16>(a, run);

  const int begin = run.begin * kUnit;
  const int end = run.end * kUnit < t.most ? run.end * kUnit : t.most;
  const int subs = end > begin ? (end - begin + 15) >> 4 : 0;
  const int total = subs > wave ? (subs - wave + 3) >> 2 : 0;

  int r = t.r0 + n;
  r = r < t.R ? r : t.R - 1;
  const int token = r / a.group;
  const int bound = keys_seen(t.m - t.n + token, t.m, a.mask_block);
  f32x4 q[kSteps];
  {
    const float* from = static_cast<const float*>(a.q.ptr) + (t.q0 + token) * a.q.sl + (hk * a.group + r % a.group) * a.q.sh + 4 * g;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) q[c] = *reinterpret_cast<const f32x4*>(from + 16 * c);
  }
  float M = kNoReference, l = 0.f;
  f32x4 o[kCols][4];
#pragma unroll
  for (int b = 0; b < kCols; ++b)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float c2 = a.scale_log2;
  const char* const kbase = static_cast<const char*>(a.k.ptr) + (hk * a.k.sh + run.k0 * a.k.sl) * 4;
  const char* const vbase = static_cast<const char*>(a.v.ptr) + (hk * a.v.sh + run.k0 * a.v.sl) * 4;
  const int klane = n * (int)a.k.sl * 4 + 16 * g, vlane = 4 * g * (int)a.v.sl * 4 + 16 * n;

  // In pages: 64 sub-tiles of this wave at a time, a lane holds the page of each.
  constexpr int kSegment = in_pages<Args> ? 64 : 0x7fffffff;
  for (int seg = 0; seg < total;) {
    const int mine = total - seg < kSegment ? total - seg : kSegment;
    const int key0 = begin + 16 * (wave + 4 * seg);
    int pages = 0;
    if constexpr (in_pages<Args>) {
      const int key = key0 + 64 * lane;
      pages = page_of(a, run.s, key < end ? key : end - 1);
    }
    // Keys of sub-tile i. Packed: those of the sequence; the descriptor ends with it, and what lies behind reads as zeros.
    auto sub_at = [&](int i, const char* base, const auto& p) {
      const int key = key0 + 64 * i;
      if constexpr (in_pages<Args>) {
        return make_rsrc(base + (__builtin_amdgcn_readlane(pages, i) * p.sp + (key & ((1 << a.page_shift) - 1)) * p.sl) * 4, 0x7fffffff);
      } else {
        return make_rsrc(base + key * p.sl * 4, ((int64_t)(t.m - 1 - key) * p.sl + D) * 4);
      }
    };
    auto load = [](const __amdgpu_buffer_rsrc_t& from, int at) { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, 0)); };
    f32x4 kr[kSteps], vr[4][kCols];
    auto load_k = [&](int i) {
      const __amdgpu_buffer_rsrc_t from = sub_at(i, kbase, a.k);
#pragma unroll
      for (int c = 0; c < kSteps; ++c) kr[c] = load(from, klane + 64 * c);
    };
    auto load_v = [&](int i) {
      const __amdgpu_buffer_rsrc_t from = sub_at(i, vbase, a.v);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int b = 0; b < kCols; ++b) vr[s][b] = load(from, vlane + s * (int)a.v.sl * 4 + 256 * b);
    };
    auto step = [&](auto more, int i) {
      const int k0 = key0 + 64 * i;
      // two sums, even and odd columns: half the wait for the result of the step before
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int c = 0; c < kSteps; ++c)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[c][e], q[c][e], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[c][e + 1], q[c][e + 1], s1, 0, 0, 0);
        }
      if constexpr (decltype(more)::value) load_k(i + 1);
      __builtin_amdgcn_sched_barrier(0);
      const int left = bound - k0 - 4 * g;
      float s[4], top = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = j < left ? (s0[j] + s1[j]) * c2 : -__builtin_inff();
        top = fmaxf(top, s[j]);
      }
      if (__builtin_amdgcn_ballot_w64(top > M + kSlack) != 0) {
        const float Mn = fmaxf(M, quad_max(top)), alpha = __builtin_amdgcn_exp2f(M - Mn);
        M = Mn;
        l *= alpha;
#pragma unroll
        for (int b = 0; b < kCols; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[b][e] *= alpha;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = __builtin_amdgcn_exp2f(s[j] - M);
        l += s[j];
      }
      bool odd_values = false;                                  // infinite or not a number, where not every row sees every key
      if (k0 + 16 > t.least) {
        float zero = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int b = 0; b < kCols; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) zero = __builtin_fmaf(vr[j][b][e], 0.f, zero);
        odd_values = __builtin_amdgcn_ballot_w64(!(zero == 0.f)) != 0;
      }
      if (!odd_values) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int b = 0; b < kCols; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[b][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[j][b][e], s[j], o[b][e], 0, 0, 0);
      } else {
#pragma unroll 1
        for (int bd = 1; bd <= 16; ++bd) {
          const int mine_b = bound - k0;
          const bool has = (mine_b < 16 ? mine_b : 16) == bd;
          if (__builtin_amdgcn_ballot_w64(has) == 0) continue;
#pragma unroll
          for (int b = 0; b < kCols; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              f32x4 add = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int j = 0; j < 4; ++j) add = __builtin_amdgcn_mfma_f32_16x16x4f32(4 * g + j < bd ? vr[j][b][e] : 0.f, s[j], add, 0, 0, 0);
#pragma unroll
              for (int x = 0; x < 4; ++x) o[b][e][x] += has ? add[x] : 0.f;
            }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (decltype(more)::value) load_v(i + 1);
      __builtin_amdgcn_sched_barrier(0);
    };
    load_k(0);
    load_v(0);
    for (int i = 0; i < mine - 1; ++i) step(Yes{}, i);
    step(No{}, mine - 1);
    seg += mine;
  }

  const float sum = quad_sum(l);
  if (g == 0) {
    refs[wave][n] = M;
    sums[wave][n] = sum;
  }
  // row 4 g + x of output tile (b, e) is column 64 b + 16 g + 4 x + e
#pragma unroll
  for (int b = 0; b < kCols; ++b)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *reinterpret_cast<f32x4*>(stage + wave * (16 * D * 4) + n * (D * 4) + (((16 * b + 4 * g + x) ^ n) << 4)) =
          f32x4{o[b][0][x], o[b][1][x], o[b][2][x], o[b][3][x]};
  __syncthreads();
  merge_rows<float, D>(a, run, t, hk, t.r0, stage, &refs[0][0], &sums[0][0]);
#endif
}

// ---- joining the parts of a row --------------------------------------------------------------------

// A work-group takes a row. Its threads are 256 / (D / 4) lines; a line adds every (256 / (D / 4))th part, a thread four columns of them.
// 4.6 us for 28 rows of 256 / 4 parts each, mostly the trips to memory for descriptor, statistics and columns.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kThreads = D / 4, kLines = 256 / kThreads;
  __shared__ float refs[4], sums[4], factor[256];
  __shared__ f32x4 out[kLines][kThreads];
  const int t = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq;
  if (a.cu_q != nullptr) {  // only rows of a sequence have parts
    const int s = seq_of_row(a.cu_q, a.n_seqs, t);
    if (s >= a.n_seqs) return;
    const SeqRows r = seq_rows(a.cu_q, s, a.Tq);
    if (t < r.begin || t >= r.end) return;
  }
  const PartsOut p = parts_out(a);
  const int2 d = p.desc[(int64_t)t * a.Hq + h];
  if (d.y <= 1) return;  // stored whole
  const int line = threadIdx.x / kThreads, x = threadIdx.x % kThreads, lane = threadIdx.x & 63;
  const int64_t stride = (int64_t)(a.Hq / a.group) * p.rows;
  if (d.x < 0 || d.x + (d.y - 1) * stride >= a.ws_parts) return;
  // 256 parts at a time: the factors of all of them first, then loads that wait for nothing
  float M = kNoReference, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < d.y; i0 += 256) {
    const int here = d.y - i0 < 256 ? d.y - i0 : 256;
    const int64_t first = d.x + i0 * stride;
    const float2 st = (int)threadIdx.x < here ? p.stat[first + threadIdx.x * stride] : float2{kNoReference, 0.f};
    float top = st.x;
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, 64));
    if (lane == 0) refs[threadIdx.x >> 6] = top;
    __syncthreads();
    const float Mn = fmaxf(fmaxf(fmaxf(refs[0], refs[1]), fmaxf(refs[2], refs[3])), M), f = __builtin_amdgcn_exp2f(M - Mn);
    M = Mn;
    const float mine = __builtin_amdgcn_exp2f(st.x - M);
    factor[threadIdx.x] = mine;
    const float sum = wave_sum(st.y * mine);
    if (lane == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    l = l * f + ((sums[0] + sums[1]) + (sums[2] + sums[3]));
    o *= f;
    const float* const from = p.o + first * D + 4 * x;
#pragma unroll 8
    for (int i = line; i < here; i += kLines) o += *reinterpret_cast<const f32x4*>(from + i * stride * D) * factor[i];
    __syncthreads();  // (the factors are read before the next ones are written)
  }
  out[line][x] = o;
  __syncthreads();
  if (line != 0) return;
#pragma unroll
  for (int i = 1; i < kLines; ++i) o += out[i][x];
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store_four(static_cast<T*>(a.o) + t * a.o_sl + h * a.o_sh + 4 * x, o * inv);
  if (a.lse != nullptr && x == 0) a.lse[(int64_t)h * a.Tq + t] = l == 0.f ? -__builtin_inff() : (M + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
#endif
}

// ---- launches --------------------------------------------------------------------------------------

PagedShape paged_shape(bool bf16, int64_t Tq, int64_t n_seqs, int64_t Hq, int64_t heads, bool one_each, int64_t max_tokens) {
  PagedShape s{};
  const int64_t group = Hq / heads, rows = Tq * group;
  s.tile_rows = bf16 && rows > 16 * n_seqs ? 32 : 16;
  const int64_t tiles = one_each ? n_seqs * ((group + s.tile_rows - 1) / s.tile_rows) : rows / s.tile_rows + (n_seqs < Tq ? n_seqs : Tq);
  const int64_t units = (max_tokens + kUnit - 1) / kUnit;
  s.splits = units > kWholeUnits;
  // A tile has one run, and a further one for every full run length of keys behind it. Of these there are work / run_units(work) at
  // most, for the work there is, which is at most that of full pages.
  const int64_t most = tiles * units * heads;
  int64_t further = most / 8 < kMaxRuns ? most / 8 : kMaxRuns;
  further = further > 256 ? further : 256;
  further = (further < most ? further : most) / heads + 1;
  s.groups = (tiles + (s.splits ? further : 0)) * heads;
  if (s.splits) {
    s.part_rows = rows < s.tile_rows ? (int)rows : s.tile_rows;
    s.parts = 2 * further * heads * s.part_rows;  // only tiles of two runs or more have parts: at most twice as many as full run lengths
  }
  return s;
}

template <typename T, int D>
static hipError_t launch_one(const PagedArgs& a, const PagedShape& sh, hipStream_t s) {
  const dim3 grid((unsigned)sh.groups), block(256);
  if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((few_rows_f32_kernel<D, PagedArgs>), grid, block, 0, s, a);
  else if (sh.tile_rows == 32) hipLaunchKernelGGL((few_rows_bf16_kernel<D, 2, PagedArgs>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((few_rows_bf16_kernel<D, 1, PagedArgs>), grid, block, 0, s, a);
  if (sh.splits) hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3((unsigned)((int64_t)a.Tq * a.Hq)), block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_attn_paged(bool bf16, int D, const PagedArgs& a, const PagedShape& sh, hipStream_t s) {
  if (bf16) return D == 128 ? launch_one<__bf16, 128>(a, sh, s) : launch_one<__bf16, 64>(a, sh, s);
  return D == 128 ? launch_one<float, 128>(a, sh, s) : launch_one<float, 64>(a, sh, s);
}

static int64_t prompt_groups(int tile_rows, const PromptArgs& a) {
  const int64_t heads = a.Hq / a.group, rows = (int64_t)a.Tq * a.group;
  return (rows / tile_rows + (a.n_seqs < a.Tq ? a.n_seqs : a.Tq)) * heads;
}

hipError_t launch_prompt_few_rows_bf16(int D, const PromptArgs& a, hipStream_t s) {
  const int64_t groups = prompt_groups(32, a);
  if (!grid_fits(groups, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)groups), block(256);
  if (D == 128) hipLaunchKernelGGL((few_rows_bf16_kernel<128, 2, PromptArgs>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((few_rows_bf16_kernel<64, 2, PromptArgs>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_prompt_few_rows_f32(int D, const PromptArgs& a, hipStream_t s) {
  const int64_t groups = prompt_groups(16, a);
  if (!grid_fits(groups, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)groups), block(256);
  if (D == 128) hipLaunchKernelGGL((few_rows_f32_kernel<128, PromptArgs>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((few_rows_f32_kernel<64, PromptArgs>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace sparsed
