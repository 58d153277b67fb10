// Attention of packed prompts, bf16 (gfx950): causal, or in blocks of mask_block tokens.
//
// A work-group takes 32 NW query rows of one head of one sequence and walks 64-key tiles up to the last key its last row
// sees. Tiles, LDS layouts, the transposed formulation, the pipeline of 32-key sub-steps (the next sub-tile's logits, this one's
// softmax and the product of the one before in one instruction stream) and the fixed softmax reference are those of the
// dense kernel (tile_bf16.hpp, attn_bf16_kernel.hpp). What a mask adds:
//
//  * Keys seen are a prefix of the sequence, so the tiles of a work-group are full for all of its rows, then a few that are full for
//    some, then nothing. The first run unmasked steps; the others masked ones, in which a lane compares the keys with its own
//    query's bound, and a wave whose rows see nothing more only helps to copy. The first sub-tile holds a key that a row sees
//    if it sees any, so the reference is a logit of the row (rows that see nothing: 0 weights throughout).
//  * Work-groups have 1 to L / 64 tiles. They are launched longest first over all sequences: tile number j of a sequence
//    has about (j + 1) 32 NW keys wherever it belongs, so the order is by j, downwards. A work-group finds its place from
//    the offsets on the device (the host does not know the lengths).
//  * 0 times what V holds at a hidden key need not be 0. A wave whose result is not finite looks at V behind its
//    first row's bound; if something infinite or NaN lies there it does its rows again in a plain loop that
//    never lets a row meet a value it does not see (attend_again). So does a wave that met logits beyond 2^28 octaves.
#include "cache.hpp"
#include "kernels.hpp"
#include "prompt_tiles.hpp"
#include "tile_bf16.hpp"

namespace sparsed {

// ---- rows done again -------------------------------------------------------------------------------

// The wave's 32 rows in a plain loop over 32-key sub-tiles, K and V straight from memory, every scaled logit rounded as the reference
// is, which is one of them. Where a sub-tile is not seen by all
// rows, its product with V is formed for every bound among them, from V zeroed behind it, and taken by the rows that have it.
// Slow, and only for values of V that are infinite or not numbers next to the diagonal and for logits beyond 2^28 octaves.
template <int D>
__device__ __forceinline__ void attend_again(const __bf16* k, const __bf16* v, int64_t ksl, int64_t vsl, int m, int bound, int least,
                                                       int most, float c, const bf16x8 (&qf)[D / 16], f32x16 (&o)[D / 32], float* M_out,
                                                       float* l_out, int lane) {
  const int j = lane & 31, g = lane >> 5;
  float M = -3e38f, l = 0.f;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[dt][x] = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < most; k0 += 32) {
    f32x16 s;
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = 0.f;
    int row = k0 + krow_perm(j);
    row = row < m ? row : m - 1;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(k + row * ksl + 16 * kk + 8 * g), qf[kk], s, 0, 0, 0);
    float top = -__builtin_inff();
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      s[x] = k0 + 16 * (x >> 3) + 8 * g + (x & 7) < bound ? s[x] * c : -__builtin_inff();
      top = fmaxf(top, s[x]);
    }
    const float Mn = fmaxf(M, pair_max(top)), alpha = __builtin_amdgcn_exp2f(M - Mn);
    M = Mn;
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[dt][x] *= alpha;
    bf16x8 p[2];
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const float e = __builtin_amdgcn_exp2f(s[x] - M);
      l += e;
      p[x >> 3][x & 7] = (__bf16)e;
    }
    const int first = k0 + 32 <= least ? 32 : 1;
#pragma unroll 1
    for (int b = first; b <= 32; ++b) {
      const bool has = first == 32 || (bound - k0 < 32 ? bound - k0 : 32) == b;
      if (__builtin_amdgcn_ballot_w64(has) == 0) continue;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        f32x16 add;
#pragma unroll
        for (int x = 0; x < 16; ++x) add[x] = 0.f;
#pragma unroll
        for (int mp = 0; mp < 2; ++mp) {
          bf16x8 vf;
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const int key = 16 * mp + 8 * g + x;
            vf[x] = key < b && k0 + key < m ? v[(k0 + key) * vsl + 32 * dt + j] : (__bf16)0.f;
          }
          add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[mp], add, 0, 0, 0);
        }
#pragma unroll
        for (int x = 0; x < 16; ++x) o[dt][x] += has ? add[x] : 0.f;
      }
    }
  }
  *M_out = M;
  *l_out = l;
}

// ---- the kernel ------------------------------------------------------------------------------------

struct Even { static constexpr int value = 0; };
struct Odd { static constexpr int value = 1; };
struct Plain { static constexpr bool value = false; };
struct Masked { static constexpr bool value = true; };

// The layout of a masked sub-step: as sched_substep_interleave, with the 32 instructions of the mask handed out among the
// matrix instructions as well (six behind each).
template <int D>
__device__ __forceinline__ void sched_masked_substep() {
  constexpr int kMfma = D / 32 * 2 + D / 16, kReads = D / 32 * 4 + D / 16, kAhead = 4;
  constexpr int kValuPer = (D == 128 ? 96 : 92) / kMfma;
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
  for (int i = 0; i < kMfma; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, (kReads - kAhead + kMfma - 1) / kMfma, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, kValuPer, 0);
  }
}

template <int D, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void prompt_bf16_kernel(const PromptArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NT = NW * 64, QT = 32 * NW;
  constexpr int kKBytes = KLayout<D>::kTileBytes, kVBytes = VLayout<D>::kTileBytes;
  constexpr float kOverflow = 1.152921504606847e18f;  // 2^60: a 16-key partial sum at or above this re-references the row
  constexpr float kFar = 268435456.f, kNoReference = -3e38f;
  __shared__ __attribute__((aligned(1024))) char kbuf0[kKBytes];
  __shared__ __attribute__((aligned(1024))) char kbuf1[kKBytes];
  __shared__ __attribute__((aligned(1024))) char vbuf0[kVBytes];
  __shared__ __attribute__((aligned(1024))) char vbuf1[kVBytes];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t ksl = a.k.sl, vsl = a.v.sl;
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  // What a work-group takes at place `unit` of the launch order. (The same lines without the structure and the calls compile to slower code:
  // two prompts of 1000 tokens, 32 heads of 128, 28.2 -> 29.6 us, 8192 tokens, 28/4 heads of 64, 264 -> 266.)
  struct Place {
    int valid, h, q0, n_rows, row0, least, most, n, n_full, n_mine, m, shift;
    const __bf16 *kbase, *vbase;
  };
  auto bound_at = [&](const Place& p, int i) { return keys_seen(p.shift + (i < p.n_rows ? i : p.n_rows - 1), p.m, a.mask_block); };
  auto place = [&](int unit) {
    Place p{};
    // Heads of a place go to the XCDs in turn; where they divide evenly, those that share K and V to the same one.
    const int pos = uniform(unit / a.Hq), hh = unit - pos * a.Hq;
    const PromptTile at = find_tile<QT>(a, pos, lane);
    p.valid = at.s >= 0;
    if (!p.valid) return p;
    p.h = (a.Hq & 7) == 0 ? (hh & 7) * (a.Hq >> 3) + (hh >> 3) : hh;
    const int hk = uniform(p.h / a.group);
    p.q0 = at.q.begin;
    p.n_rows = at.q.end - at.q.begin;
    p.m = at.k.end - at.k.begin;
    p.shift = p.m - p.n_rows;                                       // row i stands at position shift + i
    p.row0 = at.tile * QT + wave * 32;                              // first row of this wave in its sequence
    p.least = uniform(bound_at(p, p.row0));
    p.most = uniform(bound_at(p, p.row0 + 31));
    p.n = uniform((bound_at(p, at.tile * QT + QT - 1) + kTileK - 1) / kTileK);  // tiles of the work-group
    p.n_full = uniform(bound_at(p, at.tile * QT) / kTileK);         // of them seen by all of its rows
    p.n_mine = p.row0 < p.n_rows ? (p.most + kTileK - 1) / kTileK : 0;  // of this wave
    p.kbase = static_cast<const __bf16*>(a.k.ptr) + at.k.begin * a.k.sl + hk * a.k.sh;
    p.vbase = static_cast<const __bf16*>(a.v.ptr) + at.k.begin * a.v.sl + hk * a.v.sh;
    return p;
  };
  const Place pl = place(blockIdx.x);
  if (!pl.valid) return;

  float M = 0.f, lsum = 0.f;
  f32x16 o[1][D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[0][dt][x] = 0.f;
  const int bound = bound_at(pl, pl.row0 + (lane & 31));  // keys this lane's query sees
  f32x16 s_even[1], s_odd[1];
  bf16x8 p_even[1][2], p_odd[1][2];

  TileDma<D, NT, false> kdma;
  TileDma<D, NT, true> vdma;
  kdma.init(ksl, wave, lane);
  vdma.init(vsl, wave, lane);
  KFragAddr<D> kaddr;
  VFragAddr<D> vaddr;
  kaddr.init(lane);
  vaddr.init(lane);
  QFrag<D, 1> qf;

  // a tile's descriptor from its own 64-bit address: a packed array may be larger than 32-bit offsets reach
  auto tile_rsrc = [&](const __bf16* base, int64_t sl, int tile) { return make_rsrc(base + (int64_t)tile * kTileK * sl, 0x7fffffff); };
  auto copy = [&](const auto& dma, const __bf16* base, int64_t sl, int tile, char* dst) { dma.issue(tile_rsrc(base, sl, tile), 0, dst, wave); };
  // the same for a tile that may be the partial last one, or behind it (any real tile will do)
  auto copy_any = [&](const auto& dma, const __bf16* base, int64_t sl, int m, int tile, char* dst) {
    const int last_tile = (m - 1) / kTileK, tail_keys = m - last_tile * kTileK;
    const int t = tile < last_tile ? tile : last_tile;
    if (t == last_tile && tail_keys < kTileK) dma.issue_partial(tile_rsrc(base, sl, t), 0, dst, wave, lane, sl, tail_keys);
    else copy(dma, base, sl, t, dst);
  };
  // the first tiles and the queries of a place
  auto begin = [&](const Place& p) {
    if (p.n == 0) return;
    copy_any(kdma, p.kbase, ksl, p.m, 0, kbuf0);
    copy_any(kdma, p.kbase, ksl, p.m, 1, kbuf1);
    copy_any(vdma, p.vbase, vsl, p.m, 0, vbuf0);
    qf.load(static_cast<const __bf16*>(a.q.ptr) + p.q0 * a.q.sl + p.h * a.q.sh, p.row0, p.n_rows, a.q.sl, lane);
  };

  const float c = a.scale_log2;
  auto mask_sub = [&](f32x16& s, int k0) {
    const int mine = bound - k0 - 8 * (lane >> 5);  // register x holds key 16*(x/8) + 8*g + x%8 of the sub-tile
#pragma unroll
    for (int x = 0; x < 16; ++x)
      s[x] = 16 * (x >> 3) + (x & 7) < mine ? s[x] : -__builtin_inff();
  };
  auto exp_sub = [&](const f32x16& s, bf16x8(&p)[2], float& part) {
    part = 0.f;
#pragma unroll
    for (int mm = 0; mm < 2; ++mm) {
      u32x4 pk;
#pragma unroll
      for (int x = 0; x < 8; x += 2) {
        const f32x2 two = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * mm + x], c, -M)), __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * mm + x + 1], c, -M))};
        // rounded for the bf16 matrix cores, to half a step of 2^-8; the sum keeps them as they are
        pk[x >> 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2));
        part += two[0];
        part += two[1];
      }
      asm volatile("" : "+v"(pk));  // here, not sunk past the branch that follows
      p[mm] = __builtin_bit_cast(bf16x8, pk);
    }
    asm volatile("" : "+v"(part));
  };
  auto row_max = [&](const f32x16& s) -> float {
    float mx = fmaxf(s[0], s[1]);
#pragma unroll
    for (int x = 2; x < 16; x += 2) mx = fmaxf(fmaxf(mx, s[x]), s[x + 1]);
    return pair_max(mx) * c;
  };
  // exp_sub leaves the product of logit and scale unrounded and subtracts a reference that is rounded: its weights are all off by one
  // factor, 2^8 at most for references below 2^28 octaves and without bounds beyond. A reference that far out is lifted by more than its rounding,
  // so that no weight overflows (they vanish), and rows that end with one are done again.
  auto is_far = [&](float m) { return fabsf(m) >= kFar; };
  auto reference = [&](float top) { return is_far(top) ? top + fabsf(top) * 1.1920929e-7f : top; };
  auto overflowed = [&](float part) -> bool { return __builtin_amdgcn_ballot_w64(!(part < kOverflow)) != 0; };
  auto re_reference = [&](const f32x16& s, bf16x8(&p)[2], float& part) {
    const float Mn = fmaxf(M, reference(row_max(s))), alpha = __builtin_amdgcn_exp2f(M - Mn);
    M = Mn;
    lsum *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[0][dt][x] *= alpha;
    exp_sub(s, p, part);
  };

  // Tile step t (LDS parity t & 1) = sub-steps 2t+1 and 2t+2, as in the dense kernel: on entry S(2t+1) in s_odd, P(2t) in
  // p_even, K(t+1) and V(t) in LDS; K(t+2) and V(t+1) are asked for.
  auto step = [&](auto parity, auto masked, int t) {
    constexpr int P = decltype(parity)::value;
    constexpr bool kMasked = decltype(masked)::value;
    char* const kb_free = P ? kbuf1 : kbuf0;
    char* const kb_next = P ? kbuf0 : kbuf1;
    char* const vb_this = P ? vbuf1 : vbuf0;
    char* const vb_free = P ? vbuf0 : vbuf1;
    if (kMasked) {
      copy_any(kdma, pl.kbase, ksl, pl.m, t + 2, kb_free);
      copy_any(vdma, pl.vbase, vsl, pl.m, t + 1, vb_free);
    } else {
      copy(kdma, pl.kbase, ksl, t + 2, kb_free);
      copy(vdma, pl.vbase, vsl, t + 1, vb_free);
    }
    if (!kMasked || t < pl.n_mine) {
      float part;
      logits_sub<D, 1, false>(kb_next, 0, kaddr, qf, s_even);
      pv_sub<D, 1, false>(vb_this, 0, vaddr, p_even, o);
      if (kMasked) mask_sub(s_odd[0], t * kTileK + 32);
      exp_sub(s_odd[0], p_odd[0], part);
      if (kMasked) sched_masked_substep<D>();
      else sched_substep_interleave<D, 1, true>();
      if (__builtin_expect(overflowed(part), 0)) re_reference(s_odd[0], p_odd[0], part);
      lsum += part;
      __builtin_amdgcn_sched_barrier(0);
      logits_sub<D, 1, false>(kb_next, 1, kaddr, qf, s_odd);
      pv_sub<D, 1, false>(vb_this, 1, vaddr, p_odd, o);
      if (kMasked) mask_sub(s_even[0], (t + 1) * kTileK);
      exp_sub(s_even[0], p_even[0], part);
      if (kMasked) sched_masked_substep<D>();
      else sched_substep_interleave<D, 1, true>();
      if (__builtin_expect(overflowed(part), 0)) re_reference(s_even[0], p_even[0], part);
      lsum += part;
    }
    __syncthreads();
  };

  begin(pl);
  if (pl.n > 0) {
    __syncthreads();
    logits_sub<D, 1, true>(kbuf0, 0, kaddr, qf, s_even);
    logits_sub<D, 1, true>(kbuf0, 1, kaddr, qf, s_odd);
    mask_sub(s_even[0], 0);
    M = fmaxf(reference(row_max(s_even[0])), kNoReference);
    exp_sub(s_even[0], p_even[0], lsum);
    __syncthreads();
    // an unmasked step at t has the softmax of tiles t and t + 1, which all rows see, and the copy of tile t + 2, which has to be whole
    const int whole = pl.m / kTileK, plain = pl.n_full - 1 < whole - 2 ? pl.n_full - 1 : whole - 2;  // steps t < plain
    int t = 0;
    while (t + 1 < plain) {
      step(Even{}, Plain{}, t);
      step(Odd{}, Plain{}, t + 1);
      t += 2;
    }
    if (t < plain) {
      step(Even{}, Plain{}, t);
      step(Odd{}, Masked{}, t + 1);
      t += 2;
    }
    // in twos as well (a step behind the last tile only copies)
    for (; t < pl.n; t += 2) {
      step(Even{}, Masked{}, t);
      step(Odd{}, Masked{}, t + 1);
    }
  }

  // Each wave passes its 32 x D tile through its own slice of the idle K/V buffers and stores whole rows (as the dense kernel).
  float ltot = pair_sum(lsum);
  {
    float worst = 0.f;  // NaN if a value is infinite or not a number
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int x = 0; x < 16; ++x) worst = __builtin_fmaf(o[0][dt][x], 0.f, worst);
    bool again = __builtin_amdgcn_ballot_w64(is_far(M) && fabsf(M) < -0.5f * kNoReference) != 0;  // (a scaled logit is below 2^126)
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(worst == 0.f)) != 0, 0) && pl.row0 < pl.n_rows) {
      // anything infinite or not a number behind the first row's bound, as far as the last row's tile goes? (behind the last
      // key that repeats)
      bool odd = false;
      const int from = pl.n_mine * kTileK > pl.m && pl.least > pl.m - 1 ? pl.m - 1 : pl.least;
      for (int key = from + (lane >> 3); key < pl.n_mine * kTileK && key < pl.m; key += 8) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(pl.vbase + key * vsl);
        for (int x = lane & 7; x < D / 2; x += 8) odd = odd || (((w[x] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0;
      }
      again = again || __builtin_amdgcn_ballot_w64(odd) != 0;
    }
    if (__builtin_expect(again, 0) && pl.row0 < pl.n_rows) {
      attend_again<D>(pl.kbase, pl.vbase, ksl, vsl, pl.m, bound, pl.least, pl.most, c, qf.f[0], o[0], &M, &lsum, lane);
      ltot = pair_sum(lsum);
    }
  }
  constexpr int kRowBytes = 2 * D, kSlots = D / 8, kRowsPerStore = 64 / kSlots;
  static_assert(32 * kRowBytes * 2 <= kKBytes && 32 * kRowBytes * 2 <= kVBytes, "two waves share one buffer");
  const int je = lane & 31, ge = lane >> 5;
  char* const stage = ((wave >> 1) == 0 ? kbuf0 : (wave >> 1) == 1 ? kbuf1 : (wave >> 1) == 2 ? vbuf0 : vbuf1) + (wave & 1) * (32 * kRowBytes);
  if (a.lse != nullptr && ge == 0 && pl.row0 + je < pl.n_rows)
    a.lse[(int64_t)pl.h * a.Tq + pl.q0 + pl.row0 + je] = ltot == 0.f ? -__builtin_inff() : (M + __builtin_amdgcn_logf(ltot)) * 0.6931471805599453f;
  const float inv = ltot == 0.f ? 0.f : 1.0f / ltot;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const f32x2 lo = {o[0][dt][4 * q4] * inv, o[0][dt][4 * q4 + 1] * inv};
      const f32x2 hi = {o[0][dt][4 * q4 + 2] * inv, o[0][dt][4 * q4 + 3] * inv};
      u32x2 w;
      w[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2));
      w[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2));
      *reinterpret_cast<u32x2*>(stage + je * kRowBytes + (((4 * dt + q4) ^ (je & (kSlots - 1))) << 4) + 8 * ge) = w;
    }
  __bf16* const obase = static_cast<__bf16*>(a.o) + pl.q0 * a.o_sl + pl.h * a.o_sh;
#pragma unroll
  for (int it = 0; it < 32 / kRowsPerStore; ++it) {
    const int r = it * kRowsPerStore + lane / kSlots, slot = lane % kSlots;
    const u32x4 w = *reinterpret_cast<const u32x4*>(stage + r * kRowBytes + ((slot ^ (r & (kSlots - 1))) << 4));
    if (pl.row0 + r < pl.n_rows) *reinterpret_cast<u32x4*>(obase + (int64_t)(pl.row0 + r) * a.o_sl + slot * 8) = w;
  }
#endif
}

template <int D, int NW>
static hipError_t launch_one(const PromptArgs& a, hipStream_t s) {
  constexpr int QT = 32 * NW;
  // at most: every full tile there is room for, and a partial one of every sequence that has rows
  const int64_t groups = ((int64_t)a.Tq / QT + (a.n_seqs < a.Tq ? a.n_seqs : a.Tq)) * a.Hq;
  if (!grid_fits(groups, NW * 64)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((prompt_bf16_kernel<D, NW>), dim3((unsigned)(groups)), dim3(NW * 64), 0, s, a);
  return hipGetLastError();
}

// Which form a call takes. Rows: tokens times heads.
//   few rows  32 rows a work-group whose waves split the keys (attn_paged.hip): a call that leaves most of the chip idle is as long as its
//             longest row, which they walk in a quarter of the steps. us, 128 rows a work-group -> this: 32 heads of 128 over 300 tokens
//             12.2 -> 9.3, 8 over 1000 20.7 -> 14.2, 8 over 2000 33 -> 26; even at 32 over 600 (17.1, 17.3), 22 -> 27 at 32 over 1000.
//             Head dim 64, where a step is shorter, by rows: 8 heads over 2000 24.2 -> 20.1, 3500 38.3 -> 37.8, 4096 43.5 -> 45.4; 24 prompts of
//             1-600 (23144 rows, 27256, 28616) 11.9 -> 9.9, 12.2 -> 10.7, 12.3 -> 12.3; where all are as long the others win earlier, 4 of 500
//             (16000 rows) 10.6 -> 9.2, 5 10.7 -> 11.0, 7 11.2 -> 13.0, 12 of 330 (31680) 10.2 -> 11.3: the rows do not tell, and from 28672 on
//             nothing is won. And up to 8 tokens a sequence, where larger
//             tiles are mostly empty: 256 prompts of 8, 32 heads of 128 111 -> 80, 28/4 heads 97 -> 26 (of 16, 118 -> 90 and 99 -> 45; but
//             the others may be empty, and a prompt of 2048, 32 heads, would take 43 -> 72, of 4096 125 -> 240: up to 65536 rows, 131072 at
//             head dim 64).
//   128 rows  four waves, two work-groups a compute unit: where 256 rows would leave units idle (32 heads over 2048 tokens 50 -> 45 us).
//   256 rows  eight waves, a tile copied for twice the rows: us, 128 rows -> this: 16384 tokens x 8 heads 495 -> 450, 4096 x 32 132 -> 124; 6
//             prompts of 500-6000 391 -> 396, 16 of 500-1000 165 -> 152, 32 of 300 107 -> 127, 256 of 64 156 -> 247: where sequences have
//             256 tokens or more on average. Head dim 64, where the start of a work-group that is alone on its compute unit weighs more:
//             16 of 500-1000 47 -> 53, 4 of 2000 46 -> 46, one of 4096 82 -> 78, of 8192 156 -> 146: from 4096 on.
hipError_t launch_prompt_bf16(int D, const PromptArgs& a, hipStream_t s) {
  if (few_rows(true, D, a)) return launch_prompt_few_rows_bf16(D, a, s);
  const bool wide = (int64_t)(a.Tq / 256) * a.Hq >= 512 && a.Tq >= (int64_t)a.n_seqs * (D == 64 ? 4096 : 256);
  if (D == 128) return wide ? launch_one<128, 8>(a, s) : launch_one<128, 4>(a, s);
  return wide ? launch_one<64, 8>(a, s) : launch_one<64, 4>(a, s);
}

}  // namespace sparsed
