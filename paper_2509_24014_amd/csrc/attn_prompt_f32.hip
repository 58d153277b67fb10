// Attention of packed prompts, fp32 (gfx950): causal, or in blocks of mask_block tokens.
//
// Both products run on the fp32 matrix instruction (32 x 32, 2 columns a step, 64 cycles), which is what bounds the kernel:
// 128 of them for 32 keys and 32 rows of 128 columns, against some 150 vector instructions of the softmax that run beside the
// other wave's. A work-group owns 32 rows; its four waves take 32-key sub-tiles in turn, each with its own reference, sum
// and output, and merge them once, so that a call of few rows has four times the waves and the longest row a quarter of the steps.
//
// K and V go from global memory straight into the registers that feed the products, a wave's share once; Q, which all four
// waves need, lies in LDS in the order of its use. Transposed as everywhere: S^T = K Q^T leaves a lane one query and 16 keys.
//   first product:  lane (i, g) holds columns 8 c + 4 g .. + 3 of key i; step e of c contracts columns 8 c + 4 g' + e.
//   second product: register x of the first contracts keys 8 (x / 4) + x % 4 + 4 g'; lane (i, g) loads D/32 consecutive
//                   columns of that key; element e of them makes output tile e, whose row i is column (D/32) i + e.
// 16384 tokens, 8 heads of 128: 3.99 ms = 138 TFLOP/s, what a large fp32 product reaches (136 at 4096^3); 4096 x 32: 132; 2000 and 1489
// tokens x 8: 98 (131 us), where 880 work-groups of 1 to 63 sub-tiles on 256 compute units leave the matrix units busy 64 % of the time.
// Softmax as in the paged kernels: the reference moves when a logit exceeds it by 8 octaves.
#include "cache.hpp"
#include "prompt_tiles.hpp"
#include "tile_f32.hpp"

namespace sparsed {

template <int N>
struct Columns;  // N consecutive fp32 columns
template <>
struct Columns<4> { typedef f32x4 T; };
template <>
struct Columns<2> { typedef f32x2f T; };

struct More { static constexpr bool value = true; };
struct Last { static constexpr bool value = false; };

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void prompt_f32_kernel(const PromptArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kSteps = D / 8, kTiles = D / 32;
  typedef typename Columns<kTiles>::T Cols;
  constexpr float kNoReference = -3e38f, kSlack = 8.f;
  __shared__ __attribute__((aligned(16))) float stage[4][32][D];
  f32x4(*const q_lds)[64] = reinterpret_cast<f32x4(*)[64]>(&stage[0][0][0]);  // until the waves' parts are merged
  __shared__ float refs[4][32], sums[4][32];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int i = lane & 31, g = lane >> 5;
  // Heads of a place go to the XCDs in turn; where they divide evenly, those that share K and V to the same one.
  const int pos = (int)blockIdx.x / a.Hq, hh = (int)blockIdx.x % a.Hq;
  const int h = (a.Hq & 7) == 0 ? (hh & 7) * (a.Hq >> 3) + (hh >> 3) : hh, hk = h / a.group;
  const PromptTile at = find_tile<32>(a, pos, lane);
  if (at.s < 0) return;
  const SeqRows rq = at.q, rk = at.k;
  const int n_rows = rq.end - rq.begin, m = rk.end - rk.begin, shift = m - n_rows;
  const int row0 = at.tile * 32, last_row = row0 + 32 < n_rows ? row0 + 31 : n_rows - 1;
  const int my_row = row0 + i < n_rows ? row0 + i : n_rows - 1;  // rows that are not there repeat the last one
  const int bound = keys_seen(shift + my_row, m, a.mask_block);
  const int least = __builtin_amdgcn_readfirstlane(keys_seen(shift + row0, m, a.mask_block));
  const int most = __builtin_amdgcn_readfirstlane(keys_seen(shift + last_row, m, a.mask_block));
  const int subs = (most + 31) >> 5;

  {
    const float* const from = static_cast<const float*>(a.q.ptr) + (rq.begin + my_row) * a.q.sl + h * a.q.sh + 4 * g;
    for (int c = wave; c < kSteps; c += 4) q_lds[c][lane] = *reinterpret_cast<const f32x4*>(from + 8 * c);
  }
  const char* const kbase = reinterpret_cast<const char*>(static_cast<const float*>(a.k.ptr) + rk.begin * a.k.sl + hk * a.k.sh);
  const char* const vbase = reinterpret_cast<const char*>(static_cast<const float*>(a.v.ptr) + rk.begin * a.v.sl + hk * a.v.sh);
  const int ksl = (int)a.k.sl * 4, vsl = (int)a.v.sl * 4;        // 128 rows span less than 2^31 bytes
  const float c2 = a.scale_log2;

  float M = kNoReference, l = 0.f;
  f32x16 o[kTiles];
#pragma unroll
  for (int e = 0; e < kTiles; ++e)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[e][x] = 0.f;
  f32x4 kr[kSteps];
  Cols vr[16];

  // Buffer loads: a 32-bit offset a lane where a flat load takes a 64-bit address. Keys behind the end repeat the last one (their
  // logits are masked).
  auto rsrc_at = [&](const char* base, int64_t sl, int sub) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base + (int64_t)sub * 32 * sl * 4), 0, 0x7fffffff, 0x00020000);
  };
  struct KFrom {
    __amdgpu_buffer_rsrc_t rsrc;
    int off;
    __device__ __forceinline__ f32x4 chunk(int c) const { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + 32 * c, 0, 0)); }
  };
  auto k_from = [&](int sub) {
    const int left = m - 1 - 32 * sub, row = i < left ? i : left;
    return KFrom{rsrc_at(kbase, a.k.sl, sub), row * ksl + 16 * g};
  };
  auto v_row = [&](const __amdgpu_buffer_rsrc_t& from, int sub, int x) -> Cols {
    const int left = m - 1 - 32 * sub, key = 8 * (x >> 2) + (x & 3) + 4 * g, row = key < left ? key : left;
    const int off = row * vsl + i * 4 * kTiles;
    if constexpr (kTiles == 4) return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, off, 0, 0));
    else return __builtin_bit_cast(f32x2f, __builtin_amdgcn_raw_buffer_load_b64(from, off, 0, 0));
  };
  // logits to probabilities; reference and sum with them
  auto softmax = [&](f32x16& s, int k0) {
    const int left = bound - k0 - 4 * g;                          // keys 8 (x / 4) + x % 4 (+ 4 g) below it are seen
    float top = -__builtin_inff();
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      s[x] = 8 * (x >> 2) + (x & 3) < left ? s[x] * c2 : -__builtin_inff();
      top = fmaxf(top, s[x]);
    }
    if (__builtin_amdgcn_ballot_w64(top > M + kSlack) != 0) {
      const float Mn = fmaxf(M, pair_max_f(top)), alpha = __builtin_amdgcn_exp2f(M - Mn);
      M = Mn;
      l *= alpha;
#pragma unroll
      for (int e = 0; e < kTiles; ++e)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[e][x] *= alpha;
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      s[x] = __builtin_amdgcn_exp2f(s[x] - M);
      l += s[x];
    }
  };
  auto step = [&](auto more, int sub) {
    constexpr bool kMore = decltype(more)::value;
    const int k0 = 32 * sub;
    const KFrom k_next = k_from(kMore ? sub + 4 : sub);
    f32x4 q = q_lds[0][lane];
    f32x16 s;
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
      const f32x4 q_next = q_lds[c + 1 < kSteps ? c + 1 : 0][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kr[c][e], q[e], s, 0, 0, 0);
      q = q_next;
      __builtin_amdgcn_sched_barrier(0);  // one read ahead, not all; and a reload behind its fragment's last use takes its registers
      if (kMore) kr[c] = k_next.chunk(c);
    }
    __builtin_amdgcn_sched_barrier(0);
    softmax(s, k0);
    const __amdgpu_buffer_rsrc_t v_next = rsrc_at(vbase, a.v.sl, kMore ? sub + 4 : sub);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
#pragma unroll
      for (int e = 0; e < kTiles; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[x][e], s[x], o[e], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (kMore) vr[x] = v_row(v_next, sub + 4, x);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  if (wave < subs) {
    const KFrom k_first = k_from(wave);
    const __amdgpu_buffer_rsrc_t v_first = rsrc_at(vbase, a.v.sl, wave);
#pragma unroll
    for (int c = 0; c < kSteps; ++c) kr[c] = k_first.chunk(c);
#pragma unroll
    for (int x = 0; x < 16; ++x) vr[x] = v_row(v_first, wave, x);
  }
  __syncthreads();
  if (wave < subs) {
    int sub = wave;
    for (; sub + 4 < subs; sub += 4) step(More{}, sub);
    step(Last{}, sub);
  }

  // 0 times what V holds at a hidden key is not 0 if that is infinite or NaN. A wave whose part is not finite looks for such a
  // value behind its first row's bound, and with one does its share again: the product of a sub-tile that not all rows see is then formed
  // for every bound among them, from V zeroed behind it, and taken by the rows that have it.
  {
    float worst = 0.f;  // NaN if a value is infinite or not a number
#pragma unroll
    for (int e = 0; e < kTiles; ++e)
#pragma unroll
      for (int x = 0; x < 16; ++x) worst = __builtin_fmaf(o[e][x], 0.f, worst);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(worst == 0.f)) != 0, 0)) {
      bool odd = false;
      const int from = 32 * subs > m && least > m - 1 ? m - 1 : least;  // behind the last key that repeats
      for (int key = from + g; key < 32 * subs && key < m; key += 2)
        for (int d = i; d < D; d += 32) odd = odd || !(fabsf(*reinterpret_cast<const float*>(vbase + (int64_t)key * a.v.sl * 4 + 4 * d)) < __builtin_inff());
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
        M = kNoReference;
        l = 0.f;
#pragma unroll
        for (int e = 0; e < kTiles; ++e)
#pragma unroll
          for (int x = 0; x < 16; ++x) o[e][x] = 0.f;
#pragma unroll 1
        for (int sub = wave; sub < subs; sub += 4) {
          const int k0 = 32 * sub;
          const KFrom k = k_from(sub);
          f32x16 s;
#pragma unroll
          for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll 1
          for (int c = 0; c < kSteps; ++c) {
            const f32x4 kc = k.chunk(c), q = q_lds[c][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kc[e], q[e], s, 0, 0, 0);
          }
          softmax(s, k0);
#pragma unroll 1
          for (int b = k0 + 32 <= least ? 32 : 1; b <= 32; ++b) {
            const bool has = k0 + 32 <= least || (bound - k0 < 32 ? bound - k0 : 32) == b;
            if (__builtin_amdgcn_ballot_w64(has) == 0) continue;
            const __amdgpu_buffer_rsrc_t v = rsrc_at(vbase, a.v.sl, sub);
            f32x16 add[kTiles];
#pragma unroll
            for (int e = 0; e < kTiles; ++e)
#pragma unroll
              for (int x = 0; x < 16; ++x) add[e][x] = 0.f;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              const Cols row = v_row(v, sub, x);
#pragma unroll
              for (int e = 0; e < kTiles; ++e)
                add[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(8 * (x >> 2) + (x & 3) + 4 * g < b ? row[e] : 0.f, s[x], add[e], 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < kTiles; ++e)
#pragma unroll
              for (int x = 0; x < 16; ++x) o[e][x] += has ? add[e][x] : 0.f;
          }
        }
      }
    }
  }
  const float sum = pair_sum_f(l);
  __syncthreads();  // Q has been read for the last time
  if (g == 0) {
    refs[wave][i] = M;
    sums[wave][i] = sum;
  }
  // row 8 (x / 4) + 4 g + x % 4 of output tile e is column kTiles times that, + e; 16-byte slot c of row i at c ^ (i % 16)
#pragma unroll
  for (int x = 0; x < 16; ++x) {
    const int r = 8 * (x >> 2) + 4 * g + (x & 3);
    float* const to = &stage[wave][i][0];
    if constexpr (kTiles == 4) {
      *reinterpret_cast<f32x4*>(to + 4 * (r ^ (i & 15))) = f32x4{o[0][x], o[1][x], o[2][x], o[3][x]};
    } else {
      *reinterpret_cast<f32x2f*>(to + 4 * ((r >> 1) ^ (i & 15)) + 2 * (r & 1)) = f32x2f{o[0][x], o[1][x]};
    }
  }
  __syncthreads();
  // a thread: slots x, x + 8, ... of one row
  const int r = threadIdx.x >> 3, x = threadIdx.x & 7;
  if (row0 + r >= n_rows) return;
  float Mr = refs[0][r];
#pragma unroll
  for (int w = 1; w < 4; ++w) Mr = fmaxf(Mr, refs[w][r]);
  float lr = 0.f, f[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = __builtin_amdgcn_exp2f(refs[w][r] - Mr);
    lr += sums[w][r] * f[w];
  }
  const float inv = lr == 0.f ? 0.f : 1.f / lr;
  float* const to = static_cast<float*>(a.o) + (int64_t)(rq.begin + row0 + r) * a.o_sl + h * a.o_sh;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) acc += *reinterpret_cast<const f32x4*>(&stage[w][r][4 * ((8 * c + x) ^ (r & 15))]) * f[w];
    *reinterpret_cast<f32x4*>(to + 4 * (8 * c + x)) = acc * inv;
  }
  if (a.lse != nullptr && x == 0)
    a.lse[(int64_t)h * a.Tq + rq.begin + row0 + r] = lr == 0.f ? -__builtin_inff() : (Mr + __builtin_amdgcn_logf(lr)) * 0.6931471805599453f;
#endif
}

// Calls of few rows take 16 a work-group (attn_paged.hip), which is as long as half the longest row's products; with more, every key
// passes through a compute unit's registers twice as often. us, 32 rows -> 16: 8 heads of 128 over 300 tokens 18.5 -> 10.7, 1000
// 39.8 -> 33.9, 2000 101 -> 98, 4096 295 -> 337; 32 over 300 23.7 -> 18.7, 600 40.9 -> 47.5; 8 of 64 over 300 11.4 -> 7.7, 2000 56 -> 51, 2500
// 72 -> 74, 4096 162 -> 171. Batches whose sequences are all as long turn earlier (2 of 1000, 8 heads of 128 56 -> 69; 4 of 500, 8 of 64
// 19.5 -> 24.2, 6 of 300 17.4 -> 14.5). And up to 8 tokens a sequence: 256 prompts of 8, 32 heads of 128 179 -> 81, 28/4 heads 151 -> 39.
hipError_t launch_prompt_f32(int D, const PromptArgs& a, hipStream_t s) {
  if (few_rows(false, D, a)) return launch_prompt_few_rows_f32(D, a, s);
  const int64_t groups = ((int64_t)a.Tq / 32 + (a.n_seqs < a.Tq ? a.n_seqs : a.Tq)) * a.Hq;
  if (!grid_fits(groups, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)groups), block(256);
  if (D == 128) hipLaunchKernelGGL((prompt_f32_kernel<128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((prompt_f32_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace sparsed
