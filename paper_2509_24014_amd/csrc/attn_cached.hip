// Attention of packed prompts and of newest tokens over a paged cache, one wave a row.
//
// A row (one query head of one token) sees the keys [0, n) of its sequence. A wave walks them 64 at a time: lane i takes
// the logit of key i (its K row against q from LDS), the wave the maximum; then lanes take columns and the 64 rows of V
// are added with their probabilities. Online softmax with a running maximum, everything in fp32. Keys that are not
// seen are never read, so nothing they hold matters.
#include "cache.hpp"

namespace sparsed {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return (float)x; }

template <typename T, int D, typename KeyRow, typename ValueRow>
__device__ __forceinline__ void attend_row(const T* q, int n, float scale_log2, float* q_lds, float* p_lds, int lane, KeyRow key_row,
                                           ValueRow value_row, float (&acc)[D / 64], float* m_out, float* l_out) {
  constexpr int kCols = D / 64;
  for (int c = 0; c < kCols; ++c) q_lds[c * 64 + lane] = to_f32(q[c * 64 + lane]);
  float M = -__builtin_inff(), l = 0.f;
  for (int c = 0; c < kCols; ++c) acc[c] = 0.f;
  for (int k0 = 0; k0 < n; k0 += 64) {
    const int here = n - k0 < 64 ? n - k0 : 64;
    float s = -__builtin_inff();
    if (lane < here) {
      const T* k = key_row(k0 + lane);
      float dot = 0.f;
      for (int d = 0; d < D; ++d) dot += to_f32(k[d]) * q_lds[d];
      s = dot * scale_log2;
    }
    float top = s;
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float Mn = fmaxf(M, top), ref = Mn == -__builtin_inff() ? 0.f : Mn;
    const float p = lane < here ? __builtin_amdgcn_exp2f(s - ref) : 0.f;
    const float alpha = __builtin_amdgcn_exp2f(M - ref);
    M = Mn;
    float part = p;
    for (int o = 32; o >= 1; o >>= 1) part += __shfl_xor(part, o, 64);
    l = l * alpha + part;
    p_lds[lane] = p;
    for (int c = 0; c < kCols; ++c) acc[c] *= alpha;
    for (int j = 0; j < here; ++j) {
      const T* v = value_row(k0 + j);
      for (int c = 0; c < kCols; ++c) acc[c] += p_lds[j] * to_f32(v[c * 64 + lane]);
    }
  }
  *m_out = M;
  *l_out = l;
}

template <typename T, int D>
__device__ __forceinline__ void store_row(T* o, float* lse, const float (&acc)[D / 64], float M, float l, int lane) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int c = 0; c < D / 64; ++c) o[c * 64 + lane] = (T)(acc[c] * inv);
  if (lse != nullptr && lane == 0) *lse = l == 0.f ? -__builtin_inff() : (M + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void attn_prompt_rows_kernel(const PromptArgs a) {
  __shared__ float q_lds[4][D];
  __shared__ float p_lds[4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  if (id >= (int64_t)a.Tq * a.Hq) return;
  const int t = (int)(id / a.Hq), h = (int)(id % a.Hq), hk = h / a.group;
  const int s = seq_of_row(a.cu_q, a.n_seqs, t);
  if (s >= a.n_seqs) return;
  const SeqRows rq = seq_rows(a.cu_q, s, a.Tq), rk = seq_rows(a.cu_k, s, a.Tk);
  if (t < rq.begin || t >= rq.end) return;
  const int m = rk.end - rk.begin;
  const int n = keys_seen(m - (rq.end - t), m, a.mask_block);
  const T* q = static_cast<const T*>(a.q.ptr) + t * a.q.sl + h * a.q.sh;
  const T* k = static_cast<const T*>(a.k.ptr) + rk.begin * a.k.sl + hk * a.k.sh;
  const T* v = static_cast<const T*>(a.v.ptr) + rk.begin * a.v.sl + hk * a.v.sh;
  float acc[D / 64], M, l;
  attend_row<T, D>(q, n, a.scale_log2, q_lds[wave], p_lds[wave], lane, [&](int j) { return k + j * a.k.sl; },
                   [&](int j) { return v + j * a.v.sl; }, acc, &M, &l);
  store_row<T, D>(static_cast<T*>(a.o) + t * a.o_sl + h * a.o_sh, a.lse ? a.lse + (int64_t)h * a.Tq + t : nullptr, acc, M, l, lane);
}

hipError_t launch_attn_prompt(bool bf16, int D, const PromptArgs& a, hipStream_t s) {
  if (bf16) return launch_prompt_bf16(D, a, s);
  const int64_t groups = ((int64_t)a.Tq * a.Hq + 3) / 4;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid((unsigned)groups), block(256);
  if (D == 128) hipLaunchKernelGGL((attn_prompt_rows_kernel<float, 128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((attn_prompt_rows_kernel<float, 64>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace sparsed
