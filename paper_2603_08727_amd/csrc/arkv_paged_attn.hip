// Attention of new tokens over a paged cache, and the weight that the cached rows collect from them.
#include "arkv_dev.h"
#include "arkv_paged_dev.h"

namespace arkv {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ int find_seq(const int32_t* cu_q, int B, int t, int lane) {
  int b = 0;
  for (int i = 0; i < B; i += 64) b += __popcll(__ballot(i + lane < B && cu_q[min(i + lane, B - 1) + 1] <= t));
  return b;
}

// logit of a raw dot product (natural units)
__device__ __forceinline__ float logit_of(const Scores& S, float dot, float slope, int qp, int kp) {
  float x = dot * S.scale;
  if (S.cap > 0.f) x = S.cap * tanhf(x / S.cap);
  if (S.slopes) x -= slope * fabsf((float)(qp - kp));
  return x;
}

// One wave per (new token, query head): a lane per key, then a lane per channel.
template <typename T, int D>
__global__ __launch_bounds__(64) void k_paged_attn(PagedAttnArgs A) {
  __shared__ float qs[D];
  const Paged& P = A.P;
  const int lane = threadIdx.x, t = blockIdx.x, hq = blockIdx.y, h = hq / A.G;
  const int b = find_seq(P.cu_q, P.B, t, lane);
  if (b >= P.B) return;
  const Seq s = clamp_seq(P.cu_q[b], P.cu_q[b + 1], P.kv_len[b], P.N, P.max_q, P.max_kv);
  if (t < s.q0 || t >= s.q0 + s.nq) return;
  const T* q = (const T*)A.q.p + (size_t)t * A.q.ts + (size_t)hq * A.q.hs;
  for (int c = lane; c < D; c += 64) qs[c] = (float)q[c];
  __syncthreads();
  int end = s.kv - s.nq + t - s.q0 + 1;
  if (A.S.prefix) end = max(end, A.S.prefix[b]);
  end = min(end, s.kv);
  const float slope = A.S.slopes ? A.S.slopes[hq] : 0.f;
  const int qp = A.S.slopes ? A.S.q_pos[t] : 0;
  const int32_t* table = P.table + (size_t)b * P.width;
  float m = -INFINITY, l = 0.f, acc[D / 64] = {};
  for (int j0 = 0; j0 < end; j0 += 64) {
    const int j = j0 + lane;
    const int row = j < end ? slot_row(table, P.n_pages, P.H, h, P.lg_page, s.kv, j) : -1;
    float x = -INFINITY;
    if (row >= 0) {
      const T* k = (const T*)P.k + (size_t)row * D;
      float dot = 0.f;
      for (int c = 0; c < D; ++c) dot += qs[c] * (float)k[c];
      x = logit_of(A.S, dot, slope, qp, A.S.slopes ? P.pos[row] : 0);
    }
    const float mn = fmaxf(m, wave_max(x));
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float f = __expf(m - ref), p = row >= 0 ? __expf(x - ref) : 0.f;
    m = mn;
    l = l * f + wave_sum(p);
    for (int e = 0; e < D / 64; ++e) acc[e] *= f;
    for (int i = 0; i < 64; ++i) {
      const int r = __shfl(row, i);
      const float w = __shfl(p, i);
      if (r < 0) continue;
      for (int e = 0; e < D / 64; ++e) acc[e] += w * (float)((const T*)P.v)[(size_t)r * D + 64 * e + lane];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;          // (NaN stays)
  for (int e = 0; e < D / 64; ++e) ((T*)A.out)[((size_t)t * A.Hq + hq) * D + 64 * e + lane] = (T)(acc[e] * inv);
  if (A.lse && lane == 0) A.lse[(size_t)t * A.Hq + hq] = l == 0.f ? -INFINITY : m + __logf(l);
}

// One wave per 64 slots of a (sequence, kv-head): a lane per key, all query rows of the group in turn.
template <typename T, int D>
__global__ __launch_bounds__(64) void k_paged_weights(PagedAttnArgs A) {
  const Paged& P = A.P;
  const int h = blockIdx.y, b = blockIdx.z, j = blockIdx.x * 64 + threadIdx.x;
  const Seq s = clamp_seq(P.cu_q[b], P.cu_q[b + 1], P.kv_len[b], P.N, P.max_q, P.max_kv);
  const int row = slot_row(P.table + (size_t)b * P.width, P.n_pages, P.H, h, P.lg_page, s.kv, j);
  if (row < 0) return;
  const T* k = (const T*)P.k + (size_t)row * D;
  const int ctx = s.kv - s.nq, prefix = A.S.prefix ? A.S.prefix[b] : 0;
  const int kp = A.S.slopes ? P.pos[row] : 0;
  float sum = 0.f;
  for (int i = j < prefix ? 0 : max(0, j - ctx); i < s.nq; ++i) {
    const int t = s.q0 + i;
    for (int g = 0; g < A.G; ++g) {
      const int hq = h * A.G + g;
      const T* q = (const T*)A.q.p + (size_t)t * A.q.ts + (size_t)hq * A.q.hs;
      float dot = 0.f;
      for (int c = 0; c < D; ++c) dot += (float)q[c] * (float)k[c];
      const float x = logit_of(A.S, dot, A.S.slopes ? A.S.slopes[hq] : 0.f, A.S.slopes ? A.S.q_pos[t] : 0, kp);
      sum += expf(x - A.lse[(size_t)t * A.Hq + hq]);
    }
  }
  P.weight[row] = (A.decay == 0.f ? 0.f : A.decay * A.carried[row]) + sum;
}

size_t paged_attention_floats(const Paged&, int, int) { return 0; }

hipError_t launch_paged_attention(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  const dim3 grid(A.P.N, A.Hq);
  if (dtype == ARKV_DTYPE_BF16) {
    if (D == 64) k_paged_attn<__bf16, 64><<<grid, 64, 0, st>>>(A);
    else k_paged_attn<__bf16, 128><<<grid, 64, 0, st>>>(A);
  } else {
    if (D == 64) k_paged_attn<_Float16, 64><<<grid, 64, 0, st>>>(A);
    else k_paged_attn<_Float16, 128><<<grid, 64, 0, st>>>(A);
  }
  return hipGetLastError();
}

hipError_t launch_paged_weights(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  const dim3 grid((A.P.max_kv + 63) / 64, A.P.H, A.P.B);
  if (dtype == ARKV_DTYPE_BF16) {
    if (D == 64) k_paged_weights<__bf16, 64><<<grid, 64, 0, st>>>(A);
    else k_paged_weights<__bf16, 128><<<grid, 64, 0, st>>>(A);
  } else {
    if (D == 64) k_paged_weights<_Float16, 64><<<grid, 64, 0, st>>>(A);
    else k_paged_weights<_Float16, 128><<<grid, 64, 0, st>>>(A);
  }
  return hipGetLastError();
}

}  // namespace arkv
