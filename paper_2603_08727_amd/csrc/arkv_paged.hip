// Rows of a paged cache: rotary positions on the way in (k_paged_append), and eviction by collected weight
// (k_evict_select, k_evict_move).
#include <algorithm>

#include "arkv_dev.h"
#include "arkv_paged_dev.h"

namespace arkv {

typedef uint32_t u32x4p __attribute__((ext_vector_type(4)));   // a 16-byte chunk the compiler keeps in registers

template <typename T> struct Half2 { typedef T type __attribute__((ext_vector_type(2))); };

template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w) {
  const auto h = __builtin_bit_cast(typename Half2<T>::type, w);
  return make_float2((float)h[0], (float)h[1]);
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b) {   // one rounding to nearest even each
  typename Half2<T>::type h;
  h[0] = (T)a; h[1] = (T)b;
  return __builtin_bit_cast(uint32_t, h);
}

// Sequence of token t: how many sequences end at or before it.  Lanes look at 64 ends at a time.
__device__ __forceinline__ int find_seq(const int32_t* cu_q, int B, int t, int lane) {
  int b = 0;
  for (int i = 0; i < B; i += 64) b += __popcll(__ballot(i + lane < B && cu_q[min(i + lane, B - 1) + 1] <= t));
  return b;
}

constexpr int kAppendWaves = 4;

// One wave per new token.  The wave's lanes form the token's angles (position times frequency in turns, in 64 bits: at
// position 2^17 a 32-bit product is off by up to 2^-8 turns; the fraction that is left fits 32), then walk its heads'
// 16-byte chunks in pairs: item i of a row is the pair of chunks whose channels turn together.
template <typename T, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void k_paged_append(AppendArgs A) {
  __shared__ float2 turn[kAppendWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * kAppendWaves + wave;
  const Paged& P = A.P;
  if (t < P.N && lane < A.half) {
    const double turns = (double)A.positions[(size_t)A.axis[lane] * P.N + t] * (A.freq[lane] * 0.15915494309189533577);
    const float f = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.0f * f, &s, &c);
    turn[wave][lane] = make_float2(c, s);
  }
  __syncthreads();
  if (t >= P.N) return;
  const int b = find_seq(P.cu_q, P.B, t, lane);
  if (b >= P.B) return;
  const Seq s = clamp_seq(P.cu_q[b], P.cu_q[b + 1], P.kv_len[b], P.N, P.max_q, P.max_kv);
  if (t < s.q0 || t >= s.q0 + s.nq) return;
  const int slot = s.kv - s.nq + t - s.q0;
  const int row0 = slot_row(P.table + (size_t)b * P.width, P.n_pages, P.H, 0, P.lg_page, s.kv, slot);
  if (row0 >= 0)
    for (int h = lane; h < P.H; h += 64) {
      P.pos[(size_t)row0 + ((size_t)h << P.lg_page)] = A.positions[t];
      if (P.weight) P.weight[(size_t)row0 + ((size_t)h << P.lg_page)] = 0.f;
    }
  constexpr int IPR = D / 16;                       // items of a row
  const int Hr = A.Hq + P.H, rot = A.half / 8;      // heads that turn; items that turn
  const int n_items = (A.Hq + 2 * P.H) * IPR;
  for (int it = lane; it < n_items; it += 64) {
    const int h = it / IPR, i = it % IPR;
    const Rows& src = h < A.Hq ? A.q : h < Hr ? A.k : A.v;
    const int hs = h < A.Hq ? h : h < Hr ? h - A.Hq : h - Hr;
    T* to;
    if (h < A.Hq) to = (T*)A.q_out + ((size_t)t * A.Hq + h) * D;
    else {
      if (row0 < 0) continue;
      to = (T*)(h < Hr ? P.k : P.v) + ((size_t)row0 + ((size_t)hs << P.lg_page)) * D;
    }
    const T* from = (const T*)src.p + (size_t)t * src.ts + (size_t)hs * src.hs;
    // chunks of this item: with halves, chunk i turns with chunk i + rot; else (and behind rot_dim) two adjacent ones
    const bool turns = i < rot && h < Hr;
    const bool halves = i < rot && !A.adjacent;
    const int c0 = halves ? i : 2 * i, c1 = halves ? i + rot : 2 * i + 1;
    u32x4p x = *reinterpret_cast<const u32x4p*>(from + 8 * c0), y = *reinterpret_cast<const u32x4p*>(from + 8 * c1);
    if (turns) {
      if (!A.adjacent) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 a = unpack2<T>(x[e]), o = unpack2<T>(y[e]);
          const float2 t0 = turn[wave][8 * i + 2 * e], t1 = turn[wave][8 * i + 2 * e + 1];
          x[e] = pack2<T>(a.x * t0.x - o.x * t0.y, a.y * t1.x - o.y * t1.y);
          y[e] = pack2<T>(o.x * t0.x + a.x * t0.y, o.y * t1.x + a.y * t1.y);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 a = unpack2<T>(x[e]), o = unpack2<T>(y[e]);
          const float2 t0 = turn[wave][8 * i + e], t1 = turn[wave][8 * i + 4 + e];
          x[e] = pack2<T>(a.x * t0.x - a.y * t0.y, a.y * t0.x + a.x * t0.y);
          y[e] = pack2<T>(o.x * t1.x - o.y * t1.y, o.y * t1.x + o.x * t1.y);
        }
      }
    }
    *reinterpret_cast<u32x4p*>(to + 8 * c0) = x;
    *reinterpret_cast<u32x4p*>(to + 8 * c1) = y;
  }
}

hipError_t launch_paged_append(int dtype, int D, const AppendArgs& A, hipStream_t st) {
  const dim3 grid((A.P.N + kAppendWaves - 1) / kAppendWaves), block(64 * kAppendWaves);
  if (dtype == ARKV_DTYPE_BF16) {
    if (D == 64) k_paged_append<__bf16, 64><<<grid, block, 0, st>>>(A);
    else k_paged_append<__bf16, 128><<<grid, block, 0, st>>>(A);
  } else {
    if (D == 64) k_paged_append<_Float16, 64><<<grid, block, 0, st>>>(A);
    else k_paged_append<_Float16, 128><<<grid, block, 0, st>>>(A);
  }
  return hipGetLastError();
}

// ---- eviction -------------------------------------------------------------------------------------

constexpr int kEvictThreads = 1024;

// Order of weights as an order of words: NaN (and a row that is not there) lowest, -0 with +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (!(w == w)) return 0;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// What a unit keeps: m rows, the first `front` and the last `back` of n among them.
struct Kept { int n, m, front, back; };
__device__ __forceinline__ Kept kept_of(const EvictArgs& A, int b) {
  Kept k;
  k.n = min(max(A.P.kv_len[b], 0), A.P.max_kv);
  k.m = min(k.n, min(max(A.keep[b], 0), A.max_keep));
  k.front = min(A.sink, k.m);
  k.back = min(A.recent, k.m - k.front);
  return k;
}

// Which rows of a (sequence, kv-head) stay: one workgroup finds the weight of the last one by four passes over the
// weights, eight bits of their order each, then writes the survivors' slots in order.
__global__ __launch_bounds__(kEvictThreads) void k_evict_select(EvictArgs A) {
  __shared__ int hist[256];
  __shared__ int sums[2][kEvictThreads / 64];
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Kept K = kept_of(A, b);
  const int32_t* table = A.P.table + (size_t)b * A.P.width;
  int32_t* kept = A.kept + ((size_t)b * A.P.H + h) * A.max_keep;
  if (h == 0 && tid == 0) A.new_len[b] = K.m;
  const int lo = K.front, hi = K.n - K.back;          // ranked slots
  int need = K.m - K.front - K.back;
  auto key = [&](int j) {
    const int r = slot_row(table, A.P.n_pages, A.P.H, h, A.P.lg_page, K.n, j);
    return r < 0 ? 0u : weight_key(A.P.weight[r]);
  };
  uint32_t prefix = 0;                                 // the key of the last row that stays, digit by digit
  if (need > 0 && need < hi - lo) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += kEvictThreads) {
        const uint32_t x = key(j);
        if (shift == 24 || x >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[x >> shift & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int left = need, d = 255;
        for (; d > 0 && hist[d] < left; --d) left -= hist[d];
        s_prefix = prefix | (uint32_t)d << shift;
        s_need = left;
      }
      __syncthreads();
      prefix = s_prefix;
      need = s_need;                                   // rows of the prefix's digits that stay
      __syncthreads();
    }
  }
  const bool all = K.m - K.front - K.back >= hi - lo, none = K.m - K.front - K.back <= 0;
  int at = 0, ties = 0;                                // survivors and equal keys in front of this block of slots
  for (int j0 = 0; j0 < K.n; j0 += kEvictThreads) {
    const int j = j0 + tid;
    bool take = false, tie = false;
    if (j < K.n) {
      if (j < lo || j >= hi || all) take = true;
      else if (!none) {
        const uint32_t x = key(j);
        take = x > prefix;
        tie = x == prefix;
      }
    }
    const uint64_t below = (1ull << lane) - 1;
    const uint64_t tb = __ballot(tie);
    if (lane == 0) sums[0][wave] = __popcll(tb);
    __syncthreads();
    int before = ties;
    for (int w = 0; w < kEvictThreads / 64; ++w) {
      if (w < wave) before += sums[0][w];
      ties += sums[0][w];
    }
    if (tie && before + __popcll(tb & below) < need) take = true;
    const uint64_t kb = __ballot(take);
    if (lane == 0) sums[1][wave] = __popcll(kb);
    __syncthreads();
    int mine = at;
    for (int w = 0; w < kEvictThreads / 64; ++w) {
      if (w < wave) mine += sums[1][w];
      at += sums[1][w];
    }
    if (take) {
      mine += __popcll(kb & below);
      if (mine < A.max_keep) kept[mine] = j;
    }
    __syncthreads();
  }
  for (int i = K.m + tid; i < A.max_keep; i += kEvictThreads) kept[i] = -1;
}

// Copies the survivors to their new slots.  D / 8 lanes per row.
template <int D>
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs A) {
  constexpr int LPR = D / 8, RPW = 256 / LPR;
  const int h = blockIdx.y, b = blockIdx.z;
  const int i = blockIdx.x * RPW + threadIdx.x / LPR, c = threadIdx.x % LPR;
  const Kept K = kept_of(A, b);
  if (i >= K.m) return;
  const Paged& P = A.P;
  const int j = A.kept[((size_t)b * P.H + h) * A.max_keep + i];
  const int from = slot_row(P.table + (size_t)b * P.width, P.n_pages, P.H, h, P.lg_page, K.n, j);
  const int to = slot_row(A.dst_table + (size_t)b * A.dst_width, P.n_pages, P.H, h, P.lg_page, K.m, i);
  if (from < 0 || to < 0) return;
  const u32x4p* k = (const u32x4p*)P.k + (size_t)from * LPR + c;
  const u32x4p* v = (const u32x4p*)P.v + (size_t)from * LPR + c;
  const u32x4p x = *k, y = *v;
  ((u32x4p*)P.k)[(size_t)to * LPR + c] = x;
  ((u32x4p*)P.v)[(size_t)to * LPR + c] = y;
  if (c == 0) { P.pos[to] = P.pos[from]; P.weight[to] = P.weight[from]; }
}

hipError_t launch_paged_evict(int D, const EvictArgs& A, hipStream_t st) {
  k_evict_select<<<dim3(A.P.H, A.P.B), kEvictThreads, 0, st>>>(A);
  const int rows = std::min(A.max_keep, A.P.max_kv), rpw = 256 / (D / 8);
  if (rows > 0) {
    const dim3 grid((rows + rpw - 1) / rpw, A.P.H, A.P.B);
    if (D == 64) k_evict_move<64><<<grid, 256, 0, st>>>(A);
    else k_evict_move<128><<<grid, 256, 0, st>>>(A);
  }
  return hipGetLastError();
}

}  // namespace arkv
