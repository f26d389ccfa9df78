// Rows of packed pages: quantised on the way in, with rotary positions (k_packed_append), and read back (k_packed_read).
//
// A row's channels lie in blocks of 32 that share a power of two, 2^(s - 127): what a code stands for is exact in the rows' type, so the
// attention's conversion instructions, which take such scales, add no rounding.  s is the smallest with max|x| <= 448 (6) 2^(s - 127): none of a
// block saturates.  Codes are rounded once: keys are turned in 64 bits and go to 32 by rounding to odd, which leaves every later comparison and
// rounding to fewer bits as it would have been from 64.  What is left is the angle's own error: freq / 2 pi and its product with the position are rounded
// to 64 bits, 2^-51 of the angle, so that a key within that of a border between codes (1e-9 radians at 2^20, 1e-6 at 2^31) may get the next one.
#include <algorithm>
#include <type_traits>

#include "arkv_dev.h"
#include "arkv_paged_rows.h"

namespace arkv {

template <typename T> struct Limits;      // the largest finite magnitude, as a float's bits; scale bytes from `high` on put it at the type's top exponent
template <> struct Limits<__bf16> { static constexpr uint32_t top = 0x7F7F0000u; static constexpr int exponent = 254; };
template <> struct Limits<_Float16> { static constexpr uint32_t top = 0x477FE000u; static constexpr int exponent = 142; };

// x to 32 bits: where that is not exact, to the neighbour whose last bit is odd.
__device__ __forceinline__ float round_to_odd(double x) {
  const float f = (float)x;
  const double back = (double)f;
  if (back == x) return f;
  uint32_t u = __float_as_uint(f);
  if (fabs(back) > fabs(x)) --u;
  return __uint_as_float(u | 1);
}

// Quantises the eight channels of each of four adjacent lanes, which make a block: codes (BITS / 4 words), returns the scale byte.
template <typename T, int BITS> __device__ __forceinline__ uint32_t quantise(const float (&x)[8], uint32_t (&code)[BITS / 4]) {
  uint32_t most = 0, odd = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    if (u > Limits<T>::top) odd |= 1u << i;                        // not finite in T
    else most = max(most, u);
  }
  most = max(most, (uint32_t)__shfl_xor((int)most, 1));
  most = max(most, (uint32_t)__shfl_xor((int)most, 2));
  // (448 = 1.75 * 2^8, 6 = 1.5 * 2^2)
  constexpr int up = BITS == 8 ? 8 : 2;
  constexpr uint32_t mantissa = BITS == 8 ? 0x600000u : 0x400000u;
  const int s = max(1, (int)(most >> 23) - up + ((most & 0x7FFFFFu) > mantissa ? 1 : 0));
  // under the largest scale, codes above half of the format's top power of two are out of T's range
  const float lim = s > Limits<T>::exponent - up ? (BITS == 8 ? 240.f : 3.f) : (BITS == 8 ? 448.f : 6.f);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = fminf(fmaxf(ldexpf(x[i], 127 - s), -lim), lim);
    if (BITS == 8 && (odd >> i & 1)) y[i] = __uint_as_float(0x7FC00000u);
  }
  if constexpr (BITS == 8) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
      code[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], c, true);
    }
    return (uint32_t)s;
  } else {
    uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, y[0], y[1], 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.0f, 2);
    code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.0f, 3);
    odd |= (uint32_t)__shfl_xor((int)odd, 1);
    odd |= (uint32_t)__shfl_xor((int)odd, 2);
    return odd ? 255u : (uint32_t)s;
  }
}

constexpr int kPackWaves = 4;

// A token's sequence, its slot, and the sequence's rows.
struct Place { int b, slot, kv; };        // b < 0: a row of no sequence
// Of a wave's token, out of the lengths of 64 sequences (from `at` on, a lane each) that it holds already, and of those behind them.
__device__ __forceinline__ Place place_of(const Paged& P, int t, int lane, int sq0, int sq1, int skv) {
  for (int i = 0; i < P.B; i += 64) {
    if (i) {
      const int at = min(i + lane, P.B - 1);
      sq0 = P.cu_q[at]; sq1 = P.cu_q[at + 1]; skv = P.kv_len[at];
    }
    const uint64_t hit = __ballot(i + lane < P.B && sq1 > t);
    if (!hit) continue;
    const int l = __builtin_ctzll(hit);
    const Seq s = clamp_seq(__builtin_amdgcn_readlane(sq0, l), __builtin_amdgcn_readlane(sq1, l), __builtin_amdgcn_readlane(skv, l), P.N, P.max_q, P.max_kv);
    if (t < s.q0 || t >= s.q0 + s.nq) break;
    return {i + l, s.kv - s.nq + t - s.q0, s.kv};
  }
  return {-1, 0, 0};
}
__device__ __forceinline__ int row_of(const Paged& P, const Place& o) {
  return o.b < 0 ? -1 : slot_row(P.table + (size_t)o.b * P.width, P.n_pages, P.H, 0, P.lg_page, o.kv, o.slot);
}

// Rounds of 64 lanes that a wave has under way together: chunks of keys and values, and pairs of chunks of queries.
constexpr int kPackKv = 4, kPackQ = 3;
__host__ __device__ constexpr int kv_batches(int H, int D) { return (2 * H * (D / 8) + 64 * kPackKv - 1) / (64 * kPackKv); }
__host__ __device__ constexpr int q_batches(int Hq, int D) { return (Hq * (D / 16) + 64 * kPackQ - 1) / (64 * kPackQ); }

// One wave per new token, or a share of its batches.  Its lanes form the token's angles, then walk its keys and values a 16-byte chunk a lane (a key's
// partner chunk is read again: it comes out of the cache), so that four adjacent lanes hold a block, and its query heads in pairs of
// chunks whose channels turn together.  The first batch's rows are requested with the lengths and angles, the page behind them.  Many tokens are bound
// by memory (7817 tokens of 32 + 2 x 8 heads to 4 bits: 39 us, 4.3 TB/s), few by round trips (16 tokens: 5.6 us).
template <typename T, int D, int BITS>
__global__ __launch_bounds__(64 * kPackWaves) void k_packed_append(AppendArgs A, PackedArgs X, int per_wave) {
  __shared__ float2 turn[kPackWaves][64];
  __shared__ double2 turn64[kPackWaves][64];
  constexpr int CPR = D / 8, IPR = D / 16;                         // chunks, pairs of chunks of a row
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * kPackWaves + wave;
  const Paged& P = A.P;
  if (t >= P.N) return;
  const int rot = A.half / 8;                                      // pairs that turn
  const int n_kv = 2 * P.H * CPR, n_q = A.Hq * IPR, kvb = kv_batches(P.H, D), all = kvb + q_batches(A.Hq, D);
  const int first = (int)blockIdx.y * per_wave, last = min(first + per_wave, all);
  const int at0 = min(lane, P.B - 1);
  int sq0 = P.cu_q[at0], sq1 = P.cu_q[at0 + 1], skv = P.kv_len[at0];
  const int axis = A.axis[lane], pos0 = A.positions[t];
  const double freq = A.freq[min(lane, max(A.half, 1) - 1)];
  const int pos = A.positions[(size_t)min(axis, A.n_axes - 1) * P.N + t];
  int row0 = -1;
  bool placed = false;
  const T *qp = (const T*)A.q.p + (size_t)t * A.q.ts, *kp = (const T*)A.k.p + (size_t)t * A.k.ts, *vp = (const T*)A.v.p + (size_t)t * A.v.ts;
  // whether the token is a sequence's; what its rows turn by
  auto place = [&]() {
    asm volatile("" : "+v"(sq0), "+v"(sq1), "+v"(skv));            // (requested above, not where they turn out to be needed)
    const Place o = place_of(P, t, lane, sq0, sq1, skv);
    row0 = row_of(P, o);
    if (lane < A.half) {
      const double turns = (double)pos * (freq * 0.15915494309189533577), rest = turns - rint(turns);
      if (last > kvb) {
        float sn, cs;
        sincospif(2.0f * (float)rest, &sn, &cs);
        turn[wave][lane] = make_float2(cs, sn);                    // (read by this wave alone)
      }
      if (first < kvb) {
        double sn, cs;
        sincospi(2.0 * rest, &sn, &cs);
        turn64[wave][lane] = make_double2(cs, sn);
      }
    }
    placed = true;
    return o.b >= 0;
  };
  for (int batch = first; batch < min(last, kvb); ++batch) {
    const int it0 = batch * 64 * kPackKv + lane;
    u32x4g x[kPackKv], o[kPackKv];
#pragma unroll
    for (int u = 0; u < kPackKv; ++u) {
      const int it = min(it0 + 64 * u, n_kv - 1), h = it / CPR, c = it % CPR;
      const T* from = h < P.H ? kp + A.k.hs * h : vp + A.v.hs * (h - P.H);
      x[u] = *reinterpret_cast<const u32x4g*>(from + 8 * c);
      const int partner = h < P.H && !A.adjacent && c < 2 * rot ? (c < rot ? c + rot : c - rot) : c;
      o[u] = *reinterpret_cast<const u32x4g*>(from + 8 * partner);
    }
    if (!placed) {
      if (!place()) return;
      if (row0 >= 0 && batch == 0)
        for (int h = lane; h < P.H; h += 64) P.pos[(size_t)row0 + ((size_t)h << P.lg_page)] = pos0;
    }
    if (row0 < 0) continue;
#pragma unroll
    for (int u = 0; u < kPackKv; ++u) {
      const int it = it0 + 64 * u, h = it / CPR, c = it % CPR;     // (a block's four lanes are in or out together)
      if (it >= n_kv) continue;
      const bool key = h < P.H;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = Mfma<T>::get(x[u][e / 2], e & 1);
      if (key && c < 2 * rot) {
        if (A.adjacent) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const double2 w = turn64[wave][4 * c + e];
            const double a = y[2 * e], z = y[2 * e + 1];
            y[2 * e] = round_to_odd(fma(a, w.x, -(z * w.y)));
            y[2 * e + 1] = round_to_odd(fma(z, w.x, a * w.y));
          }
        } else {
          const bool front = c < rot;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const double2 w = turn64[wave][8 * (front ? c : c - rot) + e];
            const double z = Mfma<T>::get(o[u][e / 2], e & 1);
            y[e] = round_to_odd(fma((double)y[e], w.x, front ? -(z * w.y) : z * w.y));
          }
        }
      }
      uint32_t code[BITS / 4];
      const uint32_t s = quantise<T, BITS>(y, code);
      const size_t row = (size_t)row0 + ((size_t)(key ? h : h - P.H) << P.lg_page);
      uint8_t* to = (uint8_t*)(key ? P.k : P.v) + row * (D * BITS / 8) + c * BITS;
      if constexpr (BITS == 8) *reinterpret_cast<u32x2g*>(to) = u32x2g{code[0], code[1]};
      else *reinterpret_cast<uint32_t*>(to) = code[0];
      if ((c & 3) == 0) (key ? X.k_scale : X.v_scale)[row * (D / 32) + c / 4] = (uint8_t)s;
    }
  }
  for (int batch = max(first, kvb); batch < last; ++batch) {
    const int it0 = (batch - kvb) * 64 * kPackQ + lane;
    u32x4g x[kPackQ], y[kPackQ];
    // with halves, chunk i turns with chunk i + rot; else (and behind rot_dim) two adjacent ones
    auto chunk0 = [&](int i) { return i < rot && !A.adjacent ? i : 2 * i; };
    auto chunk1 = [&](int i) { return i < rot && !A.adjacent ? i + rot : 2 * i + 1; };
#pragma unroll
    for (int u = 0; u < kPackQ; ++u) {
      const int it = min(it0 + 64 * u, n_q - 1), h = it / IPR, i = it % IPR;
      x[u] = *reinterpret_cast<const u32x4g*>(qp + A.q.hs * h + 8 * chunk0(i));
      y[u] = *reinterpret_cast<const u32x4g*>(qp + A.q.hs * h + 8 * chunk1(i));
    }
    if (!placed && !place()) return;
#pragma unroll
    for (int u = 0; u < kPackQ; ++u) {
      const int it = it0 + 64 * u, h = it / IPR, i = it % IPR;
      if (it >= n_q) continue;
      if (i < rot) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float ax = Mfma<T>::get(x[u][e], 0), ay = Mfma<T>::get(x[u][e], 1), zx = Mfma<T>::get(y[u][e], 0), zy = Mfma<T>::get(y[u][e], 1);
          if (!A.adjacent) {
            const float2 t0 = turn[wave][8 * i + 2 * e], t1 = turn[wave][8 * i + 2 * e + 1];
            x[u][e] = Mfma<T>::pack(ax * t0.x - zx * t0.y, ay * t1.x - zy * t1.y);
            y[u][e] = Mfma<T>::pack(zx * t0.x + ax * t0.y, zy * t1.x + ay * t1.y);
          } else {
            const float2 t0 = turn[wave][8 * i + e], t1 = turn[wave][8 * i + 4 + e];
            x[u][e] = Mfma<T>::pack(ax * t0.x - ay * t0.y, ay * t0.x + ax * t0.y);
            y[u][e] = Mfma<T>::pack(zx * t1.x - zy * t1.y, zy * t1.x + zx * t1.y);
          }
        }
      }
      T* to = (T*)A.q_out + ((size_t)t * A.Hq + h) * D;
      *reinterpret_cast<u32x4g*>(to + 8 * chunk0(i)) = x[u];
      *reinterpret_cast<u32x4g*>(to + 8 * chunk1(i)) = y[u];
    }
  }
}

// One wave per token; a lane takes a chunk of codes at a time, up to kReadRounds of them under way.  Bound by memory where there are many (55591 rows of
// 8 x 128 channels, 8 bits: 77 us, 4.5 TB/s).  A token of 8 x 128 channels of 4 bits is one chunk a lane behind three round trips, and 7817 of them take
// 15 us where their bytes take 8.  Two changes were measured together, four tokens a wave and stores past the caches: 83 us, and 26; not each by itself.
constexpr int kReadRounds = 4;
template <typename T, int D, int BITS>
__global__ __launch_bounds__(64 * kPackWaves) void k_packed_read(Paged P, PackedArgs X) {
  typedef PoolRow<T, D, BITS> Row;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * kPackWaves + wave;
  if (t >= P.N) return;
  const int at0 = min(lane, P.B - 1);
  const Place o = place_of(P, t, lane, P.cu_q[at0], P.cu_q[at0 + 1], P.kv_len[at0]);
  if (o.b < 0) return;
  const int row0 = row_of(P, o), n = 2 * P.H * Row::kLanes;        // chunks of the token
  for (int it0 = lane; it0 < n; it0 += 64 * kReadRounds) {
    typename Row::Chunk chunk[kReadRounds];
    auto row = [&](int h) { return (size_t)row0 + ((size_t)(h < P.H ? h : h - P.H) << P.lg_page); };
#pragma unroll
    for (int u = 0; u < kReadRounds; ++u) {
      const int it = it0 + 64 * u, h = it / Row::kLanes, c = it % Row::kLanes;
      if (it < n && row0 >= 0) Row::load_chunk(h < P.H ? P.k : P.v, h < P.H ? X.k_scale : X.v_scale, row(h), c, chunk[u]);
    }
#pragma unroll
    for (int u = 0; u < kReadRounds; ++u) {
      const int it = it0 + 64 * u, h = it / Row::kLanes, c = it % Row::kLanes;
      T* out = h < P.H ? (T*)X.k : (T*)X.v;
      if (it >= n || !out) continue;
      u32x4g w[Row::kOut];
#pragma unroll
      for (int e = 0; e < Row::kOut; ++e) w[e] = u32x4g{0, 0, 0, 0};
      if (row0 >= 0) Row::expand(chunk[u], (int)row(h), c, w);
      u32x4g* to = reinterpret_cast<u32x4g*>(out + ((size_t)t * P.H + (h < P.H ? h : h - P.H)) * D) + Row::kOut * c;
#pragma unroll
      for (int e = 0; e < Row::kOut; ++e) to[e] = w[e];
    }
  }
}

template <typename F> static hipError_t dispatch_packed(int dtype, int D, int bits, F f) {
  auto by_bits = [&](auto t, auto d) { return bits == 8 ? f(t, d, Int<8>()) : f(t, d, Int<4>()); };
  auto by_dim = [&](auto t) { return D == 64 ? by_bits(t, Int<64>()) : by_bits(t, Int<128>()); };
  return dtype == ARKV_DTYPE_BF16 ? by_dim(TypeOf<__bf16>()) : by_dim(TypeOf<_Float16>());
}

hipError_t launch_packed_append(int dtype, int D, int bits, const AppendArgs& A, const PackedArgs& X, hipStream_t st) {
  // A wave takes two batches of a token where there are tokens for the whole chip, of fewer one (7817 tokens: 41 us by ones, 38 by twos, 39 by threes).
  const int all = kv_batches(A.P.H, D) + q_batches(A.Hq, D), per_wave = A.P.N >= 2048 ? 2 : 1;
  const dim3 grid((A.P.N + kPackWaves - 1) / kPackWaves, (all + per_wave - 1) / per_wave);
  return dispatch_packed(dtype, D, bits, [&](auto t, auto d, auto b) {
    k_packed_append<typename decltype(t)::type, decltype(d)::value, decltype(b)::value><<<grid, 64 * kPackWaves, 0, st>>>(A, X, per_wave);
    return hipGetLastError();
  });
}

hipError_t launch_packed_read(int dtype, int D, int bits, const Paged& P, const PackedArgs& X, hipStream_t st) {
  return dispatch_packed(dtype, D, bits, [&](auto t, auto d, auto b) {
    k_packed_read<typename decltype(t)::type, decltype(d)::value, decltype(b)::value><<<(P.N + kPackWaves - 1) / kPackWaves, 64 * kPackWaves, 0, st>>>(P, X);
    return hipGetLastError();
  });
}

}  // namespace arkv
