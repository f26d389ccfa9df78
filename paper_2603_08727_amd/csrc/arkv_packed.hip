// Rows of packed pages: quantised on the way in, with rotary positions (k_packed_append), and read back (k_packed_read).
//
// A row's channels lie in blocks of 32 that share a power of two, 2^(s - 127): what a code stands for is exact in the rows' type, so the
// attention's conversion instructions, which take such scales, add no rounding.  s is the smallest with max|x| <= 448 (6) 2^(s - 127): none of a
// block saturates.  Codes are rounded once: keys are turned in 64 bits and go to 32 by rounding to odd, which leaves every later comparison and
// rounding to fewer bits as it would have been from 64.
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

// The sequence of token t (of the wave), its new tokens' first row and their number, the token's slot; b < 0: none.
struct Place { int b, slot, row0; };      // row0: its row of kv-head 0, -1: none
__device__ __forceinline__ Place place_of(const Paged& P, int t, int lane) {
  Place o = {-1, 0, -1};
  for (int i = 0; i < P.B; i += 64) {
    const int at = min(i + lane, P.B - 1);
    const int sq0 = P.cu_q[at], sq1 = P.cu_q[at + 1], skv = P.kv_len[at];
    const uint64_t hit = __ballot(i + lane < P.B && sq1 > t);
    if (!hit) continue;
    const int l = __builtin_ctzll(hit);
    const Seq s = clamp_seq(__builtin_amdgcn_readlane(sq0, l), __builtin_amdgcn_readlane(sq1, l), __builtin_amdgcn_readlane(skv, l), P.N, P.max_q, P.max_kv);
    if (t < s.q0 || t >= s.q0 + s.nq) return o;                    // a row of no sequence
    o.b = i + l;
    o.slot = s.kv - s.nq + t - s.q0;
    o.row0 = slot_row(P.table + (size_t)o.b * P.width, P.n_pages, P.H, 0, P.lg_page, s.kv, o.slot);
    return o;
  }
  return o;
}

// One wave per new token.  Its lanes form the token's angles, then walk its query heads in pairs of 16-byte chunks whose channels turn
// together, and its keys and values a chunk a lane (a key's partner chunk is read again: it comes out of the cache), so that four
// adjacent lanes hold a block.
template <typename T, int D, int BITS>
__global__ __launch_bounds__(64 * kPackWaves) void k_packed_append(AppendArgs A, PackedArgs X) {
  __shared__ float2 turn[kPackWaves][64];
  __shared__ double2 turn64[kPackWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * kPackWaves + wave;
  const Paged& P = A.P;
  if (t >= P.N) return;
  const Place place = place_of(P, t, lane);
  if (place.b < 0) return;
  const int row0 = place.row0;
  if (lane < A.half) {
    const double turns = (double)A.positions[(size_t)A.axis[lane] * P.N + t] * (A.freq[lane] * 0.15915494309189533577);
    const double rest = turns - rint(turns);
    float sn, cs;
    sincospif(2.0f * (float)rest, &sn, &cs);
    turn[wave][lane] = make_float2(cs, sn);                        // (read by this wave alone)
    double sn64, cs64;
    sincospi(2.0 * rest, &sn64, &cs64);
    turn64[wave][lane] = make_double2(cs64, sn64);
  }
  constexpr int CPR = D / 8, IPR = D / 16;                         // chunks, pairs of chunks of a row
  const int rot = A.half / 8;                                      // pairs that turn
  for (int it = lane; it < A.Hq * IPR; it += 64) {
    const int h = it / IPR, i = it % IPR;
    const bool turns = i < rot, halves = turns && !A.adjacent;
    const int c0 = halves ? i : 2 * i, c1 = halves ? i + rot : 2 * i + 1;
    const T* from = (const T*)A.q.p + (size_t)t * A.q.ts + A.q.hs * h;
    u32x4g x = *reinterpret_cast<const u32x4g*>(from + 8 * c0), y = *reinterpret_cast<const u32x4g*>(from + 8 * c1);
    if (turns) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float ax = Mfma<T>::get(x[e], 0), ay = Mfma<T>::get(x[e], 1), zx = Mfma<T>::get(y[e], 0), zy = Mfma<T>::get(y[e], 1);
        if (!A.adjacent) {
          const float2 t0 = turn[wave][8 * i + 2 * e], t1 = turn[wave][8 * i + 2 * e + 1];
          x[e] = Mfma<T>::pack(ax * t0.x - zx * t0.y, ay * t1.x - zy * t1.y);
          y[e] = Mfma<T>::pack(zx * t0.x + ax * t0.y, zy * t1.x + ay * t1.y);
        } else {
          const float2 t0 = turn[wave][8 * i + e], t1 = turn[wave][8 * i + 4 + e];
          x[e] = Mfma<T>::pack(ax * t0.x - ay * t0.y, ay * t0.x + ax * t0.y);
          y[e] = Mfma<T>::pack(zx * t1.x - zy * t1.y, zy * t1.x + zx * t1.y);
        }
      }
    }
    T* to = (T*)A.q_out + ((size_t)t * A.Hq + h) * D;
    *reinterpret_cast<u32x4g*>(to + 8 * c0) = x;
    *reinterpret_cast<u32x4g*>(to + 8 * c1) = y;
  }
  if (row0 < 0) return;
  for (int h = lane; h < P.H; h += 64) P.pos[(size_t)row0 + ((size_t)h << P.lg_page)] = A.positions[t];
  for (int it = lane; it < 2 * P.H * CPR; it += 64) {              // (whole blocks: CPR is a multiple of 4)
    const int h = it / CPR, c = it % CPR, hs = h < P.H ? h : h - P.H;
    const bool key = h < P.H;
    const T* from = key ? (const T*)A.k.p + (size_t)t * A.k.ts + A.k.hs * hs : (const T*)A.v.p + (size_t)t * A.v.ts + A.v.hs * hs;
    const u32x4g x = *reinterpret_cast<const u32x4g*>(from + 8 * c);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = Mfma<T>::get(x[e / 2], e & 1);
    if (key && c < 2 * rot) {
      if (A.adjacent) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double2 u = turn64[wave][4 * c + e];
          const double a = y[2 * e], z = y[2 * e + 1];
          y[2 * e] = round_to_odd(fma(a, u.x, -(z * u.y)));
          y[2 * e + 1] = round_to_odd(fma(z, u.x, a * u.y));
        }
      } else {
        const bool first = c < rot;
        const u32x4g o = *reinterpret_cast<const u32x4g*>(from + 8 * (first ? c + rot : c - rot));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double2 u = turn64[wave][8 * (first ? c : c - rot) + e];
          const double z = Mfma<T>::get(o[e / 2], e & 1);
          y[e] = round_to_odd(fma((double)y[e], u.x, first ? -(z * u.y) : z * u.y));
        }
      }
    }
    uint32_t code[BITS / 4];
    const uint32_t s = quantise<T, BITS>(y, code);
    const size_t row = (size_t)row0 + ((size_t)hs << P.lg_page);
    uint8_t* to = (uint8_t*)(key ? P.k : P.v) + row * (D * BITS / 8) + c * BITS;
    if constexpr (BITS == 8) *reinterpret_cast<u32x2g*>(to) = u32x2g{code[0], code[1]};
    else *reinterpret_cast<uint32_t*>(to) = code[0];
    if ((c & 3) == 0) (key ? X.k_scale : X.v_scale)[row * (D / 32) + c / 4] = (uint8_t)s;
  }
}

// One wave per token: a lane takes a chunk of codes at a time.
template <typename T, int D, int BITS>
__global__ __launch_bounds__(64 * kPackWaves) void k_packed_read(Paged P, PackedArgs X) {
  typedef PoolRow<T, D, BITS> Row;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * kPackWaves + wave;
  if (t >= P.N) return;
  const Place place = place_of(P, t, lane);
  if (place.b < 0) return;
  for (int it = lane; it < 2 * P.H * Row::kLanes; it += 64) {
    const int h = it / Row::kLanes, c = it % Row::kLanes, hs = h < P.H ? h : h - P.H;
    const bool key = h < P.H;
    T* out = (T*)(key ? X.k : X.v);
    if (!out) continue;
    u32x4g w[Row::kOut];
    if (place.row0 >= 0) {
      typename Row::Chunk chunk;
      Row::load_chunk(key ? P.k : P.v, key ? X.k_scale : X.v_scale, (size_t)place.row0 + ((size_t)hs << P.lg_page), c, chunk);
      Row::expand(chunk, w);
    } else {
#pragma unroll
      for (int o = 0; o < Row::kOut; ++o) w[o] = u32x4g{0, 0, 0, 0};
    }
    u32x4g* to = reinterpret_cast<u32x4g*>(out + ((size_t)t * P.H + hs) * D) + Row::kOut * c;
#pragma unroll
    for (int o = 0; o < Row::kOut; ++o) to[o] = w[o];
  }
}

template <typename F> static hipError_t dispatch_packed(int dtype, int D, int bits, F f) {
  auto by_bits = [&](auto t, auto d) { return bits == 8 ? f(t, d, Int<8>()) : f(t, d, Int<4>()); };
  auto by_dim = [&](auto t) { return D == 64 ? by_bits(t, Int<64>()) : by_bits(t, Int<128>()); };
  return dtype == ARKV_DTYPE_BF16 ? by_dim(TypeOf<__bf16>()) : by_dim(TypeOf<_Float16>());
}

hipError_t launch_packed_append(int dtype, int D, int bits, const AppendArgs& A, const PackedArgs& X, hipStream_t st) {
  return dispatch_packed(dtype, D, bits, [&](auto t, auto d, auto b) {
    k_packed_append<typename decltype(t)::type, decltype(d)::value, decltype(b)::value><<<(A.P.N + kPackWaves - 1) / kPackWaves, 64 * kPackWaves, 0, st>>>(A, X);
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
