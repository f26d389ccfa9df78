// Device pieces that the attention over pages and the row weights share: MFMA by type, logits, rows' ends, loads to LDS.
#pragma once
#include <type_traits>

#include "arkv_dev.h"
#include "arkv_paged_dev.h"

namespace arkv {

template <int N> using Int = std::integral_constant<int, N>;

typedef uint32_t u32x4g __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2g __attribute__((ext_vector_type(2)));
typedef float f32x4g __attribute__((ext_vector_type(4)));
typedef float f32x16g __attribute__((ext_vector_type(16)));
typedef short s16x4g __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8g __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2g __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8g __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2g __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4g* lds_s16x4;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kUnset = -1.0e30f;      // softmax reference of a row that has seen nothing
constexpr float kSumLimit = 16384.0f;   // a lane's probabilities of a tile may sum to this before the reference moves

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
  static constexpr uint32_t kExp = 0x7F80u;      // exponent bits: all set = not finite
  static __device__ __forceinline__ f32x4g m16(u32x4g a, u32x4g b, f32x4g c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8g, a), __builtin_bit_cast(bf16x8g, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16g m32(u32x4g a, u32x4g b, f32x16g c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8g, a), __builtin_bit_cast(bf16x8g, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { bf16x2g h; h[0] = (__bf16)a; h[1] = (__bf16)b; return __builtin_bit_cast(uint32_t, h); }
  static __device__ __forceinline__ float get(uint32_t w, int hi) { return __uint_as_float(hi ? w & 0xFFFF0000u : w << 16); }
};
template <> struct Mfma<_Float16> {
  static constexpr uint32_t kExp = 0x7C00u;
  static __device__ __forceinline__ f32x4g m16(u32x4g a, u32x4g b, f32x4g c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8g, a), __builtin_bit_cast(f16x8g, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16g m32(u32x4g a, u32x4g b, f32x16g c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8g, a), __builtin_bit_cast(f16x8g, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { f16x2g h; h[0] = (_Float16)a; h[1] = (_Float16)b; return __builtin_bit_cast(uint32_t, h); }
  static __device__ __forceinline__ float get(uint32_t w, int hi) { return (float)__builtin_bit_cast(f16x2g, w)[hi]; }
};

// halves of w that are not finite, as a mask of whole halves
template <typename T> __device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return ((w & Mfma<T>::kExp) == Mfma<T>::kExp ? 0xFFFFu : 0u) | ((w >> 16 & Mfma<T>::kExp) == Mfma<T>::kExp ? 0xFFFF0000u : 0u);
}

// What the kernels are built for: bit 0 of MODE: scores have a cap, bit 1: a bias by distance, bit 2: a cap above kWideCap.
template <int MODE> struct Mode { static constexpr int cap = MODE & 4 ? 2 : MODE & 1; static constexpr bool dist = (MODE & 2) != 0; };
constexpr float kWideCap = 256.f;
inline int mode_of(const Scores& S) { return (S.cap > kWideCap ? 4 : S.cap > 0.f ? 1 : 0) | (S.slopes ? 2 : 0); }

// logit, times log2(e), of a raw dot product
struct Logit {
  float mul, inv_cap2, cap2, inv;     // scale log2(e); 2 log2(e) scale / cap; cap log2(e); scale / cap
  __device__ __forceinline__ Logit(const Scores& S) {
    mul = S.scale * kLog2e;
    cap2 = S.cap * kLog2e;
    inv = S.cap > 0.f ? S.scale / S.cap : 0.f;
    inv_cap2 = 2.f * kLog2e * inv;
  }
  // the logit less ref.  CAP 1: tanh u = 1 - 2 / (1 + e^2u), which is off by a few 2^-24 of 1, the logit by 2^-22 of the cap, in absolute
  // terms: 2^-14 at kWideCap.  CAP 2: a larger cap would drown small logits in that, so where |u| < 1 / 8 its series takes over (the first
  // term left out is u^8 / 46 of u, below 2^-24), and the logit is off by 2^-19 of itself at most.
  template <int CAP> __device__ __forceinline__ float above(float dot, float ref) const {
    if (CAP == 0) return fmaf(dot, mul, -ref);
    const float y = fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(1.f + exp2_hw(dot * inv_cap2)), cap2 - ref);
    if (CAP == 1) return y;
    const float u = dot * inv, w = u * u;
    return fabsf(u) < 0.125f ? fmaf(dot * mul, fmaf(w, fmaf(w, fmaf(w, -17.f / 315.f, 2.f / 15.f), -1.f / 3.f), 1.f), -ref) : y;
  }
  template <int CAP> __device__ __forceinline__ float logit(float dot) const { return CAP ? above<CAP>(dot, 0.f) : dot * mul; }
};

// Keeps a rare branch a branch: what depends on the result is not computed in front of it (the compiler would compute a tile's masks
// for every tile, and select).
__device__ __forceinline__ uint32_t opaque(uint32_t x) { asm volatile("" : "+v"(x)); return x; }

__device__ __forceinline__ Seq seq_of(const Paged& P, int b) {
  return clamp_seq(P.cu_q[b], P.cu_q[b + 1], P.kv_len[b], P.N, P.max_q, P.max_kv);
}
// slots that new token i of a sequence sees are those below this (0: none)
__device__ __forceinline__ int row_end(const Seq& s, int i, int prefix) { return max(0, min(s.kv, max(s.kv - s.nq + i + 1, prefix))); }

constexpr int kStepRows = 16;           // rows of a sequence that the step kernels take

// Which kernels a launch needs.  few: sequences of up to so many rows are the step kernel's; -1 where only the other one is
// launched, which then takes all of them.
struct Which { bool step, chunk; int few; };
inline Which which_kernels(const Paged& P, int Hq) {
  Which w;
  w.chunk = (long long)P.max_q * (Hq / P.H) > kStepRows;
  w.step = !w.chunk || (long long)P.B * P.max_q != P.N;            // else all sequences have max_q new tokens: one launch will do
  w.few = w.step ? kStepRows : -1;
  return w;
}

// 1 KB from memory to LDS, 16 bytes per lane, in lane order from `lds` on, without a register in between.  The caller waits
// (vm_wait) and synchronises before anyone reads.  Inline assembly, because the compiler would wait for every such load in
// front of any LDS read; it has no output register.
__device__ __forceinline__ void load_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0" : : "s"(base), "v"(off), "s"(lds) : "memory");
}
// the same from an address per lane, 4 and 16 bytes
__device__ __forceinline__ void load_lds4(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(p), "s"(lds) : "memory");
}
__device__ __forceinline__ void load_lds16(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds) : "memory");
}
__device__ __forceinline__ void vm_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Where the 16-byte chunk c of a row lies in LDS, so that operand reads (one chunk of 32 rows) meet in a bank no more often
// than they must.
template <int D> __device__ __forceinline__ int k_chunk(int row, int c) { return D == 128 ? c ^ (row & 15) : c ^ (row >> 1 & 7); }

// f(type, head dimension, mode) as compile-time values
template <typename T> struct TypeOf { typedef T type; };
template <typename T, int D, typename F> hipError_t dispatch_mode(int mode, F f) {
  switch (mode) {
    case 0: return f(TypeOf<T>(), Int<D>(), Int<0>());
    case 1: return f(TypeOf<T>(), Int<D>(), Int<1>());
    case 2: return f(TypeOf<T>(), Int<D>(), Int<2>());
    case 3: return f(TypeOf<T>(), Int<D>(), Int<3>());
    case 4: return f(TypeOf<T>(), Int<D>(), Int<4>());
    default: return f(TypeOf<T>(), Int<D>(), Int<6>());
  }
}
template <typename F> hipError_t dispatch(int dtype, int D, int mode, F f) {
  if (dtype == ARKV_DTYPE_BF16) return D == 64 ? dispatch_mode<__bf16, 64>(mode, f) : dispatch_mode<__bf16, 128>(mode, f);
  return D == 64 ? dispatch_mode<_Float16, 64>(mode, f) : dispatch_mode<_Float16, 128>(mode, f);
}

}  // namespace arkv
