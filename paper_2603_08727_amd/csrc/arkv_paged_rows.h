// What the attention over pages is built from: how a pool holds its rows (16 bits, or packed), and which of them a token sees.
// A block of 32 channels has a scale of its own, a power of two, which the conversion instructions (v_cvt_scalef32_pk_*, two channels in about five
// cycles of a SIMD) apply as they expand the codes: the products run on 16-bit operands that are exactly the rows' values.
// Under a window a workgroup's keys are numbered without the granules that none of its tokens sees, so that its pieces, tiles and loads know of no
// gap: 16 requests of 19000 to 32768 rows under a window of 4096 take 53 us, 5.1 TB/s of what they see.  Masks are worked out for the tiles that
// need them alone, 16 slots at a time, as bits.
#pragma once
#include "arkv_paged_mma.h"

namespace arkv {

// ---- rows of a pool -------------------------------------------------------------------------------

// Two channels of a packed word, as T: its bits fit T, so nothing is rounded.  BITS 8: part 0, 1; 4: 0 to 3.
template <typename T, int BITS, int PART> __device__ __forceinline__ uint32_t unpack(uint32_t w, float scale) {
  if constexpr (BITS == 8) {
    if constexpr (std::is_same<T, __bf16>::value) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, PART));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, PART));
  } else {
    if constexpr (std::is_same<T, __bf16>::value) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, PART));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, PART));
  }
}
// eight channels of BITS / 4 words
template <typename T, int BITS> __device__ __forceinline__ u32x4g unpack8(const uint32_t* w, float scale) {
  if constexpr (BITS == 8) return u32x4g{unpack<T, 8, 0>(w[0], scale), unpack<T, 8, 1>(w[0], scale), unpack<T, 8, 0>(w[1], scale), unpack<T, 8, 1>(w[1], scale)};
  else return u32x4g{unpack<T, 4, 0>(w[0], scale), unpack<T, 4, 1>(w[0], scale), unpack<T, 4, 2>(w[0], scale), unpack<T, 4, 3>(w[0], scale)};
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }   // (0: 2^-127, 255: NaN, to the conversion)

// A row of D channels.  A chunk is what one lane loads of it at a time (kLanes of them a row), kOut times eight channels.  The logits'
// contraction may run over the channels in any order that q follows: channel() is the first of the eight that lane group gq
// (of four) takes in k-step kk, so that a lane's keys are whole chunks.  Scale bytes are loaded as words, those of one row (D = 128) or of two,
// and shifted where they are used: a byte would be cut out where it arrives, at the end of a loop, and waited for there.
template <typename T, int D, int BITS> struct PoolRow {
  static constexpr int kRow = D * BITS / 8, kBytes = kRow / 4 < 16 ? kRow / 4 : 16, kWords = kBytes / 4;
  static constexpr int kLanes = kRow / kBytes, kOut = kBytes / BITS, kParts = kRow / 4 / kBytes;
  struct Chunk { uint32_t w[kWords], scales; };
  struct Keys { uint32_t w[kParts * kWords], scales; };
  static __device__ __forceinline__ uint32_t scales_of(const uint8_t* scale, size_t row) {
    return *reinterpret_cast<const uint32_t*>(scale + (D == 128 ? 4 * row : 2 * (row & ~(size_t)1)));
  }
  static __device__ __forceinline__ float scale(uint32_t scales, int row, int channel) {
    return scale_of(scales >> (8 * (channel / 32) + (D == 128 ? 0 : 16 * (row & 1))) & 255);
  }
  static __device__ __forceinline__ int channel(int gq, int kk) { return kk / kOut * (32 * kOut) + gq * (8 * kOut) + 8 * (kk % kOut); }
  static __device__ __forceinline__ void load(const uint8_t* p, uint32_t* w) {
    if constexpr (kBytes == 16) {
      const u32x4g x = *reinterpret_cast<const u32x4g*>(p);
      w[0] = x[0]; w[1] = x[1]; w[2] = x[2]; w[3] = x[3];
    } else {
      const u32x2g x = *reinterpret_cast<const u32x2g*>(p);
      w[0] = x[0]; w[1] = x[1];
    }
  }
  static __device__ __forceinline__ void load_keys(const PagedAttnArgs& A, size_t row0, int n, int gq, Keys& to) {
    const uint8_t* p = (const uint8_t*)A.P.k + (row0 + n) * kRow + gq * kBytes;
#pragma unroll
    for (int i = 0; i < kParts; ++i) load(p + 4 * kBytes * i, to.w + kWords * i);
    to.scales = scales_of(A.k_scale, row0 + n);
  }
  static __device__ __forceinline__ u32x4g operand(const Keys& k, int n, int gq, int kk) {
    return unpack8<T, BITS>(k.w + kk / kOut * kWords + kk % kOut * (BITS / 4), scale(k.scales, n, channel(gq, kk / kOut * kOut)));
  }
  static __device__ __forceinline__ void load_chunk(const void* base, const uint8_t* scale, size_t row, int c, Chunk& to) {
    load((const uint8_t*)base + row * kRow + c * kBytes, to.w);
    to.scales = scales_of(scale, row);
  }
  // (row, c: which chunk it is; of the row its last bit matters)
  static __device__ __forceinline__ void expand(const Chunk& chunk, int row, int c, u32x4g (&to)[kOut]) {
    const float s = scale(chunk.scales, row, 8 * kOut * c);
#pragma unroll
    for (int o = 0; o < kOut; ++o) to[o] = unpack8<T, BITS>(chunk.w + o * (BITS / 4), s);
  }
  static __device__ __forceinline__ float value(const PagedAttnArgs& A, size_t row, int ch) {
    const uint32_t byte = ((const uint8_t*)A.P.v)[row * kRow + ch * BITS / 8];
    return Mfma<T>::get(unpack<T, BITS, 0>(byte, scale_of(A.v_scale[row * (D / 32) + ch / 32])), BITS == 4 ? ch & 1 : 0);
  }
};
template <typename T, int D> struct PoolRow<T, D, 16> {
  static constexpr int kLanes = D / 8, kOut = 1;
  typedef u32x4g Chunk;
  struct Keys { u32x4g w[D / 32]; };
  static __device__ __forceinline__ int channel(int gq, int kk) { return 8 * gq + 32 * kk; }
  static __device__ __forceinline__ void load_keys(const PagedAttnArgs& A, size_t row0, int n, int gq, Keys& to) {
    const T* p = (const T*)A.P.k + row0 * D + n * D + 8 * gq;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) to.w[kk] = *reinterpret_cast<const u32x4g*>(p + 32 * kk);
  }
  static __device__ __forceinline__ u32x4g operand(const Keys& k, int, int, int kk) { return k.w[kk]; }
  static __device__ __forceinline__ void load_chunk(const void* base, const uint8_t*, size_t row, int c, Chunk& to) {
    to = *reinterpret_cast<const u32x4g*>((const T*)base + row * D + 8 * c);
  }
  static __device__ __forceinline__ void expand(const Chunk& chunk, int, int, u32x4g (&to)[1]) { to[0] = chunk; }
  static __device__ __forceinline__ float value(const PagedAttnArgs& A, size_t row, int ch) { return (float)((const T*)A.P.v)[row * D + ch]; }
};

// ---- which rows are seen ----------------------------------------------------------------------------

// The first n of 64 bits, n > 0; of 16, any n.
__device__ __forceinline__ uint64_t low64(int n) { return n < 64 ? (1ull << n) - 1 : ~0ull; }
__device__ __forceinline__ uint32_t first16(int n) { return (1u << max(0, min(n, 16))) - 1; }

// The slots that any of a sequence's tokens first .. last sees, as keys 0 .. end - 1: slot(j) of key j.  Under a window, granules between the
// always visible front and the first token's window are left out; keys in front of `front` are the first slots, the others lie `gap` further.
// (SIGHT = false: all slots up to the last token's, key = slot.)
template <bool SIGHT> struct Keys;
template <> struct Keys<false> {
  int end, all_end;                       // (every token sees the slots below all_end)
  __device__ __forceinline__ Keys(const Sight&, const Seq& s, int prefix, int first, int last) : end(row_end(s, last, prefix)), all_end(row_end(s, first, prefix)) {}
  __device__ __forceinline__ int slot(int j) const { return j; }
  __device__ __forceinline__ bool all_seen(int j, int n) const { return j + n <= all_end; }   // keys j .. j + n - 1, by all tokens
};
template <> struct Keys<true> {
  int end, all_end, front, gap, lo, sink, pre;   // all tokens see slots lo .. all_end - 1, those of them below sink, and all below pre
  __host__ __device__ __forceinline__ Keys(const Sight& V, const Seq& s, int prefix, int first, int last) {
    const int ctx = s.kv - s.nq;
    pre = max(0, min(prefix, s.kv));
    sink = V.sink;
    const int last_end = V.tree ? s.kv : max(0, ctx + last + 1);
    all_end = max(0, V.tree ? ctx : ctx + first + 1);
    end = max(last_end, pre);
    front = gap = lo = 0;
    if (V.window) {
      front = (max(sink, pre) + 15) & ~15;
      gap = max(0, ((ctx + (V.tree ? 0 : first) - V.window + 1) & ~15) - front);
      end -= gap;
      lo = ctx + (V.tree ? s.nq - 1 : last) - V.window + 1;
    }
  }
  __host__ __device__ __forceinline__ int slot(int j) const { return j < front ? j : j + gap; }
  __host__ __device__ __forceinline__ bool all_seen(int j, int n) const {
    const int at = slot(j);
    if (at + n - 1 != slot(j + n - 1)) return false;
    return (at + n <= all_end && (at >= lo || at + n <= sink)) || at + n <= pre;
  }
};

// What one row (a token) sees.  granule(first slot, whether it is there, off): which of its slots from `off` on, at(i): slot off + i; end(): no
// slot from there on.  live: whether the lane has a row at all.
template <bool SIGHT> struct RowView;
template <> struct RowView<false> {
  int last;                               // slots below are seen, no others
  __device__ __forceinline__ RowView(const Sight&, const Seq& s, int prefix, int i, bool live) : last(live ? row_end(s, i, prefix) : 0) {}
  __device__ __forceinline__ int end() const { return last; }
  struct Seen {
    int left;
    __device__ __forceinline__ bool at(int i) const { return i < left; }
  };
  __device__ __forceinline__ Seen granule(int slot, bool there, int off) const { return {there ? last - slot - off : 0}; }
};
template <> struct RowView<true> {
  // (the numbers of the sequence are uniform; a lane keeps two words of its own, and works the others out where a tile is masked)
  const Sight& V;
  const Seq& s;
  int i, lo, pre;                         // its token (-1: no row), the first slot of its window, the slots below which all see
  uint64_t drawn;                         // its bits of the first 64 new tokens: requested in front of the work, not where they are needed
  __device__ __forceinline__ RowView(const Sight& V, const Seq& s, int prefix, int token, bool live) : V(V), s(s) {
    i = live ? token : -1;
    pre = max(0, min(prefix, s.kv));
    const int ctx = s.kv - s.nq;
    lo = 0;
    drawn = V.tree ? V.tree[(size_t)(s.q0 + token) * V.words] : 0;
    if (V.window) {
      int above = token;                                           // its place is behind the tokens above it
      if (V.tree) {
        int n = __popcll(drawn & low64(s.nq));
        for (int w = 1; 64 * w < s.nq; ++w) n += __popcll(V.tree[(size_t)(s.q0 + token) * V.words + w] & low64(s.nq - 64 * w));
        above = max(n - 1, 0);
      }
      lo = ctx + above - V.window + 1;
    }
  }
  __device__ __forceinline__ bool has_slot(int t) const { return t >= 0 && s.kv - s.nq + t >= 0; }
  // no slot from here on is seen
  __device__ __forceinline__ int end() const {
    return i < 0 ? 0 : max(pre, !has_slot(i) ? 0 : V.tree ? s.kv : s.kv - s.nq + i + 1);
  }
  // bits t .. t + 15 of the token's, t from -15 on
  __device__ __forceinline__ uint32_t tree16(int token, int t) const {
    if (t <= -16 || t >= s.nq) return 0;                           // (uniform, as t is)
    uint64_t x;
    if (t < 0) x = drawn << -t;
    else if (s.nq <= 64) x = drawn >> t;
    else {
      const uint64_t* bits = V.tree + (size_t)(s.q0 + token) * V.words;
      const int w = t >> 6;
      const uint64_t here = bits[w], next = bits[min(w + 1, (s.nq - 1) >> 6)];
      x = here >> (t & 63);
      if (t & 63) x |= next << (64 - (t & 63));                    // (of the last word once more: behind the tokens, and cut off)
    }
    return (uint32_t)x & first16(s.nq - t) & 0xFFFFu;
  }
  struct Seen {
    uint32_t mask;
    __device__ __forceinline__ bool at(int i) const { return mask >> i & 1; }
    __device__ __forceinline__ float pick(int i, float x) const {  // x, or -infinity
      const uint32_t on = (uint32_t)((int)(mask << (31 - i)) >> 31);
      return __uint_as_float((__float_as_uint(x) & on) | (0xFF800000u & ~on));
    }
  };
  __device__ __forceinline__ Seen granule(int slot, bool there, int off) const {
    const int t = (int)opaque(i), ctx = s.kv - s.nq;
    const bool has = has_slot(t);
    uint32_t m = has ? first16((V.tree ? max(ctx, 0) : ctx + t + 1) - slot) : 0;
    if (V.window) m &= ~first16(lo - slot) | first16(V.sink - slot);
    if (V.tree && has) m |= tree16(t, slot - ctx);
    if (t >= 0) m |= first16(pre - slot);
    return {there ? m >> off : 0};
  }
};

// Keys of the longest sequence for a workgroup of up to `tokens` tokens, at most.
inline int most_keys(const Paged& P, const Sight& V, int tokens) {
  if (!V.window || V.prefixed) return P.max_kv;
  const long long n = (V.sink + 15ll) / 16 * 16 + V.window + (V.tree ? P.max_q : tokens < P.max_q ? tokens : P.max_q) + 15;
  return (int)(n < P.max_kv ? n : P.max_kv);
}

}  // namespace arkv
