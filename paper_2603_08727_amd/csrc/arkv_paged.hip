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

constexpr int kAppendWaves = 4, kAppendItems = 3;

// One wave per new token (or a share of its heads).  The wave's lanes form the token's angles (position times frequency in turns, in 64 bits: at
// position 2^17 a 32-bit product is off by up to 2^-8 turns; the fraction that is left fits 32), then walk its heads'
// 16-byte chunks in pairs: item i of a row is the pair of chunks whose channels turn together.  A generated token is bound by
// round trips to memory: its lengths, angles and rows are requested together, the page behind them, then it stores.
template <typename T, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void k_paged_append(AppendArgs A, int per_wave) {
  __shared__ float2 turn[kAppendWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * kAppendWaves + wave;
  const Paged& P = A.P;
  if (t >= P.N) return;
  constexpr int IPR = D / 16;                                      // items of a row
  const int Hr = A.Hq + P.H, rot = A.half / 8;                     // heads that turn; items that turn
  const int n_all = (A.Hq + 2 * P.H) * IPR;
  const int it00 = (int)blockIdx.y * per_wave, n_items = min(it00 + per_wave, n_all);     // this wave's share of the token
  struct Item { int h, hs, c0, c1; bool turns; };
  auto item = [&](int it) {
    Item o;
    o.h = it / IPR;
    const int i = it % IPR;
    o.hs = o.h < A.Hq ? o.h : o.h < Hr ? o.h - A.Hq : o.h - Hr;
    o.turns = i < rot && o.h < Hr;
    // with halves, chunk i turns with chunk i + rot; else (and behind rot_dim) two adjacent ones
    const bool halves = i < rot && !A.adjacent;
    o.c0 = halves ? i : 2 * i;
    o.c1 = halves ? i + rot : 2 * i + 1;
    return o;
  };
  // The first 64 sequences, the token's positions and the lane's frequency ...
  const int32_t* positions = A.positions + t;
  const int at0 = min(lane, P.B - 1);
  int sq0 = P.cu_q[at0], sq1 = P.cu_q[at0 + 1], skv = P.kv_len[at0];
  const int axis = A.axis[lane];
  const double freq = A.freq[min(lane, max(A.half, 1) - 1)];
  int pos[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) pos[i] = positions[(size_t)min(i, A.n_axes - 1) * P.N];
  // ... and its rows.  (Values, not structs, are chosen between: a lane's own choice of a struct would be read from memory.)
  const T *qp = (const T*)A.q.p + (size_t)t * A.q.ts, *kp = (const T*)A.k.p + (size_t)t * A.k.ts, *vp = (const T*)A.v.p + (size_t)t * A.v.ts;
  const int64_t qs = A.q.hs, ks = A.k.hs, vs = A.v.hs;
  u32x4p x[kAppendItems], y[kAppendItems];
  auto load = [&](int it0) {
#pragma unroll
    for (int u = 0; u < kAppendItems; ++u) {
      const Item o = item(min(it0 + 64 * u + lane, n_items - 1));
      const T* from = (o.h < A.Hq ? qp : o.h < Hr ? kp : vp) + (o.h < A.Hq ? qs : o.h < Hr ? ks : vs) * o.hs;
      x[u] = *reinterpret_cast<const u32x4p*>(from + 8 * o.c0);
      y[u] = *reinterpret_cast<const u32x4p*>(from + 8 * o.c1);
    }
  };
  load(it00);
  asm volatile("" : "+v"(sq0), "+v"(sq1), "+v"(skv));              // (requested here, not where they turn out to be needed)
  // the token's sequence: the first that ends behind it
  int b = -1;
  Seq s = {0, 0, 0};
  for (int i = 0; i < P.B; i += 64) {
    if (i) {
      const int at = min(i + lane, P.B - 1);
      sq0 = P.cu_q[at]; sq1 = P.cu_q[at + 1]; skv = P.kv_len[at];
    }
    const uint64_t hit = __ballot(i + lane < P.B && sq1 > t);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      b = i + l;
      s = clamp_seq(__builtin_amdgcn_readlane(sq0, l), __builtin_amdgcn_readlane(sq1, l), __builtin_amdgcn_readlane(skv, l), P.N, P.max_q, P.max_kv);
      break;
    }
  }
  if (b < 0 || t < s.q0 || t >= s.q0 + s.nq) return;               // a row of no sequence
  const int slot = s.kv - s.nq + t - s.q0;
  const int row0 = slot_row(P.table + (size_t)b * P.width, P.n_pages, P.H, 0, P.lg_page, s.kv, slot);
  if (lane < A.half) {
    const int p = axis == 0 ? pos[0] : axis == 1 ? pos[1] : axis == 2 ? pos[2] : pos[3];
    const double turns = (double)p * (freq * 0.15915494309189533577);
    float sn, cs;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
    turn[wave][lane] = make_float2(cs, sn);                        // (read by this wave alone)
  }
  if (row0 >= 0 && it00 == 0)
    for (int h = lane; h < P.H; h += 64) {
      P.pos[(size_t)row0 + ((size_t)h << P.lg_page)] = pos[0];
      if (P.weight) P.weight[(size_t)row0 + ((size_t)h << P.lg_page)] = 0.f;
    }
  for (int it0 = it00; it0 < n_items; it0 += 64 * kAppendItems) {
    if (it0 != it00) load(it0);
#pragma unroll
    for (int u = 0; u < kAppendItems; ++u) {
      const int it = it0 + 64 * u + lane;
      if (it >= n_items) continue;
      const Item o = item(it);
      if (o.turns) {
        const int i = o.c0;                                        // (halves: the pairs 8 i ..; adjacent: chunk c0 = 2 i holds 4 pairs)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 a = unpack2<T>(x[u][e]), z = unpack2<T>(y[u][e]);
          if (!A.adjacent) {
            const float2 t0 = turn[wave][8 * i + 2 * e], t1 = turn[wave][8 * i + 2 * e + 1];
            x[u][e] = pack2<T>(a.x * t0.x - z.x * t0.y, a.y * t1.x - z.y * t1.y);
            y[u][e] = pack2<T>(z.x * t0.x + a.x * t0.y, z.y * t1.x + a.y * t1.y);
          } else {
            const float2 t0 = turn[wave][4 * i + e], t1 = turn[wave][4 * i + 4 + e];
            x[u][e] = pack2<T>(a.x * t0.x - a.y * t0.y, a.y * t0.x + a.x * t0.y);
            y[u][e] = pack2<T>(z.x * t1.x - z.y * t1.y, z.y * t1.x + z.x * t1.y);
          }
        }
      }
      T* to;
      if (o.h < A.Hq) to = (T*)A.q_out + ((size_t)t * A.Hq + o.h) * D;
      else if (row0 < 0) continue;
      else to = (T*)(o.h < Hr ? P.k : P.v) + ((size_t)row0 + ((size_t)o.hs << P.lg_page)) * D;
      *reinterpret_cast<u32x4p*>(to + 8 * o.c0) = x[u];
      *reinterpret_cast<u32x4p*>(to + 8 * o.c1) = y[u];
    }
  }
}

hipError_t launch_paged_append(int dtype, int D, const AppendArgs& A, hipStream_t st) {
  // A token is one wave's work where there are tokens for the whole chip; fewer are dealt out, one load of each lane's at a
  // time (16 tokens of 32 + 2 x 8 heads: 6.9 us as one wave each, 5.3 as two).
  const int n_all = (A.Hq + 2 * A.P.H) * (D / 16), once = 64 * kAppendItems;
  const int per_wave = A.P.N >= 2048 ? n_all : once;
  const dim3 grid((A.P.N + kAppendWaves - 1) / kAppendWaves, (n_all + per_wave - 1) / per_wave), block(64 * kAppendWaves);
  if (dtype == ARKV_DTYPE_BF16) {
    if (D == 64) k_paged_append<__bf16, 64><<<grid, block, 0, st>>>(A, per_wave);
    else k_paged_append<__bf16, 128><<<grid, block, 0, st>>>(A, per_wave);
  } else {
    if (D == 64) k_paged_append<_Float16, 64><<<grid, block, 0, st>>>(A, per_wave);
    else k_paged_append<_Float16, 128><<<grid, block, 0, st>>>(A, per_wave);
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

// Adds one to hist[bin] for each of a lane's four bins with `on` set.  The lanes that share the bin of the first one (equal
// weights, such as those of rows that nobody looked at) add once for all: additions to one word queue.
__device__ __forceinline__ void count_bins(int* hist, const bool (&on)[4], const int (&bin)[4], int lane) {
  const uint64_t live = __ballot(on[0] || on[1] || on[2] || on[3]);
  if (!live) return;
  const int first = __builtin_ctzll(live);
  const int shared = __builtin_amdgcn_readlane(on[0] ? bin[0] : on[1] ? bin[1] : on[2] ? bin[2] : bin[3], first);
  int n = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    n += __popcll(__ballot(on[e] && bin[e] == shared));
    if (on[e] && bin[e] != shared) atomicAdd(&hist[bin[e]], 1);
  }
  if (lane == first) atomicAdd(&hist[shared], n);
}

// Survivors times channels up to which the choosing workgroup copies them, which saves a launch (8 x 2 heads, 250 of 1000 rows of 64
// channels: 11.5 us against 12.6; 8 heads, 250 of 128 channels: 12.5 and 12.4; 500: 16.6 and 12.6).
constexpr int kSelectMoves = 32768;
constexpr int kEvictBins = 2048;        // eleven bits of a key
constexpr int kEvictLdsBlocks = 9;      // blocks of 4 x kEvictThreads keys that fit LDS beside the bins

// Copies survivors first, first + step, .. to their new slots: D / 8 lanes a row, kMoveRows rows per lane whose loads are all
// under way together.
constexpr int kMoveRows = 4;
template <int D>
__device__ __forceinline__ void move_rows(const EvictArgs& A, const Kept& K, int h, int b, int first, int step) {
  constexpr int LPR = D / 8;
  const int c = threadIdx.x % LPR;
  const Paged& P = A.P;
  const int32_t* kept = A.kept + ((size_t)b * P.H + h) * A.max_keep;
  int from[kMoveRows], to[kMoveRows];
#pragma unroll
  for (int r = 0; r < kMoveRows; ++r) {
    const int i = first + r * step;
    from[r] = i < K.m ? kept[i] : -1;
  }
#pragma unroll
  for (int r = 0; r < kMoveRows; ++r) {
    from[r] = slot_row(P.table + (size_t)b * P.width, P.n_pages, P.H, h, P.lg_page, K.n, from[r]);
    to[r] = slot_row(A.dst_table + (size_t)b * A.dst_width, P.n_pages, P.H, h, P.lg_page, K.m, first + r * step);
  }
  u32x4p x[kMoveRows], y[kMoveRows];
#pragma unroll
  for (int r = 0; r < kMoveRows; ++r) {
    x[r] = ((const u32x4p*)P.k)[(size_t)max(from[r], 0) * LPR + c];
    y[r] = ((const u32x4p*)P.v)[(size_t)max(from[r], 0) * LPR + c];
  }
#pragma unroll
  for (int r = 0; r < kMoveRows; ++r) {
    if (from[r] < 0 || to[r] < 0) continue;
    ((u32x4p*)P.k)[(size_t)to[r] * LPR + c] = x[r];
    ((u32x4p*)P.v)[(size_t)to[r] * LPR + c] = y[r];
    if (c == 0) P.pos[to[r]] = P.pos[from[r]];
    if (c == 1) P.weight[to[r]] = P.weight[from[r]];
  }
}

template <int D>
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs A) {
  constexpr int RPW = 256 / (D / 8);
  const int h = blockIdx.y, b = blockIdx.z;
  move_rows<D>(A, kept_of(A, b), h, b, blockIdx.x * RPW * kMoveRows + threadIdx.x / (D / 8), RPW);
}

// Which rows of a (sequence, kv-head) stay.  One workgroup finds the key of the last one digit by digit, from the top: how
// many rows have which digit, and the digit at which the rows to keep run out; a digit whose rows all stay ends the search.
// Then every wave writes the survivors among its slots, behind those of the waves before.  A wave's slots are adjacent,
// four per lane and block (in one page: one look at the table and one 16-byte load).  IN_LDS: the keys are read from memory
// once and stay in LDS; else (more rows than it holds) they are read in every pass.  MOVE > 0: the workgroup then copies the
// survivors of MOVE channels itself.
template <bool IN_LDS, int MOVE>
__global__ __launch_bounds__(kEvictThreads) void k_evict_select(EvictArgs A) {
  constexpr int NW = kEvictThreads / 64, BPT = kEvictBins / kEvictThreads;
  extern __shared__ u32x4p held[];                                 // [block][thread]
  __shared__ int hist[kEvictBins];
  __shared__ int sums[NW], gts[NW], ties_in[NW];
  __shared__ int s_bin, s_left, s_count;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Kept K = kept_of(A, b);
  const int32_t* table = A.P.table + (size_t)b * A.P.width;
  int32_t* kept = A.kept + ((size_t)b * A.P.H + h) * A.max_keep;
  if (h == 0 && tid == 0) A.new_len[b] = K.m;
  const int lo = K.front, hi = K.n - K.back;                       // ranked slots
  const int ranked = K.m - K.front - K.back;
  const bool all = ranked >= hi - lo, none = ranked <= 0;
  const int nq = (K.n + 256 * NW - 1) / (256 * NW);                // blocks of 256 slots per wave
  const int w0 = wave * nq * 256;
  auto first_row = [&](int q) { return slot_row(table, A.P.n_pages, A.P.H, h, A.P.lg_page, K.n, w0 + 256 * q + 4 * lane); };
  auto keys_of = [](const float4& w) { return u32x4p{weight_key(w.x), weight_key(w.y), weight_key(w.z), weight_key(w.w)}; };
  auto fetch = [&](int q) {                                        // keys of the lane's four slots of block q
    const int r = first_row(q);
    return r < 0 ? u32x4p{0, 0, 0, 0} : keys_of(*reinterpret_cast<const float4*>(A.P.weight + r));
  };
  auto key = [&](int q) { return IN_LDS ? held[q * kEvictThreads + tid] : fetch(q); };
  // survivors: keys above `last`, and of those equal to it the first `need`
  uint32_t last = 0;
  int need = 0;
  if (!all && !none) {
    for (int i = tid; i < kEvictBins; i += kEvictThreads) hist[i] = 0;
    if (IN_LDS) {                                                  // (a thread's own keys: nobody else reads them)
      // all blocks' pages, then all their weights: two round trips to memory
      int r[kEvictLdsBlocks];
      float4 w[kEvictLdsBlocks];
#pragma unroll
      for (int q = 0; q < kEvictLdsBlocks; ++q) r[q] = q < nq ? first_row(q) : -1;
#pragma unroll
      for (int q = 0; q < kEvictLdsBlocks; ++q)
        if (r[q] >= 0) w[q] = *reinterpret_cast<const float4*>(A.P.weight + r[q]);
#pragma unroll
      for (int q = 0; q < kEvictLdsBlocks; ++q)
        if (q < nq) held[q * kEvictThreads + tid] = r[q] < 0 ? u32x4p{0, 0, 0, 0} : keys_of(w[q]);
    }
    __syncthreads();
    need = ranked;
    uint32_t prefix = 0;
    for (int shift = 21; ; shift = shift == 21 ? 10 : 0) {
      const int bits = shift ? 11 : 10;
      auto count = [&](int q) {
        const u32x4p x = key(q);
        const int j = w0 + 256 * q + 4 * lane;
        bool on[4];
        int bin[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          on[e] = j + e >= lo && j + e < hi && (shift == 21 || x[e] >> (shift + bits) == prefix >> (shift + bits));
          bin[e] = x[e] >> shift & ((1 << bits) - 1);
        }
        count_bins(hist, on, bin, lane);
      };
      for (int q = 0; q < nq; ++q) count(q);
      __syncthreads();
      // thread t: the bins at BPT t from the top
      int c[BPT], mine = 0;
#pragma unroll
      for (int i = 0; i < BPT; ++i) {
        c[i] = hist[kEvictBins - 1 - (BPT * tid + i)];
        hist[kEvictBins - 1 - (BPT * tid + i)] = 0;
        mine += c[i];
      }
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
      }
      if (lane == 63) sums[wave] = upto;
      __syncthreads();
      int before = upto - mine;
      for (int w = 0; w < wave; ++w) before += sums[w];
#pragma unroll
      for (int i = 0; i < BPT; ++i) {
        if (before < need && need <= before + c[i]) {
          s_bin = kEvictBins - 1 - (BPT * tid + i);
          s_left = need - before;
          s_count = c[i];
        }
        before += c[i];
      }
      __syncthreads();
      prefix |= (uint32_t)s_bin << shift;
      need = s_left;
      if (s_count == need && prefix) {                             // the whole digit stays: everything from its lowest key on
        last = prefix - 1;
        need = 0;
        break;
      }
      last = prefix;
      if (!shift) break;
    }
  }
  // bit e: slot e of the lane's four stays for certain, bit 4 + e: it is one of the equal ones
  auto fate = [&](int q) {
    const u32x4p x = all || none ? u32x4p{0, 0, 0, 0} : key(q);
    const int j = w0 + 256 * q + 4 * lane;
    uint32_t f = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool held_ = j + e < lo || j + e >= hi || all;
      if (j + e < K.n && (held_ || (!none && x[e] > last))) f |= 1u << e;
      if (j + e < K.n && !held_ && !none && x[e] == last && need > 0) f |= 16u << e;
    }
    return f;
  };
  int n_gt = 0, n_tie = 0;
  auto tally = [&](int q) {
    const uint32_t f = fate(q);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      n_gt += __popcll(__ballot(f >> e & 1));
      n_tie += __popcll(__ballot(f >> (4 + e) & 1));
    }
  };
  for (int q = 0; q < nq; ++q) tally(q);
  if (lane == 0) { gts[wave] = n_gt; ties_in[wave] = n_tie; }
  __syncthreads();
  int at = 0, tied = 0;                                            // survivors and equal keys in front of this wave's slots
  for (int w = 0; w < wave; ++w) { at += gts[w]; tied += ties_in[w]; }
  at += min(tied, need);
  const uint64_t below = (1ull << lane) - 1;
  auto write = [&](int q) {
    const uint32_t f = fate(q);
    int mine = 0, ties = 0;                                        // equal ones in lanes below, and in all
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t tb = __ballot(f >> (4 + e) & 1);
      mine += __popcll(tb & below);
      ties += __popcll(tb);
    }
    uint32_t take = f & 15;
    int rank = tied + mine;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (f >> (4 + e) & 1) {
        if (rank < need) take |= 1u << e;
        ++rank;
      }
    tied += ties;
    int to = 0, n = 0;                                             // of this block's survivors: in lanes below, in all
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t kb = __ballot(take >> e & 1);
      to += __popcll(kb & below);
      n += __popcll(kb);
    }
    // through LDS, in place of the block's keys, which are done with: adjacent lanes then store adjacent words
    int* list = reinterpret_cast<int*>(&held[q * kEvictThreads + 64 * wave]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (take >> e & 1) {
        if (IN_LDS) list[to] = w0 + 256 * q + 4 * lane + e;
        else if (at + to < A.max_keep) kept[at + to] = w0 + 256 * q + 4 * lane + e;
        ++to;
      }
    if (IN_LDS)
      for (int i = lane; i < n; i += 64)
        if (at + i < A.max_keep) kept[at + i] = list[i];
    at += n;
  };
  for (int q = 0; q < nq; ++q) write(q);
  for (int i = K.m + tid; i < A.max_keep; i += kEvictThreads) kept[i] = -1;
  if constexpr (MOVE > 0) {
    constexpr int RPW = kEvictThreads / (MOVE / 8);
    __syncthreads();                                               // the list is written
    for (int i = 0; i < K.m; i += RPW * kMoveRows) move_rows<MOVE>(A, K, h, b, i + tid / (MOVE / 8), RPW);
  }
}

hipError_t launch_paged_evict(int D, const EvictArgs& A, hipStream_t st) {
  const dim3 units(A.P.H, A.P.B);
  const int rows = std::min(A.max_keep, A.P.max_kv), rpw = 256 / (D / 8) * kMoveRows;
  const bool moves = rows * D <= kSelectMoves;
  const int blocks = (A.P.max_kv + 4 * kEvictThreads - 1) / (4 * kEvictThreads);
  if (blocks <= kEvictLdsBlocks) {
    const void* kernel = !moves ? (const void*)k_evict_select<true, 0> : D == 64 ? (const void*)k_evict_select<true, 64> : (const void*)k_evict_select<true, 128>;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 16 * kEvictThreads * kEvictLdsBlocks);
    if (e != hipSuccess) return e;
    const int bytes = 16 * kEvictThreads * blocks;
    if (!moves) k_evict_select<true, 0><<<units, kEvictThreads, bytes, st>>>(A);
    else if (D == 64) k_evict_select<true, 64><<<units, kEvictThreads, bytes, st>>>(A);
    else k_evict_select<true, 128><<<units, kEvictThreads, bytes, st>>>(A);
  } else {
    if (!moves) k_evict_select<false, 0><<<units, kEvictThreads, 0, st>>>(A);
    else if (D == 64) k_evict_select<false, 64><<<units, kEvictThreads, 0, st>>>(A);
    else k_evict_select<false, 128><<<units, kEvictThreads, 0, st>>>(A);
  }
  if (!moves && rows > 0) {
    const dim3 grid((rows + rpw - 1) / rpw, A.P.H, A.P.B);
    if (D == 64) k_evict_move<64><<<grid, 256, 0, st>>>(A);
    else k_evict_move<128><<<grid, 256, 0, st>>>(A);
  }
  return hipGetLastError();
}

}  // namespace arkv
