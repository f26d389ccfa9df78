// Attention of new tokens over a paged cache, and the weight that the cached rows collect from them.
//
// The rows of a (sequence, kv-head) are its new tokens times the G query heads of the group: row r is token r / G, head
// r % G, so the heads of a group share every key and value that is fetched.  Two kernels divide the sequences between them:
//   paged_step   up to 16 rows (a generated token, a few drafted ones): bound by reading the pages (4 x 131071 rows x 8 heads in
//                377 us, 5.7 TB/s; 31 requests of up to 16384 rows in 184 us, 4.9 TB/s)
//   paged_chunk  more rows: bound by the matrix cores and the exponentials between them (2 x 2048 tokens of 16384, 32 heads, in
//                917 to 946 us, 1.09 to 1.12 PFLOP/s)
// Both split a sequence's keys over workgroups where that fills the chip.  The last workgroup to finish joins up to 16 pieces, a
// launch of k_paged_merge more than that.
//
// In both, keys are on the M side of the logits MFMA (S^T = K Q^T), which leaves one row per lane, and the lane's
// probabilities are, as they lie, the B operand of O^T = V^T P^T once the contraction index is read in their order; the
// matching A operand comes out of row-major values in LDS by transposing reads (ds_read_b64_tr_b16: sixteen lanes read a
// 4 x 16 block, four lanes a row, and get a column each).
// Probabilities are rounded to the pages' type on the way into the second product, whose operands have that type: off by half a step each,
// in either direction, as the output's own rounding is once; the denominator sums them as they were (16384 rows in bf16: outputs 2.0e-3 from
// 64 bits, of which 1.7e-3 is the output's rounding).
// The softmax reference of a row is lazy: probabilities are taken against the row's present reference, which moves to the
// tile's maximum only when a lane's sum shows that they grew large (or when it is unset).
// Pages are at least 16 slots, so the 16 rows from a multiple of 16 on (a granule) lie in one page, whose id is uniform.
#include <algorithm>

#include "arkv_paged_mma.h"

namespace arkv {

constexpr int kStepWaves = 4;
constexpr int kStepMaxPiece = 2048;     // (at most 4096: a lane holds the page of one granule)
constexpr int kChunkRows = 128, kChunkKeys = 64;

// How a launch is cut.  step_piece, chunk_piece: keys per workgroup; the counts: pieces of the longest sequence.
// blocks: of kChunkRows rows, of all sequences, at most.  joined: the last workgroup of a (sequence, kv-head), chunk_joined: of a block
// and kv-head joins its pieces (tickets from chunk_ticket0 on), no launch is needed for that.
struct Cut { int step_piece, n_step, chunk_piece, n_chunk, blocks, chunk_ticket0; bool joined, chunk_joined; Which w; };
constexpr int kJoinPieces = 16;         // at most: a lane has all pieces' loads under way at once
constexpr int kJoinBlocks = 2048;       // pieces of blocks that are joined in the launch, at most (they take 67 KB of workspace each)

static Cut cut_of(const Paged& P, int D, int Hq) {
  Cut c = {};
  const int G = Hq / P.H;
  c.w = which_kernels(P, Hq);
  // have: workgroups without a cut; want: how many there should be; least, most: keys per piece
  auto pieces = [&](long long have, long long want, int least, int most, int unit, int& piece, int& n) {
    const long long p = (P.max_kv * std::max(1ll, have) + want - 1) / want;
    piece = (int)std::min<long long>(most, std::max<long long>(least, (p + unit - 1) / unit * unit));
    n = std::max(1, (P.max_kv + piece - 1) / piece);
  };
  // A workgroup for each CU, and no more pieces than the last workgroup joins (8 heads x 1024 rows: 6.6 us in pieces of 128
  // keys, 9.6 of 512, 12.4 in one; x 8192: 13.7 us in pieces of 128 and a launch that joins them, 11.9 of 512; 32 heads x
  // 8192: 29.6 us in pieces of 512, 28.7 of 1024), but no large ones: sequences differ in length, and the last round of
  // workgroups should end with the others (32 requests of 800 to 16384 rows x 8 heads: 177 us in pieces of 2048, 182 of
  // 4096; four of 131071 rows: 362 and 354).  Fewer than 16 heads do not fill the chip in 16 pieces.
  const long long units = (long long)P.B * P.H;
  pieces(units, std::min(256ll, kJoinPieces * units), 128, units < 16 ? kStepMaxPiece / 2 : kStepMaxPiece, 128, c.step_piece, c.n_step);
  // One workgroup for each CU; then for every place on the chip, at d = 64 three to a CU, in larger pieces (1686 tokens on up to 3001
  // rows, 12 heads: 46 us in pieces of 1024 keys, 42 of 512; d = 128, 512 tokens on 4100 rows, 16 heads, 7 single tokens: 66 us in pieces of
  // 1024, 70 of 768, 82 of 512; 128 tokens on 1024 rows: 28 us in one piece, 22 in
  // pieces of 256).
  const long long rows = (long long)P.N * G, blocks = (rows + kChunkRows - 1) / kChunkRows * P.H;
  int alone, n_alone;
  pieces(blocks, 256, 256, 1 << 28, kChunkKeys, alone, n_alone);
  pieces(blocks, D == 64 ? 768 : 512, D == 64 ? 512 : 1024, 1 << 28, kChunkKeys, c.chunk_piece, c.n_chunk);
  if (alone < c.chunk_piece) { c.chunk_piece = alone; c.n_chunk = n_alone; }
  c.joined = c.n_step <= kJoinPieces && units <= kJoinUnits;
  // (a sequence that is the chunk kernel's has more rows than the step kernel takes)
  c.blocks = (int)(rows / kChunkRows + std::min<long long>(P.B, c.w.step ? rows / (kStepRows + 1) : P.B));
  c.chunk_ticket0 = c.w.step && c.joined ? (int)units : 0;
  // (512 tokens on 4100 rows, 16 heads, beside 7 single tokens: 60 us, with a launch that joins 70)
  c.chunk_joined = c.n_chunk <= kJoinPieces && (long long)c.blocks * P.H + c.chunk_ticket0 <= kJoinUnits &&
                   (long long)c.blocks * P.H * c.n_chunk <= kJoinBlocks;
  return c;
}

// Pieces' results: sums [row][D] and (reference, denominator) [row].  Rows of paged_step: ((unit * n_step + piece) * 16 +
// row), behind them rows of paged_chunk: (piece * N + token) * Hq + head, or, where its workgroups join them, kChunkRows rows of
// ((block * H + head) * n_chunk + piece), each wave's as they lie in its lanes.
struct Parts { float* acc; float2* ml; int* tickets; size_t chunk0; };

static size_t part_rows(const Paged& P, int Hq, const Cut& c, size_t& chunk0) {
  chunk0 = c.w.step && c.n_step > 1 ? (size_t)P.B * P.H * c.n_step * kStepRows : 0;
  if (!c.w.chunk || c.n_chunk == 1) return chunk0;
  return chunk0 + (c.chunk_joined ? (size_t)c.blocks * P.H * c.n_chunk * kChunkRows : (size_t)c.n_chunk * P.N * Hq);
}

// Rows of partial results that suffice for every batch of no more sequences, tokens, new tokens and rows than P's: fewer of them
// may be cut finer, so this bounds part_rows over all such batches.  With u units and want workgroups wanted, a cut whose pieces are
// neither the shortest nor the longest allowed has at most ceil(want / u) of them, and u times that is below want + u.
static size_t part_rows_bound(const Paged& P, int D, int Hq) {
  auto parts = [](long long n, long long piece) { return (n + piece - 1) / piece; };
  const long long kv = P.max_kv, units = (long long)P.B * P.H, rows = (long long)P.N * (Hq / P.H);
  long long n = 0;
  if (kv > 128)
    n = kStepRows * std::min(units * parts(kv, 128), std::max({256 + units, units * parts(kv, kStepMaxPiece), std::min(units, 15ll) * parts(kv, kStepMaxPiece / 2)}));
  if ((long long)P.max_q * (Hq / P.H) > kStepRows && kv > 256) {
    // blocks of rows times heads: only fewer than want are cut.  a, b: pieces of the shortest length, of the two cuts in cut_of
    const long long want = D == 64 ? 768 : 512, a = parts(kv, 256), b = parts(kv, D == 64 ? 512 : 1024);
    const long long h = std::min(parts(rows, kChunkRows) * P.H, want - 1);
    const long long pieces = std::max(std::min(a * h, 255 + h), std::min(b * h, want - 1 + h));
    // those that are joined in the launch: a sequence's last block may be short, and there are at most 128 / 17 such blocks to a full one
    const long long most = std::max(std::min(parts(256, P.H), a), std::min(parts(want, P.H), b));
    const long long joined = std::min<long long>(kJoinBlocks, pieces + std::min(8 * pieces, units * most));
    n += kChunkRows * std::max(pieces, joined);
  }
  return (size_t)n;
}

size_t paged_attention_floats(const Paged& P, int D, int Hq) {
  size_t chunk0;
  return kTicketFloats + part_rows(P, Hq, cut_of(P, D, Hq), chunk0) * (D + 2);
}
size_t paged_attention_bound(const Paged& P, int D, int Hq) { return kTicketFloats + part_rows_bound(P, D, Hq) * (D + 2); }

// Partial results and tickets go past the L2 of one XCD: device-scope relaxed atomics.  A workgroup waits until its stores are
// acknowledged before it draws its ticket, and the last one reads nothing that an L2 may hold from before.
__device__ __forceinline__ void put4(float* p, f32x4g x) {
  union { float f[4]; unsigned long long u[2]; } w = {{x[0], x[1], x[2], x[3]}};
  __hip_atomic_store((unsigned long long*)p, w.u[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store((unsigned long long*)p + 1, w.u[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put2(float2* p, float a, float b) {
  union { float f[2]; unsigned long long u; } w = {{a, b}};
  __hip_atomic_store((unsigned long long*)p, w.u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x4g take4(const float* p) {
  union { float f[4]; unsigned long long u[2]; } w;
  w.u[0] = __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  w.u[1] = __hip_atomic_load((const unsigned long long*)p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return f32x4g{w.f[0], w.f[1], w.f[2], w.f[3]};
}
__device__ __forceinline__ float2 take2(const float2* p) {
  union { float f[2]; unsigned long long u; } w;
  w.u = __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(w.f[0], w.f[1]);
}

// four adjacent channels of a finished row
template <typename T> __device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
  *reinterpret_cast<u32x2g*>(p) = u32x2g{Mfma<T>::pack(a, b), Mfma<T>::pack(c, d)};
}

// ---- few rows -----------------------------------------------------------------------------------------

// One workgroup = one piece of a (sequence, kv-head); its waves take a quarter of the piece each, 32 keys at a time, with
// 16x16x32 MFMAs (lane: row lane % 16, keys 4 (lane / 16) .. + 3 of each granule).  Keys come from memory in operand
// layout; values in whole rows, through LDS of the wave's own.  A tile's loads are in flight while the tile before it
// is worked on.
template <int D> struct StepLds {
  uint16_t v[kStepWaves][32][D + 16];     // (the pitch: transposing reads of 16 rows meet each bank twice, as they must)
  float acc[kStepWaves][kStepRows][D + 4];
  float2 ml[kStepWaves][kStepRows];
  int last;                               // whether this workgroup's piece was the last one to be finished
};

template <typename T, int D, int MODE>
__device__ __forceinline__ void paged_step(const PagedAttnArgs& A, const Cut& cut, const Parts& parts, StepLds<D>& sm, int id) {
  constexpr int CAP = Mode<MODE>::cap;
  constexpr bool DIST = Mode<MODE>::dist;
  constexpr int KK = D / 32, CB = D / 16, VI = 32 * D * 2 / 1024;   // k-steps, channel blocks, 1 KB loads of a value tile
  constexpr int RPI = 1024 / (2 * D), CPR = D / 8;                 // rows per load, 16-byte chunks per row
  const int piece_keys = cut.step_piece, n_pieces = cut.n_step;
  const Paged& P = A.P;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, gq = lane >> 4;
  const int unit = id % (P.B * P.H), piece = id / (P.B * P.H), h = unit % P.H, b = unit / P.H;
  const Seq s = seq_of(P, b);
  const int R = s.nq * A.G;
  if (R == 0 || R > kStepRows) return;
  const int prefix = A.S.prefix ? A.S.prefix[b] : 0;
  const int end = row_end(s, s.nq - 1, prefix);                    // what the last token sees is what any sees
  const int np = max(1, (end + piece_keys - 1) / piece_keys);
  if (piece >= np) return;
  const int row = n < R ? n : 0;
  const int my_end = n < R ? row_end(s, row / A.G, prefix) : 0;
  const int all_end = row_end(s, 0, prefix);                       // every row sees the slots below
  const int hq = h * A.G + row % A.G, tok = s.q0 + row / A.G;
  const Logit lg(A.S);
  const float slope = DIST ? A.S.slopes[hq] * kLog2e : 0.f;
  const int qp = DIST ? A.S.q_pos[tok] : 0;

  u32x4g q[KK];
  {
    const T* p = (const T*)A.q.p + (size_t)tok * A.q.ts + (size_t)hq * A.q.hs + 8 * gq;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = *reinterpret_cast<const u32x4g*>(p + 32 * kk);
  }
  // this wave's keys: [w0, w1), whole tiles
  const int p0 = piece * piece_keys, p1 = min(p0 + piece_keys, end);
  const int tiles = (p1 - p0 + 31) / 32, per = (tiles + kStepWaves - 1) / kStepWaves;
  const int t0 = min(per * wave, tiles), t1 = min(t0 + per, tiles);
  const int w0 = p0 + 32 * t0;
  // lane i holds the page id of granule i from w0 on; one that is not there becomes page 0, whose rows nobody sees
  int my_page;
  bool page_ok;
  {
    const int j = w0 + 16 * lane;
    my_page = j < p1 ? P.table[(size_t)b * P.width + (j >> P.lg_page)] : 0;
    page_ok = (unsigned)my_page < (unsigned)P.n_pages;
    if (!page_ok) my_page = 0;
  }
  const uint64_t ok_mask = __ballot(page_ok);
  const int in_page = (1 << P.lg_page) - 1;
  auto granule_row = [&](int g) {                                  // first row of granule g
    const int page = __builtin_amdgcn_readlane(my_page, g);
    return (size_t)(unsigned)(((page * P.H + h) << P.lg_page) + ((w0 + 16 * g) & in_page));
  };

  u32x4g kb[2][2][KK], vb[VI];
  auto load_k = [&](int t, u32x4g (&to)[2][KK]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const T* p = (const T*)P.k + granule_row(2 * t + g) * D + n * D + 8 * gq;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) to[g][kk] = *reinterpret_cast<const u32x4g*>(p + 32 * kk);
    }
  };
  auto load_v = [&](int t) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const T* p = (const T*)P.v + granule_row(2 * t + g) * D + (lane / CPR) * D + 8 * (lane % CPR);
#pragma unroll
      for (int i = 0; i < VI / 2; ++i) vb[g * (VI / 2) + i] = *reinterpret_cast<const u32x4g*>(p + i * RPI * D);
    }
  };
  f32x4g acc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) acc[c] = f32x4g{0.f, 0.f, 0.f, 0.f};
  float m = kUnset, l = 0.f;
  const int nt = t1 - t0;

  auto tile = [&](int t, const u32x4g (&kc)[2][KK]) {
    const int j0 = w0 + 32 * t;
    f32x4g x[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      x[g] = f32x4g{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) x[g] = Mfma<T>::m16(kc[g][kk], q[kk], x[g]);
    }
    const bool masked = j0 + 32 > all_end || (ok_mask >> (2 * t) & 3) != 3;
    float mul = lg.mul;
    if (CAP || DIST) {
      mul = 1.f;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[g][i] = lg.logit<CAP>(x[g][i]);
        if (DIST) {
          const int4 kp = *reinterpret_cast<const int4*>(P.pos + granule_row(2 * t + g) + 4 * gq);
          x[g][0] = fmaf(-slope, fabsf((float)(qp - kp.x)), x[g][0]);
          x[g][1] = fmaf(-slope, fabsf((float)(qp - kp.y)), x[g][1]);
          x[g][2] = fmaf(-slope, fabsf((float)(qp - kp.z)), x[g][2]);
          x[g][3] = fmaf(-slope, fabsf((float)(qp - kp.w)), x[g][3]);
        }
      }
    }
    uint32_t odd = 0;                                              // keys of this tile whose values are not all finite
    if (masked) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x[g][i] = j0 + 16 * g + 4 * gq + i < my_end && (ok_mask >> (2 * t + g) & 1) ? x[g][i] * mul : -INFINITY;
      mul = 1.f;
      // a value that is not finite would spoil the rows that do not see it: it leaves the product, and is added below
#pragma unroll
      for (int i = 0; i < VI; ++i) {
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t f = not_finite<T>(vb[i][e]);
          vb[i][e] &= ~f;
          any |= f;
        }
        const uint64_t who = __ballot(any != 0);
#pragma unroll
        for (int r = 0; r < RPI; ++r)
          if (who >> (CPR * r) & ((1ull << CPR) - 1)) odd |= 1u << (RPI * i + r);
      }
    }
#pragma unroll
    for (int i = 0; i < VI; ++i)
      *reinterpret_cast<u32x4g*>(&sm.v[wave][RPI * i + lane / CPR][8 * (lane % CPR)]) = vb[i];
    if (t + 1 < nt) load_v(t + 1);
    float p[8];
    auto probs = [&]() {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = exp2_hw(fmaf(x[i >> 2][i & 3], mul, -m));
        sum += p[i];
      }
      return sum;
    };
    float sum = probs();
    uint64_t big = __ballot(!(sum <= kSumLimit));
    if (big) {
      big |= big >> 32;                                            // of the four lanes of a row any one: that row alone moves
      big |= big >> 16;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i >> 2][i & 3] * mul);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = big >> n & 1 ? fmaxf(m, top) : m, f = exp2_hw(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int c = 0; c < CB; ++c) acc[c] *= f;
      sum = probs();
    }
    l += sum;
    const u32x4g pb = {Mfma<T>::pack(p[0], p[1]), Mfma<T>::pack(p[2], p[3]), Mfma<T>::pack(p[4], p[5]), Mfma<T>::pack(p[6], p[7])};
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      const s16x4g a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)&sm.v[wave][4 * gq + (n >> 2)][16 * c + 4 * (n & 3)]);
      const s16x4g a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)&sm.v[wave][16 + 4 * gq + (n >> 2)][16 * c + 4 * (n & 3)]);
      const u32x2g w0_ = __builtin_bit_cast(u32x2g, a0), w1_ = __builtin_bit_cast(u32x2g, a1);
      acc[c] = Mfma<T>::m16(u32x4g{w0_[0], w0_[1], w1_[0], w1_[1]}, pb, acc[c]);
    }
    while (odd) {                                                  // (uniform; hardly ever)
      const int j = __builtin_ctz(odd);
      odd &= odd - 1;
      const int g = j >> 4, i = j & 3, from = (j & 12) >> 2;
      float pj = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e == 4 * g + i) pj = Mfma<T>::get(opaque(pb[e / 2]), e & 1);
      pj = __shfl(pj, n + 16 * from);
      const bool seen = j0 + j < my_end && (ok_mask >> (2 * t + g) & 1);
      const T* v = (const T*)P.v + (granule_row(2 * t + g) + (j & 15)) * D + 4 * gq;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = (float)v[16 * c + e];
          if (seen && !(fabsf(w) < INFINITY)) acc[c][e] += pj * w;
        }
    }
  };
  if (nt > 0) {
    load_k(0, kb[0]);
    load_v(0);
    for (int t = 0; t < nt; t += 2) {
      if (t + 1 < nt) load_k(t + 1, kb[1]);
      tile(t, kb[0]);
      if (t + 1 < nt) {
        if (t + 2 < nt) load_k(t + 2, kb[0]);
        tile(t + 1, kb[1]);
      }
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int c = 0; c < CB; ++c) *reinterpret_cast<f32x4g*>(&sm.acc[wave][n][16 * c + 4 * gq]) = acc[c];
  if (gq == 0) sm.ml[wave][n] = make_float2(m, l);
  __syncthreads();
  auto finish = [&](int r, int c, f32x4g o, float mm, float ll) {  // four channels of a row's result
    const size_t orow = (size_t)(s.q0 + r / A.G) * A.Hq + h * A.G + r % A.G;
    const float inv = ll == 0.f ? 0.f : 1.f / ll;                  // (NaN stays)
    store4((T*)A.out + orow * D + c, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (c == 0 && A.lse) A.lse[orow] = ll == 0.f ? -INFINITY : kLn2 * (mm + log2f(ll));
  };
  // the waves' parts: thread = four channels of a row
  for (int it = threadIdx.x; it < R * (D / 4); it += 64 * kStepWaves) {
    const int r = it / (D / 4), c = 4 * (it % (D / 4));
    float mm = kUnset, ll = 0.f;
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) mm = fmaxf(mm, sm.ml[w][r].x);
    f32x4g o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) {
      const float f = exp2_hw(sm.ml[w][r].x - mm);
      ll += f * sm.ml[w][r].y;
      o += f * *reinterpret_cast<const f32x4g*>(&sm.acc[w][r][c]);
    }
    if (np > 1) {
      const size_t pr = ((size_t)unit * n_pieces + piece) * kStepRows + r;
      put4(parts.acc + pr * D + c, o);
      if (c == 0) put2(parts.ml + pr, mm, ll);
    } else {
      finish(r, c, o, mm, ll);
    }
  }
  if (np == 1 || !cut.joined) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // this wave's stores are where everyone sees them
  __syncthreads();
  int* ticket = parts.tickets + unit * kTicketWords;
  if (threadIdx.x == 0) {
    const int drawn = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sm.last = drawn == np - 1;
    if (sm.last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // as the next call wants it
  }
  __syncthreads();
  if (!sm.last) return;
  for (int it = threadIdx.x; it < R * (D / 4); it += 64 * kStepWaves) {
    const int r = it / (D / 4), c = 4 * (it % (D / 4));
    const size_t first = (size_t)unit * n_pieces * kStepRows + r;
    float2 ml[kJoinPieces];
    f32x4g x[kJoinPieces];
#pragma unroll
    for (int p = 0; p < kJoinPieces; ++p) {
      if (p < np) {
        ml[p] = take2(parts.ml + first + p * kStepRows);
        x[p] = take4(parts.acc + (first + p * kStepRows) * D + c);
      }
    }
    float mm = kUnset, ll = 0.f;
#pragma unroll
    for (int p = 0; p < kJoinPieces; ++p)
      if (p < np) mm = fmaxf(mm, ml[p].x);
    f32x4g o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < kJoinPieces; ++p)
      if (p < np) {
        const float f = exp2_hw(ml[p].x - mm);
        ll += f * ml[p].y;
        o += f * x[p];
      }
    finish(r, c, o, mm, ll);
  }
}

// ---- many rows ----------------------------------------------------------------------------------------

// Blocks of kChunkRows rows that paged_chunk makes of a sequence.
__host__ __device__ __forceinline__ int chunk_blocks(int nq, int G, int few) { return nq * G <= few ? 0 : (nq * G + kChunkRows - 1) / kChunkRows; }

// Sequence and block of the rank-th block of a launch; the lanes of a wave look at 64 sequences at a time.
__device__ __forceinline__ bool find_block(const Paged& P, int G, int few, int rank, int lane, int& b, int& blk, Seq& s) {
  for (int i = 0; i < P.B; i += 64) {
    const Seq own = seq_of(P, min(i + lane, P.B - 1));
    const int mine = i + lane < P.B ? chunk_blocks(own.nq, G, few) : 0;
    int sum = mine;                                                // blocks up to and with this lane's sequence
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int below = __shfl_up(sum, o);
      if (lane >= o) sum += below;
    }
    const uint64_t hit = __ballot(sum > rank);
    if (hit) {
      const int first = __builtin_ctzll(hit);
      b = i + first;
      const int n = __builtin_amdgcn_readlane(mine, first);
      blk = n - 1 - (rank - (__builtin_amdgcn_readlane(sum, first) - n));   // the block that sees most comes first
      s = {__builtin_amdgcn_readlane(own.q0, first), __builtin_amdgcn_readlane(own.nq, first), __builtin_amdgcn_readlane(own.kv, first)};
      return true;
    }
    rank -= __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

// One workgroup = 128 rows of a (sequence, kv-head) and a piece of the keys they see; a wave takes 32 rows with 32x32x16
// MFMAs (lane: row lane % 32, keys 8 (i / 4) + 4 (lane / 32) + i % 4 of each half of a 64-key tile).  Keys and values of
// a tile go to LDS as they lie in the pages, sixteen rows per wave, while the tile before is worked on: two buffers, one
// barrier a tile.  The rows' 16-byte chunks are stored in an order in which neither the keys' reads (one chunk of 32
// rows) nor the values' transposing reads (64 bytes of 8 rows) meet in a bank more often than they must.
template <int D> struct ChunkLds {
  uint16_t k[2][kChunkKeys * D];
  uint16_t v[2][kChunkKeys * D];
  int pos[2][kChunkKeys];
  uint32_t odd[2];
  int last;                               // whether this workgroup's piece was the last one to be finished
};
template <int D> __device__ __forceinline__ int v_chunk(int row, int c) { return D == 128 ? c ^ (row & 3) << 2 : c ^ (row >> 1 & 1) << 2; }

template <typename T, int D, int MODE>
__device__ __forceinline__ void paged_chunk(const PagedAttnArgs& A, const Cut& cut, const Parts& parts, ChunkLds<D>& sm, int id) {
  constexpr int CAP = Mode<MODE>::cap;
  constexpr bool DIST = Mode<MODE>::dist;
  const int piece_keys = cut.chunk_piece;
  constexpr int KK = D / 16, CB = D / 32, CPR = D / 8, RPI = 64 / CPR, LPG = 16 / RPI;   // LPG: 1 KB loads of a granule
  const Paged& P = A.P;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int h = id % P.H, piece = id / (cut.blocks * P.H), bh = id % (cut.blocks * P.H);
  int b, blk;
  Seq s;
  if (!find_block(P, A.G, cut.w.few, bh / P.H, lane, b, blk, s)) return;
  const int prefix = A.S.prefix ? A.S.prefix[b] : 0;
  const int R = s.nq * A.G, r0 = blk * kChunkRows;
  const int end = row_end(s, min(R - 1, r0 + kChunkRows - 1) / A.G, prefix);
  const int np = max(1, (end + piece_keys - 1) / piece_keys);
  if (piece >= np) return;
  const int r = r0 + 32 * wave + n;
  const int rc = min(r, R - 1);
  const int my_end = r < R ? row_end(s, rc / A.G, prefix) : 0;
  const int all_end = row_end(s, r0 / A.G, prefix);                // every row of the workgroup sees the slots below
  const int hq = h * A.G + rc % A.G, tok = s.q0 + rc / A.G;
  const Logit lg(A.S);
  const float slope = DIST ? A.S.slopes[hq] * kLog2e : 0.f;
  const int qp = DIST ? A.S.q_pos[tok] : 0;

  u32x4g q[KK];
  {
    const T* p = (const T*)A.q.p + (size_t)tok * A.q.ts + (size_t)hq * A.q.hs + 8 * hh;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = *reinterpret_cast<const u32x4g*>(p + 16 * kk);
  }
  const int p0 = piece * piece_keys, p1 = min(p0 + piece_keys, end), nt = (p1 - p0 + kChunkKeys - 1) / kChunkKeys;
  const int32_t* table = P.table + (size_t)b * P.width;
  const int in_page = (1 << P.lg_page) - 1;

  // where this lane's chunk of a 1 KB load lies in a granule: row RPI i + lane / CPR
  uint32_t koff[LPG], voff[LPG];
#pragma unroll
  for (int i = 0; i < LPG; ++i) {
    const int rr = RPI * i + lane / CPR;
    koff[i] = 2 * (rr * D + 8 * k_chunk<D>(rr, lane % CPR));
    voff[i] = 2 * (rr * D + 8 * v_chunk<D>(rr, lane % CPR));
  }
  const uint32_t lds_k = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)sm.k;
  const uint32_t lds_v = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)sm.v;
  const uint32_t lds_pos = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)sm.pos;
  // Lane i holds the page of granule i of a group of sixteen tiles, this one and the next one; one that is not there becomes
  // page 0, whose rows nobody sees.
  int pages[2];
  uint64_t there[2];
  auto load_pages = [&](int group, int which) {
    const int j = p0 + 16 * (64 * group + lane);
    int page = j < p1 ? table[j >> P.lg_page] : -1;
    const bool ok = (unsigned)page < (unsigned)P.n_pages;
    there[which] = __ballot(ok);
    pages[which] = ok ? page : 0;
  };
  auto granule_row = [&](int which, int t, int g) {                // first row of granule g of tile t
    const int page = __builtin_amdgcn_readlane(which ? pages[1] : pages[0], 4 * (t & 15) + g);
    return (size_t)(unsigned)(((page * P.H + h) << P.lg_page) + ((p0 + kChunkKeys * t + 16 * g) & in_page));
  };
  auto fetch = [&](int which, int t, int buf) {                    // this wave's granule of tile t
    const size_t row = granule_row(which, t, wave);
    const T* kp = (const T*)P.k + row * D;
    const T* vp = (const T*)P.v + row * D;
    const uint32_t at = (uint32_t)(buf * kChunkKeys * D * 2 + wave * 16 * D * 2);
#pragma unroll
    for (int i = 0; i < LPG; ++i) load_lds(kp, koff[i], lds_k + at + 1024 * i);
#pragma unroll
    for (int i = 0; i < LPG; ++i) load_lds(vp, voff[i], lds_v + at + 1024 * i);
    if (DIST && lane < 16) load_lds4(P.pos + row + lane, lds_pos + 4 * (buf * kChunkKeys + 16 * wave));
  };

  f32x16g acc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
  // The row's softmax reference; rows that see none of this piece need none.
  float m = my_end > p0 ? kUnset : 0.f, l = 0.f;
  load_pages(0, 0);
  if (nt > 0) fetch(0, 0, 0);
  auto tile = [&](int t, auto which_buf) {
    const int buf = which_buf;
    const int j0 = p0 + kChunkKeys * t;
    if ((t & 15) == 0) {
      if (t) { pages[0] = pages[1]; there[0] = there[1]; }
      load_pages((t >> 4) + 1, 1);
    }
    vm_wait();                                                     // this wave's part of tile t is in LDS,
    __syncthreads();                                               // everyone's is, and the other buffer's readers are done
    if (t + 1 < nt) fetch((t & 15) == 15, t + 1, buf ^ 1);
    const uint32_t ok = (uint32_t)(there[0] >> (4 * (t & 15))) & 15;   // granules that are there
    const bool masked = j0 + kChunkKeys > all_end || ok != 15;
    uint64_t odd = 0;
    if (masked) {
      // Values that are not finite would spoil the rows that do not see them: they leave the product, and are added below.
      if (tid < 2) sm.odd[tid] = 0;
      __syncthreads();
      constexpr int PT = kChunkKeys * CPR / 256;                   // chunks per thread
#pragma unroll
      for (int i = 0; i < PT; ++i) {
        const int at = tid + 256 * i, rr = at / CPR;
        u32x4g* p = reinterpret_cast<u32x4g*>(&sm.v[buf][8 * at]);
        u32x4g w = *p;
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t f = not_finite<T>(w[e]);
          w[e] &= ~f;
          any |= f;
        }
        if (any) {
          *p = w;
          if (j0 + rr < end && (ok >> (rr >> 4) & 1)) atomicOr(&sm.odd[rr >> 5], 1u << (rr & 31));
        }
      }
      __syncthreads();
      odd = (uint64_t)sm.odd[1] << 32 | sm.odd[0];
    }
    f32x16g x[2];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[g][i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const u32x4g a = *reinterpret_cast<const u32x4g*>(&sm.k[buf][(32 * g + n) * D + 8 * k_chunk<D>(n, 2 * kk + hh)]);
        x[g] = Mfma<T>::m32(a, q[kk], x[g]);
      }
    // logits above the reference (above 0 where that is unset)
    const bool unset = m == kUnset;
    const float ref = unset ? 0.f : m;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        int kp[4] = {0, 0, 0, 0};
        if (DIST) {
          const int4 k4 = *reinterpret_cast<const int4*>(&sm.pos[buf][32 * g + 8 * e + 4 * hh]);
          kp[0] = k4.x; kp[1] = k4.y; kp[2] = k4.z; kp[3] = k4.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y = lg.above<CAP>(x[g][4 * e + i], ref);
          if (DIST) y = fmaf(-slope, fabsf((float)(qp - kp[i])), y);
          x[g][4 * e + i] = y;
        }
      }
    if (masked) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {                                // granules
        const int left = opaque(ok >> g & 1 ? my_end - j0 - 16 * g - 4 * hh : 0);   // (what depends on it stays in this branch)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (8 * (i >> 2) + (i & 3) >= left) x[g >> 1][8 * (g & 1) + i] = -INFINITY;
      }
    }
    u32x4g pb[4];                                                  // probabilities of keys 16 i .. 16 i + 15, eight per lane
    auto probs = [&]() {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        const float a = exp2_hw(x[i >> 4][i & 15]), e = exp2_hw(x[i >> 4][(i & 15) + 1]);
        sum += a;
        sum += e;
        pb[i >> 3][(i & 7) >> 1] = Mfma<T>::pack(a, e);
      }
      return sum;
    };
    float sum = probs();
    if (__any(unset || !(sum <= kSumLimit))) {                     // rare after the first tile
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 32; ++i) top = fmaxf(top, x[i >> 4][i & 15]);
      top = fmaxf(top, __shfl_xor(top, 32));
      // (both lanes of a row alike; a NaN beside a small sum: stays, and so does the NaN)
      const bool move = unset ? top > -INFINITY : !(fmaxf(sum, __shfl_xor(sum, 32)) <= kSumLimit);
      const float mn = !move ? m : unset ? top : fmaxf(m, top + m);
      const float f = !move || unset ? 1.f : exp2_hw(m - mn);      // (an unset row has nothing yet)
      const float shift = move ? ref - mn : 0.f;
      m = mn;
      l *= f;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] *= f;
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i >> 4][i & 15] += shift;
      sum = probs();
    }
    l += sum;
#pragma unroll
    for (int jj = 0; jj < 4; ++jj)
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const int r4 = 16 * jj + 4 * hh + (lane >> 2 & 3), ch = 32 * c + 16 * (lane >> 4 & 1) + 4 * (lane & 3);
        const s16x4g a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)&sm.v[buf][r4 * D + 8 * v_chunk<D>(r4, ch >> 3) + (ch & 7)]);
        const s16x4g a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)&sm.v[buf][(r4 + 8) * D + 8 * v_chunk<D>(r4, ch >> 3) + (ch & 7)]);
        const u32x2g w0 = __builtin_bit_cast(u32x2g, a0), w1 = __builtin_bit_cast(u32x2g, a1);
        acc[c] = Mfma<T>::m32(u32x4g{w0[0], w0[1], w1[0], w1[1]}, pb[jj], acc[c]);
      }
    while (odd) {                                                  // (uniform; hardly ever)
      const int j = __builtin_ctzll(odd);
      odd &= odd - 1;
      float pj = 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e)
        if (e == 16 * (j >> 5) + 4 * (j >> 3 & 3) + (j & 3)) pj = Mfma<T>::get(opaque(pb[e >> 3][(e & 7) >> 1]), e & 1);
      pj = __shfl(pj, n + 32 * (j >> 2 & 1));
      const bool seen = j0 + j < my_end;
      const T* v = (const T*)P.v + (granule_row(0, t, j >> 4) + (j & 15)) * D + 4 * hh;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float w = (float)v[32 * c + 8 * (i >> 2) + (i & 3)];
          if (seen && !(fabsf(w) < INFINITY)) acc[c][i] += pj * w;
        }
    }
  };
  if constexpr (DIST || D == 64) {                                 // (two copies of the tile do not fit the registers of two and three waves per SIMD)
    for (int t = 0; t < nt; ++t) tile(t, t & 1);
  } else {
    for (int t = 0; t < nt; t += 2) {
      tile(t, Int<0>());
      if (t + 1 < nt) tile(t + 1, Int<1>());
    }
  }
  l += __shfl_xor(l, 32);
  if (l == 0.f) m = kUnset;
  const size_t orow = (size_t)tok * A.Hq + hq;
  if (np > 1 && !cut.chunk_joined) {
    if (r >= R) return;
    const size_t pr = parts.chunk0 + (size_t)piece * P.N * A.Hq + orow;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4g*>(parts.acc + pr * D + 32 * c + 8 * e + 4 * hh) =
            f32x4g{acc[c][4 * e], acc[c][4 * e + 1], acc[c][4 * e + 2], acc[c][4 * e + 3]};
    if (hh == 0) parts.ml[pr] = make_float2(m, l);
    return;
  }
  if (np > 1) {
    // 8 bytes per lane, adjacent lanes adjacent: where wave w's two channels i, i + 1 of block c lie in a piece's rows
    const size_t row0 = parts.chunk0 + (size_t)bh * cut.n_chunk * kChunkRows + 32 * wave;
    const uint32_t at = 8 * (uint32_t)lane;                        // (beside a uniform address: 64 bits a lane would not fit the registers)
    auto sums = [&](int p, int c, int i) {
      return reinterpret_cast<float2*>(reinterpret_cast<char*>(parts.acc + (row0 + (size_t)p * kChunkRows) * D) + (8 * c + i / 2) * 512 + at);
    };
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int i = 0; i < 16; i += 2) put2(sums(piece, c, i), acc[c][i], acc[c][i + 1]);
    if (hh == 0) put2(parts.ml + row0 + (size_t)piece * kChunkRows + n, m, l);
    vm_wait();                                                     // this wave's stores are where everyone sees them
    __syncthreads();
    int* ticket = parts.tickets + (cut.chunk_ticket0 + bh) * kTicketWords;
    if (tid == 0) {
      sm.last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == np - 1;
      if (sm.last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // as the next call wants it
    }
    __syncthreads();
    if (!sm.last) return;
    m = kUnset;
    l = 0.f;
    for (int p = 0; p < np; ++p) m = fmaxf(m, take2(parts.ml + row0 + (size_t)p * kChunkRows + n).x);
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
    for (int p = 0; p < np; ++p) {                                 // (always in this order, whoever is last)
      const float2 z = take2(parts.ml + row0 + (size_t)p * kChunkRows + n);
      float2 x[CB * 8];
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 2) x[8 * c + i / 2] = take2(sums(p, c, i));
      const float f = exp2_hw(z.x - m);
      l += f * z.y;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          acc[c][i] += f * x[8 * c + i / 2].x;
          acc[c][i + 1] += f * x[8 * c + i / 2].y;
        }
    }
  }
  if (r >= R) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;                      // (NaN stays)
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      store4((T*)A.out + orow * D + 32 * c + 8 * e + 4 * hh, acc[c][4 * e] * inv, acc[c][4 * e + 1] * inv, acc[c][4 * e + 2] * inv,
             acc[c][4 * e + 3] * inv);
  if (hh == 0 && A.lse) A.lse[orow] = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
}

// A launch: chunk_wgs workgroups for sequences of many rows (cut.blocks blocks of each kv-head, piece by piece), behind them those for
// few (unit by unit, piece by piece).  One launch for both: a prompt's chunk and the other requests' tokens share the chip.
// KIND: bit 0: there are the former, bit 1: the latter.
template <typename T, int D, int MODE, int KIND>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void k_paged_attn(PagedAttnArgs A, Cut cut, Parts parts, int chunk_wgs) {
  constexpr size_t kMost = sizeof(ChunkLds<D>) > sizeof(StepLds<D>) ? sizeof(ChunkLds<D>) : sizeof(StepLds<D>);
  __shared__ __align__(16) char lds[KIND == 1 ? sizeof(ChunkLds<D>) : KIND == 2 ? sizeof(StepLds<D>) : kMost];
  const int id = (int)blockIdx.x;
  if ((KIND & 1) && (KIND == 1 || id < chunk_wgs)) {
    if constexpr (KIND & 1) paged_chunk<T, D, MODE>(A, cut, parts, *reinterpret_cast<ChunkLds<D>*>(lds), id);
  } else {
    if constexpr (KIND & 2) paged_step<T, D, MODE>(A, cut, parts, *reinterpret_cast<StepLds<D>*>(lds), id - chunk_wgs);
  }
}

// ---- joining the pieces -------------------------------------------------------------------------------

__device__ __forceinline__ int find_seq(const int32_t* cu_q, int B, int t, int lane) {
  int b = 0;
  for (int i = 0; i < B; i += 64) b += __popcll(__ballot(i + lane < B && cu_q[min(i + lane, B - 1) + 1] <= t));
  return b;
}

// Joins the pieces of rows whose keys were split.  Rows of paged_step come first, `few_rows` of every unit (step_ids with them filled up
// to eight), then all rows where those of paged_chunk are to be joined; rows that one workgroup finished are left alone.  32 lanes hold a
// row's channels.  MANY pieces: the eight groups of 32 share a row's pieces; else each has a row of its own.
template <typename T, int D, bool MANY>
__global__ __launch_bounds__(256) void k_paged_merge(PagedAttnArgs A, Cut cut, Parts parts, int few_rows, int step_ids) {
  constexpr int C = D / 32;
  typedef float chan __attribute__((ext_vector_type(C)));
  __shared__ float s_acc[MANY ? 8 : 1][D];
  __shared__ float s_l[8];
  const Paged& P = A.P;
  const int lane = threadIdx.x & 63, c = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const int at = MANY ? (int)blockIdx.x : (int)blockIdx.x * 8 + grp;
  const bool step = (MANY ? (int)blockIdx.x : (int)blockIdx.x * 8) < step_ids;   // (uniform)
  int b, t, hq, r;
  Seq s;
  bool mine;                                                       // the row is one of the kind that is joined here
  if (step) {
    const int unit = at / few_rows;
    r = at % few_rows;
    b = min(unit / P.H, P.B - 1);
    s = seq_of(P, b);
    t = s.q0 + r / A.G;
    hq = unit % P.H * A.G + r % A.G;
    mine = unit < P.B * P.H && r < s.nq * A.G && s.nq * A.G <= kStepRows;
  } else {
    const int rows = P.N * A.Hq, want = at - step_ids, row = min(want, rows - 1);
    t = row / A.Hq;
    hq = row % A.Hq;
    if constexpr (MANY) b = find_seq(P.cu_q, P.B, t, lane);
    else {                                                         // (two rows in a wave)
      const int t0 = __builtin_amdgcn_readlane(t, 0), t1 = __builtin_amdgcn_readlane(t, 32);
      const int b0 = find_seq(P.cu_q, P.B, t0, lane), b1 = t1 == t0 ? b0 : find_seq(P.cu_q, P.B, t1, lane);
      b = lane < 32 ? b0 : b1;
    }
    mine = want < rows && b < P.B;
    b = min(b, P.B - 1);
    s = seq_of(P, b);
    const int i = t - s.q0;
    r = i * A.G + hq % A.G;
    mine = mine && i >= 0 && i < s.nq && s.nq * A.G > cut.w.few;
  }
  const int prefix = A.S.prefix ? A.S.prefix[b] : 0;
  const int last = step ? s.nq - 1 : min(s.nq * A.G - 1, r / kChunkRows * kChunkRows + kChunkRows - 1) / A.G;
  const int piece = step ? cut.step_piece : cut.chunk_piece;
  int np = (row_end(s, last, prefix) + piece - 1) / piece;
  if (!mine || np <= 1) np = 0;
  if (MANY && np == 0) return;
  const size_t first = step ? (size_t)(b * P.H + hq / A.G) * cut.n_step * kStepRows + r : parts.chunk0 + (size_t)t * A.Hq + hq;
  const size_t stride = step ? kStepRows : (size_t)P.N * A.Hq;
  float m = kUnset, l = 0.f;
  for (int p = c; p < np; p += 32) m = fmaxf(m, parts.ml[first + p * stride].x);
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  chan acc;
#pragma unroll
  for (int e = 0; e < C; ++e) acc[e] = 0.f;
#pragma unroll 4
  for (int p = MANY ? grp : 0; p < np; p += MANY ? 8 : 1) {
    const float2 ml = parts.ml[first + p * stride];
    const chan x = *reinterpret_cast<const chan*>(parts.acc + (first + p * stride) * D + C * c);
    const float f = exp2_hw(ml.x - m);
    l += f * ml.y;
    acc += f * x;
  }
  if constexpr (MANY) {
    *reinterpret_cast<chan*>(&s_acc[grp][C * c]) = acc;
    if (c == 0) s_l[grp] = l;
    __syncthreads();
    if (grp) return;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < C; ++e) acc[e] = 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      l += s_l[g];
      acc += *reinterpret_cast<const chan*>(&s_acc[g][C * c]);
    }
  }
  if (np == 0) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;                      // (NaN stays)
  const size_t id = (size_t)t * A.Hq + hq;
  T* out = (T*)A.out + id * D + C * c;
#pragma unroll
  for (int e = 0; e < C; e += 2) *reinterpret_cast<uint32_t*>(out + e) = Mfma<T>::pack(acc[e] * inv, acc[e + 1] * inv);
  if (c == 0 && A.lse) A.lse[id] = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
}

// Workgroups of a call's launches.  merge: few_rows rows of every unit, if paged_step's pieces are not joined where they are made; then
// all rows, if those of paged_chunk are not (they are cut only where they are few).  Rows of few pieces are little work, and eight fit a workgroup.
struct Launches { long long chunk, step, merge; int few_rows, step_ids; bool many; };
static Launches launches_of(const Paged& P, int Hq, const Cut& c) {
  Launches l = {};
  l.chunk = c.w.chunk ? (long long)c.blocks * P.H * c.n_chunk : 0;
  l.step = c.w.step ? (long long)P.B * P.H * c.n_step : 0;
  const bool join_step = l.step && c.n_step > 1 && !c.joined, join_chunk = l.chunk && c.n_chunk > 1 && !c.chunk_joined;
  l.few_rows = (int)std::min<long long>(kStepRows, (long long)P.max_q * (Hq / P.H));
  l.step_ids = join_step ? (P.B * P.H * l.few_rows + 7) / 8 * 8 : 0;
  l.many = (join_chunk ? c.n_chunk : c.n_step) >= 8;
  const long long ids = l.step_ids + (join_chunk ? (long long)P.N * Hq : 0);
  l.merge = l.many ? ids : (ids + 7) / 8;
  return l;
}
long long paged_attention_workgroups(const Paged& P, int D, int Hq) {
  const Launches l = launches_of(P, Hq, cut_of(P, D, Hq));
  return std::max(l.chunk + l.step, l.merge);
}

template <typename T, int D, int MODE>
static hipError_t launch_attention(const PagedAttnArgs& A, hipStream_t st) {
  const Paged& P = A.P;
  const Cut c = cut_of(P, D, A.Hq);
  const Launches l = launches_of(P, A.Hq, c);
  Parts parts = {};
  const size_t n = part_rows(P, A.Hq, c, parts.chunk0);
  parts.tickets = (int*)A.ws;
  parts.acc = A.ws + kTicketFloats;
  parts.ml = (float2*)(parts.acc + n * D);
  const int chunk = (int)l.chunk, step = (int)l.step;
  if (chunk && step) k_paged_attn<T, D, MODE, 3><<<chunk + step, 256, 0, st>>>(A, c, parts, chunk);
  else if (chunk) k_paged_attn<T, D, MODE, 1><<<chunk, 256, 0, st>>>(A, c, parts, chunk);
  else k_paged_attn<T, D, MODE, 2><<<step, 256, 0, st>>>(A, c, parts, 0);
  if (l.merge) {
    if (l.many) k_paged_merge<T, D, true><<<(int)l.merge, 256, 0, st>>>(A, c, parts, l.few_rows, l.step_ids);
    else k_paged_merge<T, D, false><<<(int)l.merge, 256, 0, st>>>(A, c, parts, l.few_rows, l.step_ids);
  }
  return hipGetLastError();
}

hipError_t launch_paged_attention(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  return dispatch(dtype, D, mode_of(A.S), [&](auto t, auto d, auto m) {
    return launch_attention<typename decltype(t)::type, decltype(d)::value, decltype(m)::value>(A, st);
  });
}

}  // namespace arkv
