// Attention of new tokens over a paged cache: rows of 16 bits or packed ones (PoolRow), all slots up to a token's own or those that a window or
// a tree of drafts leaves (Keys, RowView).
//
// The rows of a (sequence, kv-head) are its new tokens times the G query heads of the group: row r is token r / G, head
// r % G, so the heads of a group share every key and value that is fetched.  Two kernels divide the sequences between them:
//   paged_step   up to 16 rows (a generated token, a few drafted ones): bound by reading the pages (4 x 131071 rows x 8 heads in
//                377 us, 5.7 TB/s; 31 requests of up to 16384 rows in 184 us, 4.9 TB/s)
//   paged_chunk  more rows: bound by the matrix cores and the exponentials between them (2 x 2048 tokens of 16384, 32 heads, in
//                917 to 946 us, 1.09 to 1.12 PFLOP/s; rows of 8 bits, which pass through registers on their way to LDS: 1000 to 1060 us)
//   packed_step  paged_step over packed rows (4 x 131071 rows of 8 bits in 209 us, 5.3 TB/s; the 31 requests' rows of 4 bits in 61 us)
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
#pragma once
#include <algorithm>

#include "arkv_paged_mma.h"
#include "arkv_paged_rows.h"

namespace arkv {

constexpr int kStepWaves = 4;
constexpr int kStepMaxPiece = 2048;     // (twice that at most: a lane holds the page of one granule)
constexpr int kChunkRows = 128, kChunkKeys = 64;

// Waves per SIMD that a build's registers are for, and with that workgroups to a CU.  Single tokens' rows of 4 bits fit three; chunks of such rows at
// d = 64 do not without spills, which the exponentials of a cap hide (2 x 2048 tokens of 16384, 32 / 8 heads: 663 us with three, 634 with two, with a cap 907
// and 943; of 8 bits, whose three spill 8 to 17 registers, 660 and 658, 907 and 945).  Cut chunks were not compared: they are planned for the places there are.
__host__ __device__ constexpr int chunk_waves(int D, int bits, bool capped) { return D == 64 && (bits != 4 || capped) ? 3 : 2; }
__host__ __device__ constexpr int waves_of(int D, int MODE, int KIND, int BITS) {
  return KIND == 2 ? (D == 64 || BITS == 4 ? 3 : 2) : chunk_waves(D, BITS, MODE & 5);
}

// How a launch is cut.  step_piece, chunk_piece: keys per workgroup; the counts: pieces of the longest sequence.
// blocks: of kChunkRows rows, of all sequences, at most.  joined: the last workgroup of a (sequence, kv-head), chunk_joined: of a block
// and kv-head joins its pieces (tickets from chunk_ticket0 on), no launch is needed for that; chunk_spread: k_chunk_join does, else k_paged_merge.
// groups: of kStepRows rows, of all sequences, at most: all rows are paged_step's, group by group (0: sequences of few rows alone are, each a unit).
// places: workgroups that the chip holds, where the kernel chooses its pieces itself (chunk_piece: the shortest), else 0.
struct Cut { int step_piece, n_step, groups, chunk_piece, n_chunk, blocks, places, chunk_ticket0; bool joined, chunk_joined, chunk_spread; Which w; };
constexpr int kJoinPieces = 16;         // at most: a lane has all pieces' loads under way at once
// Limited sight and packed rows: sequences of more than kStepRows rows are paged_step's too, in groups of kStepRows, where all groups' tiles of 64
// keys are this few (25 drafts, 4 heads a group, 2100 rows: 14 us, as blocks 20; 8 x 16 drafts: 23 and 32; 64 drafts on 8192 rows, 17408 tiles of 16 bits:
// 47 and 34); and pieces of blocks are joined by a launch from more than kFewPieces on (9 pieces: 27 us joined in the launch, 20 by another).
constexpr int kGroupTiles = 8192, kGroupWorkgroups = 256, kFewPieces = 4;
constexpr int kJoinBlocks = 2048;       // pieces of blocks that are joined in the launch, at most (they take 67 KB of workspace each)

inline Cut cut_of(const Paged& P, const Sight& V, int D, int Hq) {
  Cut c = {};
  const int G = Hq / P.H;
  c.w = which_kernels(P, Hq);
  // kv: keys of the longest; have: workgroups without a cut; want: how many there should be; least, most: keys per piece
  auto pieces = [&](int kv, long long have, long long want, int least, int most, int unit, int& piece, int& n) {
    const long long p = (kv * std::max(1ll, have) + want - 1) / want;
    piece = (int)std::min<long long>(most, std::max<long long>(least, (p + unit - 1) / unit * unit));
    n = std::max(1, (kv + piece - 1) / piece);
  };
  int kv_step = most_keys(P, V, kStepRows / G);
  const int kv_chunk = most_keys(P, V, (kChunkRows - 1) / G + 2);
  // A workgroup for each CU, and no more pieces than the last workgroup joins (8 heads x 1024 rows: 6.6 us in pieces of 128
  // keys, 9.6 of 512, 12.4 in one; x 8192: 13.7 us in pieces of 128 and a launch that joins them, 11.9 of 512; 32 heads x
  // 8192: 29.6 us in pieces of 512, 28.7 of 1024), but no large ones: sequences differ in length, and the last round of
  // workgroups should end with the others (32 requests of 800 to 16384 rows x 8 heads: 177 us in pieces of 2048, 182 of
  // 4096; four of 131071 rows: 362 and 354).  Fewer than 16 heads do not fill the chip in 16 pieces.
  const long long units = (long long)P.B * P.H;
  // Rows of 4 bits are read in half the time (31 requests of 800 to 16384 rows x 8 heads: 66 us in pieces of 2048 keys, 61 of 4096; of 8 bits, four of 131071
  // rows: 209 and 210).
  const int longest = V.bits == 4 ? 2 * kStepMaxPiece : kStepMaxPiece;
  pieces(kv_step, units, std::min(256ll, kJoinPieces * units), 128, units < 16 ? longest / 2 : longest, 128, c.step_piece, c.n_step);
  // One workgroup for each CU; then for every place on the chip, two or three to a CU, in larger pieces (1686 tokens on up to 3001
  // rows, 12 heads: 46 us in pieces of 1024 keys, 42 of 512; d = 128, 512 tokens on 4100 rows, 16 heads, 7 single tokens: 66 us in pieces of
  // 1024, 70 of 768, 82 of 512; 128 tokens on 1024 rows: 28 us in one piece, 22 in
  // pieces of 256).
  const long long rows = (long long)P.N * G, blocks = (rows + kChunkRows - 1) / kChunkRows * P.H;
  const int places = 256 * chunk_waves(D, V.bits, V.capped);
  int alone, n_alone;
  pieces(kv_chunk, blocks, 256, 256, 1 << 28, kChunkKeys, alone, n_alone);
  pieces(kv_chunk, blocks, places, D == 64 ? 512 : 1024, 1 << 28, kChunkKeys, c.chunk_piece, c.n_chunk);
  if (alone < c.chunk_piece) { c.chunk_piece = alone; c.n_chunk = n_alone; }
  if (V.bits && c.w.chunk) {
    const long long groups = rows / kStepRows + std::min<long long>(P.B, rows), keys = most_keys(P, V, (kStepRows - 1) / G + 2);
    int piece, n;
    pieces((int)keys, groups * P.H, kGroupWorkgroups, std::max(128, ((int)keys + 2047) / 2048 * 128), kStepMaxPiece, 128, piece, n);
    if (groups * P.H <= kJoinUnits && groups * P.H * ((keys + 63) / 64) <= kGroupTiles && n <= kJoinPieces) {
      c.groups = (int)groups;
      c.step_piece = piece;
      c.n_step = n;
      c.w = {true, false, kStepRows};
      c.joined = true;
      return c;
    }
  }
  c.joined = c.n_step <= kJoinPieces && units <= kJoinUnits;
  // (a sequence that is the chunk kernel's has more rows than the step kernel takes)
  c.blocks = (int)(rows / kChunkRows + std::min<long long>(P.B, c.w.step ? rows / (kStepRows + 1) : P.B));
  c.chunk_ticket0 = c.w.step && c.joined ? (int)units : 0;
  // (512 tokens on 4100 rows, 16 heads, beside 7 single tokens: 60 us, with a launch that joins 70)
  c.chunk_joined = c.n_chunk <= kJoinPieces && (long long)c.blocks * P.H + c.chunk_ticket0 <= kJoinUnits &&
                   (long long)c.blocks * P.H * c.n_chunk <= kJoinBlocks;
  if (V.bits) {
    // the kernel may find that pieces down to half as long fit the chip at once
    const int half = std::max(D == 64 ? 256 : 512, c.chunk_piece / 2 / kChunkKeys * kChunkKeys), n = (kv_chunk + half - 1) / half;
    if (c.n_chunk > 1 && P.B <= 64 && (long long)c.blocks * P.H * n <= kJoinBlocks && half < c.chunk_piece) {
      c.chunk_piece = half;
      c.n_chunk = n;
      c.places = places;
    }
    c.chunk_joined = c.chunk_joined && c.n_chunk <= kFewPieces;
    c.chunk_spread = c.w.chunk && !c.chunk_joined && c.n_chunk > 1 && (long long)c.blocks * P.H * c.n_chunk <= kJoinBlocks;
  }
  return c;
}

// Pieces' results: sums [row][D] and (reference, denominator) [row].  Rows of paged_step: ((unit * n_step + piece) * 16 +
// row), behind them rows of paged_chunk: (piece * N + token) * Hq + head, or, where its workgroups or k_chunk_join join them, kChunkRows rows of
// ((block * H + head) * n_chunk + piece), each wave's as they lie in its lanes.
// split: what k_chunk_join needs of each block of rows and kv-head: pieces, first token, tokens, which block of the sequence's.
struct Parts { float* acc; float2* ml; int* tickets; size_t chunk0; int4* split; };

inline size_t part_rows(const Paged& P, int Hq, const Cut& c, size_t& chunk0) {
  chunk0 = c.w.step && c.n_step > 1 ? (size_t)(c.groups ? c.groups : P.B) * P.H * c.n_step * kStepRows : 0;
  if (!c.w.chunk || c.n_chunk == 1) return chunk0;
  return chunk0 + (c.chunk_joined || c.chunk_spread ? (size_t)c.blocks * P.H * c.n_chunk * kChunkRows : (size_t)c.n_chunk * P.N * Hq);
}

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

// Blocks of ROWS rows that a sequence of more than `few` makes.
template <int ROWS> __host__ __device__ __forceinline__ int row_blocks(int nq, int G, int few) { return nq * G <= few ? 0 : (nq * G + ROWS - 1) / ROWS; }

// Sequence and block of the rank-th block of a launch; the lanes of a wave look at 64 sequences at a time.
template <int ROWS>
__device__ __forceinline__ bool find_block(const Paged& P, int G, int few, int rank, int lane, int& b, int& blk, Seq& s) {
  for (int i = 0; i < P.B; i += 64) {
    const Seq own = seq_of(P, min(i + lane, P.B - 1));
    const int mine = i + lane < P.B ? row_blocks<ROWS>(own.nq, G, few) : 0;
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

// ---- few rows -----------------------------------------------------------------------------------------

// One workgroup = one piece of a (sequence, kv-head); its waves take a quarter of the piece each, 32 keys at a time, with
// 16x16x32 MFMAs (lane: row lane % 16, keys 4 (lane / 16) .. + 3 of each granule).  Keys come from memory in operand
// layout; values in whole rows, through LDS of the wave's own.  A tile's loads are in flight while the tile before it
// is worked on.
// Pages of a wave's granules, from key w0 on, of which there are 64 at most: lane i holds the page of granule i.  One that is not there, or lies
// behind the keys below `end`, becomes page 0, whose rows nobody sees.
template <bool SIGHT> struct GranulePages {
  const Paged& P;
  const Keys<SIGHT>& keys;
  int h, w0, page;
  uint64_t there;
  __device__ __forceinline__ GranulePages(const Paged& P, const Keys<SIGHT>& keys, int b, int h, int w0, int end, int lane) : P(P), keys(keys), h(h), w0(w0) {
    const int j = w0 + 16 * lane;
    page = j < end ? P.table[(size_t)b * P.width + (keys.slot(j) >> P.lg_page)] : -1;
    const bool ok = (unsigned)page < (unsigned)P.n_pages;
    there = __ballot(ok);
    if (!ok) page = 0;
  }
  __device__ __forceinline__ size_t row(int g) const {             // first row of granule g
    const int p = __builtin_amdgcn_readlane(page, g);
    return (size_t)(unsigned)(((p * P.H + h) << P.lg_page) + (keys.slot(w0 + 16 * g) & ((1 << P.lg_page) - 1)));
  }
};

template <int D> struct StepLds {
  union {                                 // a wave's values while it works, its sums behind that
    uint16_t v[32][D + 16];               // (the pitch: transposing reads of 16 rows meet each bank twice, as they must)
    float acc[kStepRows][D + 4];
  } w[kStepWaves];
  float2 ml[kStepWaves][kStepRows];
  int last;                               // whether this workgroup's piece was the last one to be finished
};

// One of the np pieces that a (sequence, kv-head) is cut into; first: rows of the workspace in front of its first piece's.  ticket: of the
// launch that joins its pieces itself; null: another launch does.
struct Piece { int np, index; size_t first; int* ticket; };

// The waves' results of a piece together: the row's output where the piece is the only one, else into the workspace, from where the
// last workgroup of the sequence's head joins them.
template <typename T, int D>
__device__ __forceinline__ void step_finish(const PagedAttnArgs& A, const Parts& parts, StepLds<D>& sm, const Seq& s, int r0, int h, const Piece& pc,
                                            const f32x4g (&acc)[D / 16], float m, float l) {
  constexpr int CB = D / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, gq = lane >> 4, R = min(s.nq * A.G - r0, kStepRows), np = pc.np;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int c = 0; c < CB; ++c) *reinterpret_cast<f32x4g*>(&sm.w[wave].acc[n][16 * c + 4 * gq]) = acc[c];
  if (gq == 0) sm.ml[wave][n] = make_float2(m, l);
  __syncthreads();
  auto finish = [&](int r, int c, f32x4g o, float mm, float ll) {  // four channels of a row's result
    const size_t orow = (size_t)(s.q0 + (r0 + r) / A.G) * A.Hq + h * A.G + (r0 + r) % A.G;
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
      o += f * *reinterpret_cast<const f32x4g*>(&sm.w[w].acc[r][c]);
    }
    if (np > 1) {
      const size_t pr = pc.first + pc.index * kStepRows + r;
      put4(parts.acc + pr * D + c, o);
      if (c == 0) put2(parts.ml + pr, mm, ll);
    } else {
      finish(r, c, o, mm, ll);
    }
  }
  if (np == 1 || !pc.ticket) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // this wave's stores are where everyone sees them
  __syncthreads();
  if (threadIdx.x == 0) {
    const int drawn = __hip_atomic_fetch_add(pc.ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sm.last = drawn == np - 1;
    if (sm.last) __hip_atomic_store(pc.ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // as the next call wants it
  }
  __syncthreads();
  if (!sm.last) return;
  for (int it = threadIdx.x; it < R * (D / 4); it += 64 * kStepWaves) {
    const int r = it / (D / 4), c = 4 * (it % (D / 4));
    float2 ml[kJoinPieces];
    f32x4g x[kJoinPieces];
#pragma unroll
    for (int p = 0; p < kJoinPieces; ++p) {
      if (p < np) {
        const size_t pr = pc.first + p * kStepRows + r;
        ml[p] = take2(parts.ml + pr);
        x[p] = take4(parts.acc + pr * D + c);
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

template <typename T, int D, int MODE, bool SIGHT>
__device__ __forceinline__ void paged_step(const PagedAttnArgs& A, const Parts& parts, StepLds<D>& sm, const Seq& s, int b, int r0, int h, int prefix,
                                           const Keys<SIGHT>& keys, int p0, int p1, const Piece& pc) {
  constexpr int CAP = Mode<MODE>::cap;
  constexpr bool DIST = Mode<MODE>::dist;
  typedef PoolRow<T, D, 16> Row;
  constexpr int KK = D / 32, CB = D / 16;                          // k-steps, channel blocks
  constexpr int CPR = Row::kLanes, RPI = 64 / CPR, VI = 32 / RPI;  // lanes per row, rows per load, loads of a value tile
  const Paged& P = A.P;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, gq = lane >> 4, R = min(s.nq * A.G - r0, kStepRows);
  const int row = r0 + (n < R ? n : 0);
  const RowView<SIGHT> view(A.V, s, prefix, row / A.G, n < R);
  const int hq = h * A.G + row % A.G, tok = s.q0 + row / A.G;
  const Logit lg(A.S);
  const float slope = DIST ? A.S.slopes[hq] * kLog2e : 0.f;
  const int qp = DIST ? A.S.q_pos[tok] : 0;

  u32x4g q[KK];
  {
    const T* p = (const T*)A.q.p + (size_t)tok * A.q.ts + (size_t)hq * A.q.hs;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = *reinterpret_cast<const u32x4g*>(p + Row::channel(gq, kk));
  }
  // this wave's of the piece's keys p0 .. p1 - 1: [w0, w1), whole tiles
  const int tiles = (p1 - p0 + 31) / 32, per = (tiles + kStepWaves - 1) / kStepWaves;
  const int t0 = min(per * wave, tiles), t1 = min(t0 + per, tiles);
  const int w0 = p0 + 32 * t0;
  const GranulePages<SIGHT> pages(P, keys, b, h, w0, p1, lane);
  auto granule_row = [&](int g) { return pages.row(g); };

  typename Row::Keys kb[2][2];
  typename Row::Chunk vb[VI];
  auto load_k = [&](int t, typename Row::Keys (&to)[2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) Row::load_keys(A, granule_row(2 * t + g), n, gq, to[g]);
  };
  auto load_v = [&](int t) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const size_t first = granule_row(2 * t + g);
#pragma unroll
      for (int i = 0; i < VI / 2; ++i) Row::load_chunk(P.v, A.v_scale, first + i * RPI + lane / CPR, lane % CPR, vb[g * (VI / 2) + i]);
    }
  };
  f32x4g acc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) acc[c] = f32x4g{0.f, 0.f, 0.f, 0.f};
  float m = kUnset, l = 0.f;
  const int nt = t1 - t0;

  auto tile = [&](int t, const typename Row::Keys (&kc)[2]) {
    const int j0 = w0 + 32 * t;
    f32x4g x[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      x[g] = f32x4g{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) x[g] = Mfma<T>::m16(Row::operand(kc[g], n, gq, kk), q[kk], x[g]);
    }
    const uint32_t ok = (uint32_t)(pages.there >> (2 * t)) & 3;
    const bool masked = !keys.all_seen(j0, 32) || ok != 3;
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
    u32x4g vw[VI][Row::kOut];                                      // values, as the product takes them
#pragma unroll
    for (int i = 0; i < VI; ++i) Row::expand(vb[i], 0, 0, vw[i]);
    if (masked) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const auto seen = view.granule(keys.slot(j0 + 16 * g), ok >> g & 1, 4 * gq);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[g][i] = seen.at(i) ? x[g][i] * mul : -INFINITY;
      }
      mul = 1.f;
      // a value that is not finite would spoil the rows that do not see it: it leaves the product, and is added below
#pragma unroll
      for (int i = 0; i < VI; ++i) {
        uint32_t any = 0;
#pragma unroll
        for (int o = 0; o < Row::kOut; ++o)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t f = not_finite<T>(vw[i][o][e]);
            vw[i][o][e] &= ~f;
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
#pragma unroll
      for (int o = 0; o < Row::kOut; ++o)
        *reinterpret_cast<u32x4g*>(&sm.w[wave].v[RPI * i + lane / CPR][8 * (Row::kOut * (lane % CPR) + o)]) = vw[i][o];
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
      const s16x4g a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)&sm.w[wave].v[4 * gq + (n >> 2)][16 * c + 4 * (n & 3)]);
      const s16x4g a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)&sm.w[wave].v[16 + 4 * gq + (n >> 2)][16 * c + 4 * (n & 3)]);
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
      const bool seen = view.granule(keys.slot(j0 + 16 * g), ok >> g & 1, 0).at(j & 15);
      const size_t vrow = granule_row(2 * t + g) + (j & 15);
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = Row::value(A, vrow, 16 * c + 4 * gq + e);
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
  step_finish<T, D>(A, parts, sm, s, r0, h, pc, acc, m, l);
}

// The same over packed rows, 64 keys at a time: a tile's codes are few registers, and are requested again as soon as they are
// expanded, so that most of a tile's time lies between request and use (8 bits: 17 KB a wave under way, 4 bits: 9 KB).  A lane's keys of a
// row are whole chunks of it (PoolRow::channel).
template <typename T, int D, int MODE, int BITS>
__device__ __forceinline__ void packed_step(const PagedAttnArgs& A, const Parts& parts, StepLds<D>& sm, const Seq& s, int b, int r0, int h, int prefix,
                                            const Keys<true>& keys, int p0, int p1, const Piece& pc) {
  constexpr int CAP = Mode<MODE>::cap;
  constexpr bool DIST = Mode<MODE>::dist;
  typedef PoolRow<T, D, BITS> Row;
  constexpr int KK = D / 32, CB = D / 16;                          // k-steps, channel blocks
  constexpr int CPR = Row::kLanes, RPI = 64 / CPR, VI = 32 / RPI;  // lanes per row, rows per load, loads of half a tile's values
  const Paged& P = A.P;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, gq = lane >> 4, R = min(s.nq * A.G - r0, kStepRows);
  const int row = r0 + (n < R ? n : 0);
  const RowView<true> view(A.V, s, prefix, row / A.G, n < R);
  const int hq = h * A.G + row % A.G, tok = s.q0 + row / A.G;
  const Logit lg(A.S);
  const float slope = DIST ? A.S.slopes[hq] * kLog2e : 0.f;
  const int qp = DIST ? A.S.q_pos[tok] : 0;

  u32x4g q[KK];
  {
    const T* p = (const T*)A.q.p + (size_t)tok * A.q.ts + (size_t)hq * A.q.hs;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = *reinterpret_cast<const u32x4g*>(p + Row::channel(gq, kk));
  }
  // this wave's of the piece's keys p0 .. p1 - 1: [w0, w1), a multiple of 32 from p0 on
  const int halves = (p1 - p0 + 31) / 32, per = (halves + kStepWaves - 1) / kStepWaves;
  const int w0 = min(p0 + 32 * per * wave, p1), w1 = min(w0 + 32 * per, p1), nt = (w1 - w0 + 63) / 64;
  const GranulePages<true> pages(P, keys, b, h, w0, w1, lane);

  typename Row::Keys kr[4];
  typename Row::Chunk vr[2][VI];
  auto load_k = [&](int t) {
#pragma unroll
    for (int g = 0; g < 4; ++g) Row::load_keys(A, pages.row(4 * t + g), n, gq, kr[g]);
  };
  auto load_v = [&](int t, int half) {
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const int first = RPI * i + lane / CPR;                      // (a load's rows lie in one granule)
      Row::load_chunk(P.v, A.v_scale, pages.row(4 * t + 2 * half + RPI * i / 16) + (first & 15), lane % CPR, vr[half][i]);
    }
  };
  f32x4g acc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) acc[c] = f32x4g{0.f, 0.f, 0.f, 0.f};
  float m = kUnset, l = 0.f;
  if (nt > 0) {
    load_k(0);
    load_v(0, 0);
    load_v(0, 1);
  }
  for (int t = 0; t < nt; ++t) {
    const int j0 = w0 + 64 * t;
    f32x4g x[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      x[g] = f32x4g{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) x[g] = Mfma<T>::m16(Row::operand(kr[g], n, gq, kk), q[kk], x[g]);
    }
    const int next = min(t + 1, nt - 1);                           // (behind the last tile that one again: a branch here would be waited for)
    load_k(next);
    const uint32_t ok = (uint32_t)(pages.there >> (4 * t)) & 15;
    const bool masked = !keys.all_seen(j0, 64) || ok != 15;
    float mul = lg.mul;
    if (CAP || DIST) {
      mul = 1.f;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[g][i] = lg.logit<CAP>(x[g][i]);
        if (DIST) {
          const int4 kp = *reinterpret_cast<const int4*>(P.pos + pages.row(4 * t + g) + 4 * gq);
          x[g][0] = fmaf(-slope, fabsf((float)(qp - kp.x)), x[g][0]);
          x[g][1] = fmaf(-slope, fabsf((float)(qp - kp.y)), x[g][1]);
          x[g][2] = fmaf(-slope, fabsf((float)(qp - kp.z)), x[g][2]);
          x[g][3] = fmaf(-slope, fabsf((float)(qp - kp.w)), x[g][3]);
        }
      }
    }
    if (masked) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const auto seen = view.granule(keys.slot(j0 + 16 * g), ok >> g & 1, 4 * gq);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[g][i] = seen.at(i) ? x[g][i] * mul : -INFINITY;
      }
      mul = 1.f;
    }
    float p[16];
    auto probs = [&]() {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
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
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[i >> 2][i & 3] * mul);
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
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const u32x4g pb = {Mfma<T>::pack(p[8 * half], p[8 * half + 1]), Mfma<T>::pack(p[8 * half + 2], p[8 * half + 3]),
                         Mfma<T>::pack(p[8 * half + 4], p[8 * half + 5]), Mfma<T>::pack(p[8 * half + 6], p[8 * half + 7])};
      uint32_t odd = 0;                                            // keys of this half whose values are not all finite
#pragma unroll
      for (int i = 0; i < VI; ++i) {
        u32x4g w[Row::kOut];
        Row::expand(vr[half][i], lane / CPR, lane % CPR, w);
        if (masked) {
          // a value that is not finite would spoil the rows that do not see it: it leaves the product, and is added below
          uint32_t any = 0;
#pragma unroll
          for (int o = 0; o < Row::kOut; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t f = not_finite<T>(w[o][e]);
              w[o][e] &= ~f;
              any |= f;
            }
          const uint64_t who = __ballot(any != 0);
#pragma unroll
          for (int r = 0; r < RPI; ++r)
            if (who >> (CPR * r) & ((1ull << CPR) - 1)) odd |= 1u << (RPI * i + r);
        }
#pragma unroll
        for (int o = 0; o < Row::kOut; ++o)
          *reinterpret_cast<u32x4g*>(&sm.w[wave].v[RPI * i + lane / CPR][8 * (Row::kOut * (lane % CPR) + o)]) = w[o];
      }
      load_v(next, half);
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const s16x4g a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)&sm.w[wave].v[4 * gq + (n >> 2)][16 * c + 4 * (n & 3)]);
        const s16x4g a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)&sm.w[wave].v[16 + 4 * gq + (n >> 2)][16 * c + 4 * (n & 3)]);
        const u32x2g w0_ = __builtin_bit_cast(u32x2g, a0), w1_ = __builtin_bit_cast(u32x2g, a1);
        acc[c] = Mfma<T>::m16(u32x4g{w0_[0], w0_[1], w1_[0], w1_[1]}, pb, acc[c]);
      }
      while (odd) {                                                // (uniform; hardly ever)
        const int j = __builtin_ctz(odd);
        odd &= odd - 1;
        const int g = j >> 4, i = j & 3, from = (j & 12) >> 2;
        float pj = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e == 4 * g + i) pj = Mfma<T>::get(opaque(pb[e / 2]), e & 1);
        pj = __shfl(pj, n + 16 * from);
        const int granule = 4 * t + 2 * half + g;
        const bool seen = view.granule(keys.slot(w0 + 16 * granule), ok >> (2 * half + g) & 1, 0).at(j & 15);
        const size_t vrow = pages.row(granule) + (j & 15);
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float w = Row::value(A, vrow, 16 * c + 4 * gq + e);
            if (seen && !(fabsf(w) < INFINITY)) acc[c][e] += pj * w;
          }
      }
    }
  }
  step_finish<T, D>(A, parts, sm, s, r0, h, pc, acc, m, l);
}

// The keys of a row of 16-bit pages, or of packed ones.
template <typename T, int D, int MODE, int BITS, bool SIGHT, typename... Rest>
__device__ __forceinline__ void few_rows(const PagedAttnArgs& A, const Parts& parts, StepLds<D>& sm, const Rest&... rest) {
  if constexpr (BITS == 16) paged_step<T, D, MODE, SIGHT>(A, parts, sm, rest...);
  else packed_step<T, D, MODE, BITS>(A, parts, sm, rest...);
}

// Workgroup id of a launch for few rows: unit by unit, piece by piece.  In groups: a unit is kStepRows rows of a sequence's, of as many as it has.
template <typename T, int D, int MODE, int BITS, bool SIGHT>
__device__ __forceinline__ void cut_step(const PagedAttnArgs& A, const Cut& cut, const Parts& parts, StepLds<D>& sm, int id) {
  const Paged& P = A.P;
  const bool grouped = SIGHT && cut.groups;
  const int units = (grouped ? cut.groups : P.B) * P.H, unit = id % units, piece = id / units, h = unit % P.H;
  int b = unit / P.H, group = 0;
  Seq s;
  if (grouped) {
    if (!find_block<kStepRows>(P, A.G, 0, b, threadIdx.x & 63, b, group, s)) return;
  } else {
    s = seq_of(P, b);
    if (s.nq == 0 || s.nq * A.G > kStepRows) return;
  }
  const int r0 = group * kStepRows, prefix = A.S.prefix ? A.S.prefix[b] : 0;
  const Keys<SIGHT> keys(A.V, s, prefix, r0 / A.G, grouped ? min(s.nq * A.G - 1, r0 + kStepRows - 1) / A.G : s.nq - 1);
  const int np = max(1, (keys.end + cut.step_piece - 1) / cut.step_piece);
  if (piece >= np) return;
  const int p0 = piece * cut.step_piece, p1 = min(p0 + cut.step_piece, keys.end);
  const Piece pc = {np, piece, (size_t)unit * cut.n_step * kStepRows, cut.joined ? parts.tickets + unit * kTicketWords : nullptr};
  few_rows<T, D, MODE, BITS, SIGHT>(A, parts, sm, s, b, r0, h, prefix, keys, p0, p1, pc);
}

// ---- many rows ----------------------------------------------------------------------------------------

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

// combine(sums, reference, denominator, token's row): what becomes of a lane's part of a row; whether the result is the row's now.
template <typename T, int D, int MODE, int BITS, bool SIGHT, typename F>
__device__ __forceinline__ void paged_chunk(const PagedAttnArgs& A, ChunkLds<D>& sm, const Seq& s, int b, int blk, int h, int prefix,
                                            const Keys<SIGHT>& keys, int p0, int p1, F combine) {
  constexpr int CAP = Mode<MODE>::cap;
  constexpr bool DIST = Mode<MODE>::dist;
  typedef PoolRow<T, D, BITS> Row;
  constexpr int KK = D / 16, CB = D / 32, CPR = D / 8;
  constexpr int RPI = 64 / Row::kLanes, LPG = 16 / RPI;            // rows per load, loads of a granule
  const Paged& P = A.P;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int R = s.nq * A.G, r0 = blk * kChunkRows, end = keys.end;
  const int r = r0 + 32 * wave + n;
  const int rc = min(r, R - 1);
  const RowView<SIGHT> view(A.V, s, prefix, rc / A.G, r < R);
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
  const int nt = (p1 - p0 + kChunkKeys - 1) / kChunkKeys;
  const int32_t* table = P.table + (size_t)b * P.width;
  const int in_page = (1 << P.lg_page) - 1;

  // where this lane's chunk of a 1 KB load lies in a granule: row RPI i + lane / CPR
  uint32_t koff[LPG], voff[LPG];
  if constexpr (BITS == 16) {
#pragma unroll
    for (int i = 0; i < LPG; ++i) {
      const int rr = RPI * i + lane / CPR;
      koff[i] = 2 * (rr * D + 8 * k_chunk<D>(rr, lane % CPR));
      voff[i] = 2 * (rr * D + 8 * v_chunk<D>(rr, lane % CPR));
    }
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
    int page = j < p1 ? table[keys.slot(j) >> P.lg_page] : -1;
    const bool ok = (unsigned)page < (unsigned)P.n_pages;
    there[which] = __ballot(ok);
    pages[which] = ok ? page : 0;
  };
  auto granule_row = [&](int which, int t, int g) {                // first row of granule g of tile t
    const int page = __builtin_amdgcn_readlane(which ? pages[1] : pages[0], 4 * (t & 15) + g);
    return (size_t)(unsigned)(((page * P.H + h) << P.lg_page) + (keys.slot(p0 + kChunkKeys * t + 16 * g) & in_page));
  };
  // Packed rows come through registers: they are requested with the tile before (fetch), and put behind its work (put).
  typename Row::Chunk kr[LPG], vr[LPG];
  auto put = [&](int buf) {
    if constexpr (BITS != 16) {
#pragma unroll
      for (int i = 0; i < LPG; ++i) {
        const int rr = RPI * i + lane / Row::kLanes, in = lane % Row::kLanes;
        uint16_t* const kt = sm.k[buf] + wave * 16 * D + rr * D;
        uint16_t* const vt = sm.v[buf] + wave * 16 * D + rr * D;
        u32x4g w[Row::kOut];
        Row::expand(kr[i], rr, in, w);
#pragma unroll
        for (int o = 0; o < Row::kOut; ++o) *reinterpret_cast<u32x4g*>(kt + 8 * k_chunk<D>(rr, Row::kOut * in + o)) = w[o];
        Row::expand(vr[i], rr, in, w);
#pragma unroll
        for (int o = 0; o < Row::kOut; ++o) *reinterpret_cast<u32x4g*>(vt + 8 * v_chunk<D>(rr, Row::kOut * in + o)) = w[o];
      }
    }
  };
  auto fetch = [&](int which, int t, int buf) {                    // this wave's granule of tile t
    const size_t row = granule_row(which, t, wave);
    if constexpr (BITS == 16) {
      const T* kp = (const T*)P.k + row * D;
      const T* vp = (const T*)P.v + row * D;
      const uint32_t at = (uint32_t)(buf * kChunkKeys * D * 2 + wave * 16 * D * 2);
#pragma unroll
      for (int i = 0; i < LPG; ++i) load_lds(kp, koff[i], lds_k + at + 1024 * i);
#pragma unroll
      for (int i = 0; i < LPG; ++i) load_lds(vp, voff[i], lds_v + at + 1024 * i);
    } else {
#pragma unroll
      for (int i = 0; i < LPG; ++i) Row::load_chunk(P.k, A.k_scale, row + RPI * i + lane / Row::kLanes, lane % Row::kLanes, kr[i]);
#pragma unroll
      for (int i = 0; i < LPG; ++i) Row::load_chunk(P.v, A.v_scale, row + RPI * i + lane / Row::kLanes, lane % Row::kLanes, vr[i]);
    }
    const uint32_t at_pos = __builtin_amdgcn_readfirstlane(lds_pos + 4 * (buf * kChunkKeys + 16 * wave));
    if (DIST && lane < 16) load_lds4(P.pos + row + lane, at_pos);
  };

  f32x16g acc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
  // The row's softmax reference; rows that see none of this piece need none.
  float m = view.end() > keys.slot(p0) ? kUnset : 0.f, l = 0.f;
  load_pages(0, 0);
  if (SIGHT && tid < 2) sm.odd[tid] = 0;
  if (nt > 0) {
    fetch(0, 0, 0);
    put(0);
  }
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
    const bool masked = !keys.all_seen(j0, kChunkKeys) || ok != 15;
    uint64_t odd = 0;
    if (masked) {
      // Values that are not finite would spoil the rows that do not see them: they leave the product, and are added below.
      // (Under a window a quarter of the tiles is masked.  There the words are zero from before, and a chunk is first looked at as a whole.)
      if constexpr (!SIGHT) {
        if (tid < 2) sm.odd[tid] = 0;
        __syncthreads();
      }
      constexpr int PT = kChunkKeys * CPR / 256;                   // chunks per thread
      bool look = true;
      if constexpr (SIGHT) {
        u16x2g most = {0, 0};
#pragma unroll
        for (int i = 0; i < PT; ++i) {
          const u32x4g w = *reinterpret_cast<const u32x4g*>(&sm.v[buf][8 * (tid + 256 * i)]);
#pragma unroll
          for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2g, w[e] & 0x7FFF7FFFu));
        }
        look = most[0] >= Mfma<T>::kExp || most[1] >= Mfma<T>::kExp;
      }
      if (look)
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
      if (SIGHT && odd) {
        __syncthreads();
        if (tid < 2) sm.odd[tid] = 0;
      }
    }
    if (SIGHT && r0 + 32 * wave >= R) {                            // no rows of this wave's: it only fetches
      if (t + 1 < nt) put(buf ^ 1);
      return;
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
        auto seen = view.granule(keys.slot(j0 + 16 * g), ok >> g & 1, 4 * hh);
        if constexpr (!SIGHT) seen.left = (int)opaque(seen.left);  // (what depends on it stays in this branch)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = 8 * (g & 1) + i;
          if constexpr (SIGHT) x[g >> 1][e] = seen.pick(8 * (i >> 2) + (i & 3), x[g >> 1][e]);
          else if (!seen.at(8 * (i >> 2) + (i & 3))) x[g >> 1][e] = -INFINITY;
        }
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
      const bool seen = view.granule(keys.slot(j0 + (j & 48)), true, 0).at(j & 15);
      const size_t vrow = granule_row(0, t, j >> 4) + (j & 15);
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float w = Row::value(A, vrow, 32 * c + 8 * (i >> 2) + 4 * hh + (i & 3));
          if (seen && !(fabsf(w) < INFINITY)) acc[c][i] += pj * w;
        }
    }
    if (t + 1 < nt) put(buf ^ 1);
  };
  if constexpr (DIST || D == 64 || (BITS != 16 && CAP)) {                                 // (two copies of the tile do not fit the registers of two and three waves per SIMD)
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
  if (!combine(acc, m, l, r < R, orow)) return;
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

// Keys of a piece.  The host knows bounds of the lengths alone; where it leaves the choice (cut.places), the pieces are the shortest, from
// cut.chunk_piece on, with which all blocks' are on the chip at once, by load_of's count (eight requests of 25 to 64 drafts, 4472 to 8192 rows of 8 bits: 1408
// keys, which the bounds give, make 536 workgroups, 83 us; 1536 make 504, 69 us).
// sum(f): of f(blocks, tiles) over the sequences, up to 64 of them.
template <typename Sum> __host__ __device__ __forceinline__ int chosen_piece(const Cut& cut, Sum sum) {
  const int most = 1 << 24, whole = sum([](int blocks, int tiles) { const int n = blocks * (tiles >> 4); return n < 1 << 24 ? n : 1 << 24; });
  const long long even = whole * 16ll / cut.places;
  int piece = even < most ? (int)even : most;
  if (piece < cut.chunk_piece / kChunkKeys) piece = cut.chunk_piece / kChunkKeys;
  for (int i = 0; i < 24 && sum([=](int blocks, int tiles) { return blocks * ((tiles + piece - 1) / piece); }) > cut.places; ++i) piece += (piece + 15) / 16;
  return piece * kChunkKeys;
}
// A sequence's blocks, of all kv-heads, and 64-key tiles of its last kChunkRows rows: as many as any block has, also under a window, where a short
// last block sees fewer, and other blocks begin elsewhere in a granule or a token.  All count as much, so the pieces may be longer than they need to be
// (causal blocks in front see fewer keys); workgroups for few rows in the same launch are not counted.
struct Load { int blocks, tiles; };
__host__ __device__ __forceinline__ Load load_of(const Paged& P, const Sight& V, const Seq& s, int prefix, int G, int few) {
  const int R = s.nq * G, blocks = row_blocks<kChunkRows>(s.nq, G, few);
  const int tiles = (Keys<true>(V, s, prefix, (R > kChunkRows ? R - kChunkRows : 0) / G - 16, s.nq - 1).end + kChunkKeys - 1) / kChunkKeys;
  return {blocks * P.H, tiles};
}
__device__ __forceinline__ int chunk_piece(const PagedAttnArgs& A, const Cut& cut, int lane) {
  if (!cut.places) return cut.chunk_piece;
  const Paged& P = A.P;
  const int b = min(lane, P.B - 1);
  const Load own = load_of(P, A.V, seq_of(P, b), A.S.prefix ? A.S.prefix[b] : 0, A.G, cut.w.few);
  const int blocks = lane < P.B ? own.blocks : 0, tiles = own.tiles;
  return chosen_piece(cut, [=](auto f) {
    int x = f(blocks, tiles);
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return __builtin_amdgcn_readfirstlane(x);
  });
}

// Workgroup id of a launch that is cut: blocks of each kv-head, piece by piece.
template <typename T, int D, int MODE, int BITS, bool SIGHT>
__device__ __forceinline__ void cut_chunk(const PagedAttnArgs& A, const Cut& cut, const Parts& parts, ChunkLds<D>& sm, int id) {
  constexpr int CB = D / 32;
  const Paged& P = A.P;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int h = id % P.H, piece = id / (cut.blocks * P.H), bh = id % (cut.blocks * P.H);
  int b, blk;
  Seq s;
  const bool split = SIGHT && cut.chunk_spread && piece == 0 && tid == 0;
  if (!find_block<kChunkRows>(P, A.G, cut.w.few, bh / P.H, lane, b, blk, s)) {
    if (split) parts.split[bh] = int4{0, 0, 0, 0};
    return;
  }
  const int prefix = A.S.prefix ? A.S.prefix[b] : 0;
  const int r0 = blk * kChunkRows;
  const Keys<SIGHT> keys(A.V, s, prefix, r0 / A.G, min(s.nq * A.G - 1, r0 + kChunkRows - 1) / A.G);
  const int length = SIGHT ? chunk_piece(A, cut, lane) : cut.chunk_piece, np = max(1, (keys.end + length - 1) / length);
  if (piece >= np) return;
  if (split) parts.split[bh] = int4{np, s.q0, s.nq, blk};
  const int p0 = piece * length, p1 = min(p0 + length, keys.end);
  paged_chunk<T, D, MODE, BITS, SIGHT>(A, sm, s, b, blk, h, prefix, keys, p0, p1, [&](f32x16g (&acc)[CB], float& m, float& l, bool live, size_t orow) {
    if (np > 1 && !cut.chunk_joined && !cut.chunk_spread) {
      if (!live) return false;
      const size_t pr = parts.chunk0 + (size_t)piece * P.N * A.Hq + orow;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<f32x4g*>(parts.acc + pr * D + 32 * c + 8 * e + 4 * hh) =
              f32x4g{acc[c][4 * e], acc[c][4 * e + 1], acc[c][4 * e + 2], acc[c][4 * e + 3]};
      if (hh == 0) parts.ml[pr] = make_float2(m, l);
      return false;
    }
    if (np > 1) {
      // 8 bytes per lane, adjacent lanes adjacent: where wave w's two channels i, i + 1 of block c lie in a piece's rows
      const size_t row0 = parts.chunk0 + (size_t)bh * cut.n_chunk * kChunkRows + 32 * wave;
      const uint32_t at = 8 * (uint32_t)lane;                        // (beside a uniform address: 64 bits a lane would not fit the registers)
      auto sums = [&](int p, int c, int i) {
        return reinterpret_cast<float2*>(reinterpret_cast<char*>(parts.acc + (row0 + (size_t)p * kChunkRows) * D) + (8 * c + i / 2) * 512 + at);
      };
      if (SIGHT && cut.chunk_spread) {                             // (k_chunk_join is another launch: ordinary stores will do)
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int i = 0; i < 16; i += 2) *sums(piece, c, i) = make_float2(acc[c][i], acc[c][i + 1]);
        if (hh == 0) parts.ml[row0 + (size_t)piece * kChunkRows + n] = make_float2(m, l);
        return false;
      }
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
      if (!sm.last) return false;
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
    return true;
  });
}

// A launch: chunk_wgs workgroups for sequences of many rows (cut.blocks blocks of each kv-head, piece by piece), behind them those for
// few (unit by unit, piece by piece).  One launch for both: a prompt's chunk and the other requests' tokens share the chip.
// KIND: bit 0: there are the former, bit 1: the latter.
template <typename T, int D, int MODE, int KIND, int BITS, bool SIGHT>
__global__ __launch_bounds__(256, waves_of(D, MODE, KIND, BITS)) void k_paged_attn(PagedAttnArgs A, Cut cut, Parts parts, int chunk_wgs) {
  constexpr size_t kMost = sizeof(ChunkLds<D>) > sizeof(StepLds<D>) ? sizeof(ChunkLds<D>) : sizeof(StepLds<D>);
  __shared__ __align__(16) char lds[KIND == 1 ? sizeof(ChunkLds<D>) : KIND == 2 ? sizeof(StepLds<D>) : kMost];
  const int id = (int)blockIdx.x;
  if ((KIND & 1) && (KIND == 1 || id < chunk_wgs)) {
    if constexpr (KIND & 1) cut_chunk<T, D, MODE, BITS, SIGHT>(A, cut, parts, *reinterpret_cast<ChunkLds<D>*>(lds), id);
  } else {
    if constexpr (KIND & 2) cut_step<T, D, MODE, BITS, SIGHT>(A, cut, parts, *reinterpret_cast<StepLds<D>*>(lds), id - chunk_wgs);
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
template <typename T, int D, bool MANY, bool SIGHT>
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
  const int block = r / kChunkRows * kChunkRows;
  const int last = step ? s.nq - 1 : min(s.nq * A.G - 1, block + kChunkRows - 1) / A.G;
  const int piece = step ? cut.step_piece : cut.chunk_piece;
  int np = (Keys<SIGHT>(A.V, s, prefix, step ? 0 : block / A.G, last).end + piece - 1) / piece;
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

// Joins the pieces of cut_chunk's blocks, in order: blockIdx.y: block and kv-head, 16 (D = 128) or 8 workgroups each.  A lane has four channels of a
// row, as paged_chunk's had them.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_chunk_join(PagedAttnArgs A, Cut cut, Parts parts) {
  constexpr int CB = D / 32;
  const Paged& P = A.P;
  const int at = (int)blockIdx.x * 256 + (int)threadIdx.x, lane = at & 63, e = at >> 6 & 3, c = at / 256 % CB, wave = at / (256 * CB);
  const int4 split = parts.split[blockIdx.y];
  const int np = split.x, h = (int)blockIdx.y % P.H, r = split.w * kChunkRows + 32 * wave + (lane & 31);
  if (np <= 1 || r >= split.z * A.G) return;
  const size_t row0 = parts.chunk0 + (size_t)blockIdx.y * cut.n_chunk * kChunkRows + 32 * wave;
  float m = kUnset, l = 0.f;
#pragma unroll 8
  for (int p = 0; p < np; ++p) m = fmaxf(m, parts.ml[row0 + (size_t)p * kChunkRows + (lane & 31)].x);
  f32x4g o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = 0; p < np; ++p) {
    const float2* from = reinterpret_cast<const float2*>(parts.acc + (row0 + (size_t)p * kChunkRows) * D) + (8 * c + 2 * e) * 64 + lane;
    const float2 z = parts.ml[row0 + (size_t)p * kChunkRows + (lane & 31)], x = from[0], y = from[64];
    const float f = exp2_hw(z.x - m);
    l += f * z.y;
    o += f * f32x4g{x.x, x.y, y.x, y.y};
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;                      // (NaN stays)
  const size_t orow = (size_t)(split.y + r / A.G) * A.Hq + h * A.G + r % A.G;
  store4((T*)A.out + orow * D + 32 * c + 8 * e + 4 * (lane >> 5), o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  if (c == 0 && e == 0 && lane < 32 && A.lse) A.lse[orow] = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
}

// Workgroups of a call's launches.  merge: few_rows rows of every unit, if paged_step's pieces are not joined where they are made; then
// all rows, if those of paged_chunk are not (they are cut only where they are few).  Rows of few pieces are little work, and eight fit a workgroup.
struct Launches { long long chunk, step, merge; int few_rows, step_ids; bool many; };
inline Launches launches_of(const Paged& P, int Hq, const Cut& c) {
  Launches l = {};
  l.chunk = c.w.chunk ? (long long)c.blocks * P.H * c.n_chunk : 0;
  l.step = c.w.step ? (long long)(c.groups ? c.groups : P.B) * P.H * c.n_step : 0;
  const bool join_step = l.step && c.n_step > 1 && !c.joined, join_chunk = l.chunk && c.n_chunk > 1 && !c.chunk_joined && !c.chunk_spread;
  l.few_rows = (int)std::min<long long>(kStepRows, (long long)P.max_q * (Hq / P.H));
  l.step_ids = join_step ? (P.B * P.H * l.few_rows + 7) / 8 * 8 : 0;
  l.many = (join_chunk ? c.n_chunk : c.n_step) >= 8;
  const long long ids = l.step_ids + (join_chunk ? (long long)P.N * Hq : 0);
  l.merge = l.many ? ids : (ids + 7) / 8;
  return l;
}
template <typename T, int D, int MODE, int BITS, bool SIGHT>
hipError_t launch_attention(const PagedAttnArgs& A, hipStream_t st) {
  const Paged& P = A.P;
  const Cut c = cut_of(P, A.V, D, A.Hq);
  const Launches l = launches_of(P, A.Hq, c);
  Parts parts = {};
  const size_t n = part_rows(P, A.Hq, c, parts.chunk0);
  parts.tickets = (int*)A.ws;
  parts.acc = A.ws + kTicketFloats;
  parts.ml = (float2*)(parts.acc + n * D);
  parts.split = (int4*)(parts.ml + (n + 1) / 2 * 2);
  const int chunk = (int)l.chunk, step = (int)l.step;
  if (chunk && step) k_paged_attn<T, D, MODE, 3, BITS, SIGHT><<<chunk + step, 256, 0, st>>>(A, c, parts, chunk);
  else if (chunk) k_paged_attn<T, D, MODE, 1, BITS, SIGHT><<<chunk, 256, 0, st>>>(A, c, parts, chunk);
  else k_paged_attn<T, D, MODE, 2, BITS, SIGHT><<<step, 256, 0, st>>>(A, c, parts, 0);
  if constexpr (SIGHT)
    if (chunk && c.chunk_spread) k_chunk_join<T, D><<<dim3(D / 8, (unsigned)(c.blocks * P.H)), 256, 0, st>>>(A, c, parts);
  if (l.merge) {
    if (l.many) k_paged_merge<T, D, true, SIGHT><<<(int)l.merge, 256, 0, st>>>(A, c, parts, l.few_rows, l.step_ids);
    else k_paged_merge<T, D, false, SIGHT><<<(int)l.merge, 256, 0, st>>>(A, c, parts, l.few_rows, l.step_ids);
  }
  return hipGetLastError();
}

}  // namespace arkv
