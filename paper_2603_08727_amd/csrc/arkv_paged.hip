// Rows of a paged cache: rotary positions on the way in (k_paged_append), and eviction by collected weight
// (k_evict_select, k_evict_move).
#include <algorithm>
#include <type_traits>

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
// round trips to memory: its lengths, angles and rows are requested together, the page behind them, then it stores (16 tokens: 5.1 us);
// many by memory itself (7817 tokens of 32 + 2 x 8 heads: 43 us, 4.5 TB/s).
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
  // time (16 tokens of 32 + 2 x 8 heads: 7.0 us as one wave each, 5.1 as two).
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

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;
constexpr int kEvictBins = 2048;        // eleven bits of a key
constexpr int kEvictRows = 4 * kEvictThreads;   // slots that a workgroup looks at at a time: four adjacent ones per lane
constexpr int kEvictRegs = 9;           // times that many slots whose keys a lane keeps in registers
constexpr int kEvictSlots = 256;        // slots per workgroup of k_evict_move: those of one wave, kEvictRows at a time
// Survivors times channels up to which the choosing workgroup copies them, which saves a launch and the workspace (8 x 2 heads,
// 250 of 1000 rows of 64 channels: 9.0 us against 9.9; 512: 10.8 and 11.1; 8 x 8 heads, 250 of 2000 rows of 128: 12.5 and 13.4).
constexpr int kSelectMoves = 32768;

// Order of weights as an order of words: NaN (and a row that is not there) lowest, -0 with +0; 0 is no weight's.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (!(w == w)) return 1;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// What a unit keeps: m of its n rows, the first `lo` and those from `hi` on among them, and `ranked` of the others.
struct Kept {
  int n, m, lo, hi, ranked;
  __device__ __forceinline__ bool all() const { return ranked >= hi - lo; }
  __device__ __forceinline__ bool by_weight() const { return !all() && ranked > 0; }
};
__device__ __forceinline__ Kept kept_of(const EvictArgs& A, int b) {
  Kept k;
  k.n = min(max(A.P.kv_len[b], 0), A.P.max_kv);
  k.m = min(k.n, min(max(A.keep[b], 0), A.max_keep));
  k.lo = min(A.sink, k.m);
  const int back = min(A.recent, k.m - k.lo);
  k.hi = k.n - back;
  k.ranked = k.m - k.lo - back;
  return k;
}

// How a launch is cut: workgroups per unit that count, slots of each; where the workspace holds what they pass on: [unit][chunk]
// histograms, per unit the key of the last survivor and how many rows of that key stay, per unit and kEvictSlots slots the
// rows in front that stay for certain and those of the last survivor's key.
struct EvictCut { int chunks, per, blocks; };
struct EvictParts { int* tickets; unsigned long long* hist; uint2* last; int2* before; };

static EvictCut evict_cut(const Paged& P) {
  // Where there are fewer units than half the CUs, several workgroups count the first digit (32 units of 32768 rows:
  // 3 us with reading the weights; by one workgroup each 12).
  const long long units = (long long)P.B * P.H;
  const int steps = std::max(1, (P.max_kv + kEvictRows - 1) / kEvictRows);
  EvictCut c;
  c.chunks = (int)std::max(1ll, std::min<long long>(steps, 256 / units));
  c.per = (steps + c.chunks - 1) / c.chunks * kEvictRows;
  c.chunks = std::max(1, (P.max_kv + c.per - 1) / c.per);
  c.blocks = steps * (kEvictRows / kEvictSlots);
  return c;
}
static_assert(kJoinUnits >= 128, "a ticket for every unit that is cut");

size_t paged_evict_floats(const Paged& P) {
  const EvictCut c = evict_cut(P);
  const size_t units = (size_t)P.B * P.H;
  return kTicketFloats + units * (c.chunks > 1 ? (size_t)c.chunks * kEvictBins : 0) + 2 * units + 2 * units * c.blocks;
}
// For every batch of no more sequences and rows than P's: fewer units are counted by more workgroups each, 256 in all at most.
size_t paged_evict_bound(const Paged& P) {
  const size_t units = (size_t)P.B * P.H, steps = std::max(1, (P.max_kv + kEvictRows - 1) / kEvictRows);
  return kTicketFloats + (steps > 1 ? std::min<size_t>(256, std::min<size_t>(128, units) * steps) * kEvictBins : 0) + 2 * units +
         2 * units * evict_cut(P).blocks;
}
bool paged_evict_needs_workspace(const Paged& P, int D, int max_keep) {
  return (int64_t)max_keep * D > kSelectMoves || P.max_kv > kEvictRegs * kEvictRows;
}

// Adds one to hist[bin] for each of a lane's four bins with `on` set.  The lanes that share the bin of the first one (equal
// weights, such as those of rows that nobody looked at) add once for all: additions to one word queue.
__device__ __forceinline__ void count_bins(int* hist, const bool (&on)[4], const int (&bin)[4], int lane) {
  const uint64_t live = __ballot(on[0] || on[1] || on[2] || on[3]);
  if (!live) return;
  if (__popcll(live) <= 8) {                                       // (few: the queue is short)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (on[e]) atomicAdd(&hist[bin[e]], 1);
    return;
  }
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

// Copies survivors i = first, first + step, .. < n, which are at slots list[i], to slots to0 + i: D / 8 lanes a row, N rows
// per lane whose loads are all under way together (k_evict_move: 4; of the few rows that k_evict_select copies 2: 8 x 2 heads x 250 rows
// 9.0 us, with 4 9.7).  The stores pass the caches by: with ordinary ones, 32 units x 8192 rows took 90 instead of 86 us.
constexpr int kMoveRows = 4, kSelectRows = 2;
template <int D, int N>
__device__ __forceinline__ void move_rows(const EvictArgs& A, const Kept& K, int h, int b, const int* list, int n, int to0, int first, int step) {
  constexpr int LPR = D / 8;
  const int c = threadIdx.x % LPR;
  const Paged& P = A.P;
  int from[N], to[N];
#pragma unroll
  for (int r = 0; r < N; ++r) {
    const int i = first + r * step;
    from[r] = i < n ? slot_row(P.table + (size_t)b * P.width, P.n_pages, P.H, h, P.lg_page, K.n, list[i]) : -1;
    to[r] = i < n ? slot_row(A.dst_table + (size_t)b * A.dst_width, P.n_pages, P.H, h, P.lg_page, K.m, to0 + i) : -1;
  }
  // (lanes 0 and 1 of a row take its position and weight)
  uint32_t* meta = c == 0 ? (uint32_t*)P.pos : (uint32_t*)P.weight;
  u32x4p x[N], y[N];
  uint32_t z[N];
#pragma unroll
  for (int r = 0; r < N; ++r) {
    z[r] = c < 2 ? meta[max(from[r], 0)] : 0;
    x[r] = ((const u32x4p*)P.k)[(size_t)max(from[r], 0) * LPR + c];
    y[r] = ((const u32x4p*)P.v)[(size_t)max(from[r], 0) * LPR + c];
  }
#pragma unroll
  for (int r = 0; r < N; ++r) {
    if (from[r] < 0 || to[r] < 0) continue;
    __builtin_nontemporal_store(x[r], (u32x4p*)P.k + (size_t)to[r] * LPR + c);
    __builtin_nontemporal_store(y[r], (u32x4p*)P.v + (size_t)to[r] * LPR + c);
    if (c < 2) meta[to[r]] = z[r];
  }
}

// Which rows of a (sequence, kv-head) stay.  The key of the last one is found digit by digit, from the top: how many rows have
// which digit, and the digit at which the rows to keep run out; a digit whose rows all stay ends the search.  The first digit,
// which every row takes part in, is counted by cut.chunks workgroups; the last one to finish goes on alone with the keys in its
// lanes' registers (REGS times 4096 of them; 0: there are more rows than fit, which are read in every pass).  MOVE > 0: it then lists the survivors
// and copies their MOVE channels itself; else it leaves to k_evict_move the last survivor's key and the counts in front of every 256 slots.
template <int REGS, int MOVE>
__global__ __launch_bounds__(kEvictThreads) void k_evict_select(EvictArgs A, EvictCut cut, EvictParts parts) {
  constexpr int NW = kEvictWaves, BPT = kEvictBins / kEvictThreads;
  __shared__ __align__(8) int hist[kEvictBins];
  __shared__ int sums[NW];
  __shared__ int s_bin, s_left, s_count, s_last;
  constexpr int GROUP = REGS ? REGS : kEvictRegs;                  // steps whose counts are added up together
  __shared__ int2 counts[GROUP * NW];                        // of every wave's slots: rows that stay for certain, equal ones
  __shared__ int list[MOVE ? kSelectMoves / (MOVE ? MOVE : 1) : 1];
  const int chunk = blockIdx.x, h = blockIdx.y, b = blockIdx.z, unit = b * A.P.H + h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Kept K = kept_of(A, b);
  const bool ranks = K.by_weight();
  // a unit that does not rank, or is short, is the first workgroup's alone
  const int chunks = ranks ? (K.n + cut.per - 1) / cut.per : 1;
  if (chunk >= chunks) return;
  const int32_t* table = A.P.table + (size_t)b * A.P.width;
  int32_t* kept = A.kept + (size_t)unit * A.max_keep;
  // keys of slots j .. j + 3, which lie in one page; 0 where a slot is not ranked
  auto first_row = [&](int j) { return slot_row(table, A.P.n_pages, A.P.H, h, A.P.lg_page, K.n, j); };
  auto keys_at = [&](int j, int row) {
    u32x4p x = {1, 1, 1, 1};
    if (ranks && row >= 0) {
      const float4 w = *reinterpret_cast<const float4*>(A.P.weight + row);
      x = u32x4p{weight_key(w.x), weight_key(w.y), weight_key(w.z), weight_key(w.w)};
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < K.lo || j + e >= K.hi) x[e] = 0;
    return x;
  };
  // counts the digit at `shift` of the keys from max(prefix, 1) up to prefix + width - 1
  auto count = [&](const u32x4p& x, int shift, uint32_t prefix, uint32_t width) {
    const uint32_t low = max(prefix, 1u), some = width - (low - prefix);
    bool on[4];
    int bin[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      on[e] = x[e] - low < some;
      bin[e] = (int)((x[e] - prefix) >> shift);
    }
    count_bins(hist, on, bin, lane);
  };
  const int steps = (K.n + kEvictRows - 1) / kEvictRows;           // of 4096 slots each
  u32x4p keys[GROUP];
  // all steps' pages, then all their weights: two round trips to memory
  int row[GROUP];
#pragma unroll
  for (int q = 0; q < REGS; ++q) row[q] = q < steps ? first_row(kEvictRows * q + 4 * tid) : -1;
  auto load_all = [&]() {
#pragma unroll
    for (int q = 0; q < REGS; ++q) keys[q] = q < steps ? keys_at(kEvictRows * q + 4 * tid, row[q]) : u32x4p{0, 0, 0, 0};
  };
  // f(keys, q) for all steps
  auto each = [&](auto f) {
    if constexpr (REGS > 0) {
#pragma unroll
      for (int q = 0; q < REGS; ++q)
        if (q < steps) f(keys[q], q);
    } else {
      for (int q = 0; q < steps; ++q) f(keys_at(kEvictRows * q + 4 * tid, first_row(kEvictRows * q + 4 * tid)), q);
    }
  };
  for (int i = tid; i < kEvictBins; i += kEvictThreads) hist[i] = 0;
  if (REGS && chunks == 1) load_all();
  __syncthreads();
  // survivors: keys above `last`, and of those equal to it the first `need`
  uint32_t last = K.all() ? 0u : ~0u;
  int need = 0;
  if (ranks) {
    if (chunks == 1) {
      each([&](const u32x4p& x, int) { count(x, 21, 0, ~0u); });   // (no weight's key is ~0)
    } else {
      for (int j = cut.per * chunk + 4 * tid; j < min(cut.per * (chunk + 1), K.n); j += kEvictRows) count(keys_at(j, first_row(j)), 21, 0, ~0u);
      __syncthreads();
      // (past the L2 of one XCD; the stores are acknowledged before the ticket is drawn)
      unsigned long long* mine = parts.hist + ((size_t)unit * cut.chunks + chunk) * (kEvictBins / 2);
      __hip_atomic_store(mine + tid, reinterpret_cast<const unsigned long long*>(hist)[tid], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      int* ticket = parts.tickets + unit * kTicketWords;
      if (tid == 0) {
        s_last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == chunks - 1;
        if (s_last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // as the next call wants it
      }
      __syncthreads();
      if (!s_last) return;
      if (REGS) load_all();
      int c0 = 0, c1 = 0;
#pragma unroll 8
      for (int c = 0; c < chunks; ++c) {
        const unsigned long long u = __hip_atomic_load(parts.hist + ((size_t)unit * cut.chunks + c) * (kEvictBins / 2) + tid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        c0 += (int)(uint32_t)u;
        c1 += (int)(u >> 32);
      }
      hist[2 * tid] = c0;
      hist[2 * tid + 1] = c1;
    }
    need = K.ranked;
    uint32_t prefix = 0;
    for (int shift = 21; ; shift = shift == 21 ? 10 : 0) {
      if (shift != 21) each([&](const u32x4p& x, int) { count(x, shift, prefix, shift ? 1u << 21 : 1u << 10); });
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
#pragma unroll
      for (int w = 0; w < NW; ++w) before += w < wave ? sums[w] : 0;
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
      if (s_count == need) {                                       // the whole digit stays: everything from its lowest key on
        last = prefix ? prefix - 1 : 0;
        need = 0;
        break;
      }
      last = prefix;
      if (!shift) break;
    }
  }
  if (h == 0 && tid == 0) A.new_len[b] = K.m;
  for (int i = K.m + tid; i < A.max_keep; i += kEvictThreads) kept[i] = -1;
  int carry_sure = 0, carry_ties = 0;                              // in front of the group of steps at hand
  for (int q0 = 0; q0 < max(1, REGS ? 1 : steps); q0 += GROUP) {
    auto tally = [&](const u32x4p& x, int q) {
      const int j = kEvictRows * q + 256 * wave;                   // the wave's slots; of those that are not ranked, which stay
      int sure = max(0, min(K.lo, j + 256) - j) + max(0, min(K.n, j + 256) - max(K.hi, j)), ties = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sure += __popcll(__ballot(x[e] > last));
        if (need > 0) ties += __popcll(__ballot(x[e] == last));
      }
      if (lane == 0) counts[(q - q0) * NW + wave] = make_int2(sure, ties);
    };
    if constexpr (REGS > 0) each(tally);
    else for (int q = q0; q < min(steps, q0 + GROUP); ++q) tally(keys_at(kEvictRows * q + 4 * tid, first_row(kEvictRows * q + 4 * tid)), q);
    __syncthreads();
    // counts become what is in front; a lane adds up three of them
    const int n = min(GROUP, steps - q0) * NW;
    if (wave == 0) {
      constexpr int PL = (GROUP * NW + 63) / 64;
      int2 c[PL];
      int sure = 0, ties = 0;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        c[i] = PL * lane + i < n ? counts[PL * lane + i] : make_int2(0, 0);
        sure += c[i].x;
        ties += c[i].y;
      }
      int us = sure, ut = ties;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int vs = __shfl_up(us, o), vt = __shfl_up(ut, o);
        if (lane >= o) { us += vs; ut += vt; }
      }
      sure = carry_sure + us - sure;
      ties = carry_ties + ut - ties;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        if (PL * lane + i < n) {
          if (MOVE) counts[PL * lane + i] = make_int2(sure, ties);
          else parts.before[(size_t)unit * cut.blocks + q0 * NW + PL * lane + i] = make_int2(sure, ties);
        }
        sure += c[i].x;
        ties += c[i].y;
      }
      carry_sure = __builtin_amdgcn_readlane(sure, 63);
      carry_ties = __builtin_amdgcn_readlane(ties, 63);
    }
    if (MOVE || !REGS) __syncthreads();
  }
  if (MOVE == 0 && tid == 0) parts.last[unit] = make_uint2(last, (uint32_t)need);
  if constexpr (MOVE > 0) {
    static_assert(REGS > 0, "");
    const uint64_t below = (1ull << lane) - 1;
    // bit e: slot e of the lane's four stays for certain, bit 4 + e: it is one of the equal ones
    auto fate = [&](const u32x4p& x, int q) {
      const int j = kEvictRows * q + 4 * tid;
      uint32_t f = 0;
  #pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (x[e] ? x[e] > last : j + e < K.n) f |= 1u << e;
        if (need > 0 && x[e] == last) f |= 16u << e;
      }
      return f;
    };
    each([&](const u32x4p& x, int q) {
      const uint32_t f = fate(x, q);
      const int2 front = counts[q * NW + wave];
      int rank = front.y;                                          // of a lane's equal slots
#pragma unroll
      for (int e = 0; e < 4; ++e) rank += __popcll(__ballot(f >> (4 + e) & 1) & below);
      uint32_t take = f & 15;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (f >> (4 + e) & 1) {
          if (rank < need) take |= 1u << e;
          ++rank;
        }
      int to = front.x + min(front.y, need);
#pragma unroll
      for (int e = 0; e < 4; ++e) to += __popcll(__ballot(take >> e & 1) & below);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (take >> e & 1) {
          if (to < K.m) list[to] = kEvictRows * q + 4 * tid + e;
          ++to;
        }
    });
    __syncthreads();
    constexpr int RPW = kEvictThreads / (MOVE / 8);
    for (int i = tid; i < K.m; i += kEvictThreads) kept[i] = list[i];
    for (int i = 0; i < K.m; i += RPW * kSelectRows) move_rows<MOVE, kSelectRows>(A, K, h, b, list, K.m, 0, i + tid / (MOVE / 8), RPW);
  }
}

// Lists the survivors among 256 slots, a slot per lane, and copies them: the units' slots are spread over the whole chip (8192 of 32768
// rows of 32 units, 272 MB: 63 us, 4.3 TB/s).
template <int D>
__global__ __launch_bounds__(kEvictSlots) void k_evict_move(EvictArgs A, EvictCut cut, EvictParts parts) {
  constexpr int NW = kEvictSlots / 64, RPW = kEvictSlots / (D / 8);
  __shared__ int list[kEvictSlots];
  __shared__ int2 counts[NW];
  const int blk = blockIdx.x, h = blockIdx.y, b = blockIdx.z, unit = b * A.P.H + h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Kept K = kept_of(A, b);
  const int j = kEvictSlots * blk + tid;
  if (kEvictSlots * blk >= K.n) return;
  const int2 front = parts.before[(size_t)unit * cut.blocks + blk];
  const uint2 pivot = parts.last[unit];
  const int need = (int)pivot.y;
  uint32_t x = 0;
  if (j >= K.lo && j < K.hi) {
    const int row = slot_row(A.P.table + (size_t)b * A.P.width, A.P.n_pages, A.P.H, h, A.P.lg_page, K.n, j);
    x = K.by_weight() && row >= 0 ? weight_key(A.P.weight[row]) : 1;
  }
  const bool sure = x ? x > pivot.x : j < K.n, tie = need > 0 && x == pivot.x;
  const uint64_t sb = __ballot(sure), tb = __ballot(tie), below = (1ull << lane) - 1;
  if (lane == 0) counts[wave] = make_int2(__popcll(sb), __popcll(tb));
  __syncthreads();
  int certain = 0, ties = front.y, n_sure = 0, n_ties = front.y;   // in front of this lane; in the whole block
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const int2 c = counts[w];
    if (w < wave) { certain += c.x; ties += c.y; }
    n_sure += c.x;
    n_ties += c.y;
  }
  certain += __popcll(sb & below);
  ties += __popcll(tb & below);
  const int taken = min(front.y, need), to0 = front.x + taken;     // equal rows of earlier blocks that stay; this block's first new slot
  if (sure || (tie && ties < need)) list[certain + min(ties, need) - taken] = j;
  __syncthreads();
  const int n = min(n_sure + min(n_ties, need) - taken, K.m - to0);
  int32_t* kept = A.kept + (size_t)unit * A.max_keep + to0;
  for (int i = tid; i < n; i += kEvictSlots) kept[i] = list[i];
  for (int i = 0; i < n; i += RPW * kMoveRows) move_rows<D, kMoveRows>(A, K, h, b, list, n, to0, i + tid / (D / 8), RPW);
}

template <int D>
static hipError_t launch_evict(const EvictArgs& A, hipStream_t st) {
  const Paged& P = A.P;
  const EvictCut c = evict_cut(P);
  const bool moves = !paged_evict_needs_workspace(P, D, A.max_keep);
  const size_t units = (size_t)P.B * P.H;
  EvictParts parts = {};
  EvictCut cut = c;
  if (A.ws) {
    parts.tickets = (int*)A.ws;
    parts.hist = (unsigned long long*)(A.ws + kTicketFloats);
    parts.last = (uint2*)(A.ws + kTicketFloats + (c.chunks > 1 ? units * c.chunks * kEvictBins : 0));
    parts.before = (int2*)(parts.last + units);
  }
  else { cut.chunks = 1; cut.per = kEvictRegs * kEvictRows; }      // (one workgroup a unit needs none)
  const dim3 grid(cut.chunks, P.H, P.B);
  auto select = [&](auto regs) {
    constexpr int N = decltype(regs)::value;
    if constexpr (N > 0) {
      if (moves) { k_evict_select<N, D><<<grid, kEvictThreads, 0, st>>>(A, cut, parts); return; }
    }
    k_evict_select<N, 0><<<grid, kEvictThreads, 0, st>>>(A, cut, parts);
  };
  // (8 x 2 units of 1000 rows: 9.2 us; with the code of nine steps, which has to come from memory, 11.9)
  if (P.max_kv <= kEvictRows) select(std::integral_constant<int, 1>());
  else if (P.max_kv <= kEvictRegs * kEvictRows) select(std::integral_constant<int, kEvictRegs>());
  else select(std::integral_constant<int, 0>());
  if (!moves && P.max_kv) k_evict_move<D><<<dim3((P.max_kv + kEvictSlots - 1) / kEvictSlots, P.H, P.B), kEvictSlots, 0, st>>>(A, c, parts);
  return hipGetLastError();
}

hipError_t launch_paged_evict(int D, const EvictArgs& A, hipStream_t st) { return D == 64 ? launch_evict<64>(A, st) : launch_evict<128>(A, st); }

}  // namespace arkv
