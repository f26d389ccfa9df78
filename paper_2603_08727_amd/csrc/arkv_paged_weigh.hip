// The attention weight that a paged cache's rows collect from new tokens: weight[j] = decay carried[j] + sum over the tokens
// that see slot j and the G heads of its group of exp(x - lse).
#include <algorithm>

#include "arkv_paged_mma.h"

namespace arkv {

// ---- weights ------------------------------------------------------------------------------------------

// Here query rows are on the M side (S = Q K^T), which leaves one key per lane: a lane adds up its rows' probabilities, and
// the lanes that share a key add theirs in a fixed order at the end.  As above, few rows and many have a kernel each.
constexpr int kWeighStepKeys = 1024;    // keys per wave of k_weigh_step, at most: a lane holds the page of one granule
constexpr int kWeighKeys = 256, kWeighRows = 64;   // keys per workgroup and rows per tile of k_weigh_chunk

__device__ __forceinline__ void store_weight(const PagedAttnArgs& A, int row, float sum) {
  A.P.weight[row] = (A.decay == 0.f ? 0.f : A.decay * A.carried[row]) + sum;
}

// Few rows: bound by reading the keys (16 requests of 5960 to 8192 rows x 8 heads, 233 MB: 50 us, 4.7 TB/s).  A wave takes wave_keys keys, 32 at a time (two granules), the next 32 in flight.
template <typename T, int D, int MODE>
__global__ __launch_bounds__(256) void k_weigh_step(PagedAttnArgs A, int wave_keys) {
  constexpr int CAP = Mode<MODE>::cap;
  constexpr bool DIST = Mode<MODE>::dist;
  constexpr int KK = D / 32;
  const Paged& P = A.P;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, gq = lane >> 4;
  const int h = blockIdx.y, b = blockIdx.z;
  const int w0 = (blockIdx.x * 4 + wave) * wave_keys;
  const Seq s = seq_of(P, b);
  const int R = s.nq * A.G;
  if (w0 >= s.kv || R > kStepRows) return;
  const int prefix = A.S.prefix ? A.S.prefix[b] : 0;
  // lane i holds the page of granule i; one that is not there becomes page 0, whose rows get nothing
  const int w1 = min(w0 + wave_keys, s.kv);
  int my_page = w0 + 16 * lane < w1 ? P.table[(size_t)b * P.width + ((w0 + 16 * lane) >> P.lg_page)] : -1;
  const bool page_ok = (unsigned)my_page < (unsigned)P.n_pages;
  if (!page_ok) my_page = 0;
  const uint64_t ok_mask = __ballot(page_ok);
  const int in_page = (1 << P.lg_page) - 1;
  auto granule_row = [&](int g) {
    const int page = __builtin_amdgcn_readlane(my_page, g);
    return ((page * P.H + h) << P.lg_page) + ((w0 + 16 * g) & in_page);
  };
  u32x4g q[KK];
  float lse[4], slope[4];
  int qp[4], end[4];
  {
    const int row = n < R ? n : 0;                                 // (rows from R on see nothing)
    const T* p = (const T*)A.q.p + (size_t)(s.q0 + row / A.G) * A.q.ts + (size_t)(h * A.G + row % A.G) * A.q.hs + 8 * gq;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = R ? *reinterpret_cast<const u32x4g*>(p + 32 * kk) : u32x4g{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * gq + i, rc = row < R ? row : 0;
    const int tok = s.q0 + rc / A.G, hq = h * A.G + rc % A.G;
    end[i] = row < R ? row_end(s, rc / A.G, prefix) : 0;
    lse[i] = R ? A.lse[(size_t)tok * A.Hq + hq] * kLog2e : 0.f;
    slope[i] = DIST && R ? A.S.slopes[hq] * kLog2e : 0.f;
    qp[i] = DIST && R ? A.S.q_pos[tok] : 0;
  }
  const Logit lg(A.S);
  // (the carried weights come with the keys: requested at the store they cost a round trip to memory every 16 keys)
  u32x4g kb[2][2][KK];
  float wb[2][2] = {};
  const bool carry = A.decay != 0.f;
  auto load_k = [&](int t, u32x4g (&to)[2][KK], float (&w)[2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int row = granule_row(2 * t + g) + n;
      if (carry) w[g] = A.carried[row];
      const T* p = (const T*)P.k + (size_t)(unsigned)row * D + 8 * gq;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) to[g][kk] = *reinterpret_cast<const u32x4g*>(p + 32 * kk);
    }
  };
  auto tile = [&](int t, const u32x4g (&kc)[2][KK], const float (&w)[2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      f32x4g x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) x = Mfma<T>::m16(q[kk], kc[g][kk], x);
      const int j = w0 + 32 * t + 16 * g + n, row = granule_row(2 * t + g) + n;
      const bool there = j < s.kv && (ok_mask >> (2 * t + g) & 1);
      const int kp = DIST ? P.pos[row] : 0;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y = lg.logit<CAP>(x[i]);
        if (DIST) y = fmaf(-slope[i], fabsf((float)(qp[i] - kp)), y);
        sum += j < end[i] ? exp2_hw(y - lse[i]) : 0.f;
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (there && gq == 0) P.weight[row] = (carry ? A.decay * w[g] : 0.f) + sum;
    }
  };
  const int nt = (w1 - w0 + 31) / 32;
  load_k(0, kb[0], wb[0]);
  for (int t = 0; t < nt; t += 2) {
    if (t + 1 < nt) load_k(t + 1, kb[1], wb[1]);
    tile(t, kb[0], wb[0]);
    if (t + 1 < nt) {
      if (t + 2 < nt) load_k(t + 2, kb[0], wb[0]);
      tile(t + 1, kb[1], wb[1]);
    }
  }
}

// Many rows: bound by the matrix cores and the exponentials.  One workgroup = 256 keys of a (sequence, kv-head), 64 per wave,
// held in registers as B operands, and a share of the rows that see them; rows come through LDS, 64 at a time, the next 64
// on their way.  The logits' MFMAs of the next 32 rows stand between the exponentials of these (2 x 1024 tokens over 8191 rows, 32 heads:
// 146 us, 0.9 PFLOP/s; with the two one behind the other, as with a cap or a bias, 169).
constexpr int kWeighBufs = 3;           // rows in use, the next ones (their first half is ahead), the ones on their way
template <int D> struct WeighLds {
  uint16_t q[kWeighBufs][kWeighRows * D];
  float lse[kWeighBufs][kWeighRows], slope[kWeighBufs][kWeighRows];
  int qp[kWeighBufs][kWeighRows];
};

template <typename T, int D, int MODE>
__global__ __launch_bounds__(256, 2) void k_weigh_chunk(PagedAttnArgs A, int few, int n_shares) {
  constexpr int CAP = Mode<MODE>::cap;
  constexpr bool DIST = Mode<MODE>::dist;
  constexpr int KK = D / 16, CPR = D / 8, RPI = 64 / CPR, LPW = kWeighRows / RPI / 4;    // LPW: 1 KB loads of a tile per wave
  __shared__ __align__(16) WeighLds<D> sm;
  const Paged& P = A.P;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int share = blockIdx.x % n_shares, blk = blockIdx.x / n_shares, h = blockIdx.y, b = blockIdx.z;
  const Seq s = seq_of(P, b);
  const int R = s.nq * A.G, j00 = blk * kWeighKeys;
  if (R <= few || j00 >= s.kv) return;
  const int prefix = A.S.prefix ? A.S.prefix[b] : 0, ctx = s.kv - s.nq;
  const int w0 = j00 + 64 * wave;                                  // this wave's keys
  const int32_t* table = P.table + (size_t)b * P.width;
  // rows that see key j start here
  auto first_row = [&](int j) { return j < prefix ? 0 : max(0, j - ctx) * A.G; };
  const int start = first_row(j00) / kWeighRows, tiles = (R + kWeighRows - 1) / kWeighRows;
  const int per = (max(0, tiles - start) + n_shares - 1) / n_shares;
  const int t0 = min(start + share * per, tiles), t1 = min(t0 + per, tiles);
  const int wave_lo = first_row(min(w0 + 63, s.kv - 1));           // rows from here on see all keys of the wave (prefixes grow with no key)
  u32x4g k[2][KK];
  int krow[2], lo[2], kp[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int j = w0 + 32 * g + n;
    krow[g] = slot_row(table, P.n_pages, P.H, h, P.lg_page, s.kv, j);
    lo[g] = krow[g] < 0 ? 0x7FFFFFFF : first_row(j);
    const T* p = (const T*)P.k + (size_t)max(krow[g], 0) * D + 8 * hh;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) k[g][kk] = *reinterpret_cast<const u32x4g*>(p + 16 * kk);
    kp[g] = DIST ? P.pos[max(krow[g], 0)] : 0;
  }
  const bool all_there = !__any(krow[0] < 0 || krow[1] < 0);
  const uint32_t lds_q = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)sm.q;
  const uint32_t lds_lse = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)sm.lse;
  const uint32_t lds_slope = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)sm.slope;
  const uint32_t lds_qp = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)sm.qp;
  // Where this lane's loads of the next tile lie: addresses move on by a tile's rows, `more` tokens and `rest` heads, without a
  // division; in a tile that ends behind the last row they are formed anew, and stop there.
  const int more = kWeighRows / A.G, rest = kWeighRows % A.G;
  const int lr0 = 16 * wave + lane / CPR;
  const T* qa[LPW];
  int head[LPW], one_head, one_tok;
  auto locate = [&](int t) {
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
      const int r = min(kWeighRows * t + lr0 + RPI * i, R - 1);
      head[i] = r % A.G;
      qa[i] = (const T*)A.q.p + (size_t)(s.q0 + r / A.G) * A.q.ts + (size_t)(h * A.G + head[i]) * A.q.hs + 8 * k_chunk<D>(lr0 + RPI * i, lane % CPR);
    }
    const int r = min(kWeighRows * t + lane, R - 1);
    one_head = r % A.G;
    one_tok = s.q0 + r / A.G;
  };
  const int64_t inc = (int64_t)more * A.q.ts + (int64_t)rest * A.q.hs, wrap = A.q.ts - (int64_t)A.G * A.q.hs;
  auto fetch = [&](int t, int buf) {
    if (t == t0 || kWeighRows * (t + 1) > R) locate(t);
#pragma unroll
    for (int i = 0; i < LPW; ++i) load_lds16(qa[i], lds_q + 2 * (buf * kWeighRows * D + (16 * wave + RPI * i) * D));
    if (wave == 0) load_lds4(A.lse + (size_t)one_tok * A.Hq + h * A.G + one_head, lds_lse + 4 * buf * kWeighRows);
    if (DIST) {
      if (wave == 1) load_lds4(A.S.slopes + h * A.G + one_head, lds_slope + 4 * buf * kWeighRows);
      if (wave == 2) load_lds4(A.S.q_pos + one_tok, lds_qp + 4 * buf * kWeighRows);
    }
#pragma unroll
    for (int i = 0; i < LPW; ++i) qa[i] += inc;
    one_tok += more;
    if (rest) {                                                    // (uniform; a group size that does not divide a tile)
#pragma unroll
      for (int i = 0; i < LPW; ++i) {
        head[i] += rest;
        if (head[i] >= A.G) { head[i] -= A.G; qa[i] += wrap; }
      }
      one_head += rest;
      if (one_head >= A.G) { one_head -= A.G; ++one_tok; }
    }
  };
  // (lse and slopes of a tile that has arrived, times log2(e), by one wave for all)
  auto to_log2 = [&](int buf) {
    if (wave == 0) sm.lse[buf][lane] *= kLog2e;
    if (DIST && wave == 1) sm.slope[buf][lane] *= kLog2e;
  };
  const Logit lg(A.S);
  float sum[2] = {0.f, 0.f};
  auto q_operand = [&](int buf, int rb, int kk) {
    return *reinterpret_cast<const u32x4g*>(&sm.q[buf][(32 * rb + n) * D + 8 * k_chunk<D>(n, 2 * kk + hh)]);
  };
  auto clear = [](f32x16g (&x)[2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[g][i] = 0.f;
  };
  // probabilities of 32 rows from their dot products x, where some row may not see some key
  auto add = [&](const f32x16g (&x)[2], int t, int buf, int rb) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int lr = 32 * rb + 8 * e + 4 * hh;
      const f32x4g z = *reinterpret_cast<const f32x4g*>(&sm.lse[buf][lr]);
      f32x4g sl = {0.f, 0.f, 0.f, 0.f};
      int4 qp = make_int4(0, 0, 0, 0);
      if (DIST) {
        sl = *reinterpret_cast<const f32x4g*>(&sm.slope[buf][lr]);
        qp = *reinterpret_cast<const int4*>(&sm.qp[buf][lr]);
      }
      const int qpv[4] = {qp.x, qp.y, qp.z, qp.w};
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y = lg.above<CAP>(x[g][4 * e + i], z[i]);
          if (DIST) y = fmaf(-sl[i], fabsf((float)(qpv[i] - kp[g])), y);
          const int r = kWeighRows * t + lr + i;
          sum[g] += r >= lo[g] && r < R ? exp2_hw(y) : 0.f;
        }
    }
  };
  // dot products of 32 rows into xn, and the probabilities of the 32 rows before, which see every key, from x
  auto unit = [&](f32x16g (&x)[2], f32x16g (&xn)[2], int buf, int rb, int buf_n, int rb_n) {
    f32x4g z[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = *reinterpret_cast<const f32x4g*>(&sm.lse[buf][32 * rb + 8 * e + 4 * hh]);
    clear(xn);
    u32x4g a[KK];
    a[0] = q_operand(buf_n, rb_n, 0);
    a[1] = q_operand(buf_n, rb_n, 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (kk + 2 < KK) a[kk + 2] = q_operand(buf_n, rb_n, kk + 2);
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        xn[g] = Mfma<T>::m32(a[kk], k[g][kk], xn[g]);
        constexpr int EPK = 16 / KK;                               // elements per MFMA
#pragma unroll
        for (int i = EPK * kk; i < EPK * kk + EPK; ++i) sum[g] += exp2_hw(fmaf(x[g][i], lg.mul, -z[i >> 2][i & 3]));
      }
      // the order is pinned by what the next MFMA and these sums need
      asm volatile("" : "+v"(sum[0]), "+v"(sum[1]) : : "memory");
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  f32x16g xa[2], xb[2];
  int cur = 0, nxt = 1, old = 2;                                   // buffers of tiles t, t + 1, t + 2
  if (t0 < t1) {
    fetch(t0, 0);
    if (t0 + 1 < t1) fetch(t0 + 1, 1);
    vm_wait();
    __syncthreads();
    to_log2(0);
    clear(xa);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int g = 0; g < 2; ++g) xa[g] = Mfma<T>::m32(q_operand(0, 0, kk), k[g][kk], xa[g]);
  }
  for (int t = t0; t < t1; ++t) {
    vm_wait();                                                     // tile t + 1 is in LDS, and tile t - 1 is done with
    __syncthreads();
    if (t + 2 < t1) fetch(t + 2, old);
    if (t + 1 < t1) to_log2(nxt);
    if (MODE == 0 && all_there && kWeighRows * t >= wave_lo && kWeighRows * (t + 1) <= R) {
      unit(xa, xb, cur, 0, cur, 1);
      unit(xb, xa, cur, 1, nxt, 0);                                // (behind the last tile: of what the buffer holds, unused)
    } else {
      clear(xb);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int g = 0; g < 2; ++g) xb[g] = Mfma<T>::m32(q_operand(cur, 1, kk), k[g][kk], xb[g]);
      add(xa, t, cur, 0);
      clear(xa);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int g = 0; g < 2; ++g) xa[g] = Mfma<T>::m32(q_operand(nxt, 0, kk), k[g][kk], xa[g]);
      add(xb, t, cur, 1);
    }
    const int c = cur;
    cur = nxt; nxt = old; old = c;
  }
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    sum[g] += __shfl_xor(sum[g], 32);
    if (hh == 0 && krow[g] >= 0) {
      if (n_shares == 1) store_weight(A, krow[g], sum[g]);
      else A.ws[kTicketFloats + ((size_t)share * P.B * P.H + (size_t)b * P.H + h) * P.max_kv + w0 + 32 * g + n] = sum[g];
    }
  }
}

// Adds the shares' sums, in order.
__global__ __launch_bounds__(256) void k_weigh_join(PagedAttnArgs A, int few, int n_shares) {
  const Paged& P = A.P;
  const int h = blockIdx.y, b = blockIdx.z, j = blockIdx.x * 256 + threadIdx.x;
  const Seq s = seq_of(P, b);
  if (s.nq * A.G <= few) return;
  const int row = slot_row(P.table + (size_t)b * P.width, P.n_pages, P.H, h, P.lg_page, s.kv, j);
  if (row < 0) return;
  float sum = 0.f;
  for (int i = 0; i < n_shares; ++i) sum += A.ws[kTicketFloats + ((size_t)i * P.B * P.H + (size_t)b * P.H + h) * P.max_kv + j];
  store_weight(A, row, sum);
}

// Shares into which the rows that see a block of keys are dealt, where the blocks alone do not fill the chip; at least four
// tiles each.
static int weigh_shares(const Paged& P, int Hq) {
  const long long rows = (long long)P.max_q * (Hq / P.H), blocks = (long long)P.B * P.H * ((P.max_kv + kWeighKeys - 1) / kWeighKeys);
  if (rows <= kStepRows || blocks == 0) return 1;
  return (int)std::max(1ll, std::min(512 / blocks, rows / (4 * kWeighRows)));
}

size_t paged_weights_floats(const Paged& P, int Hq) {
  const int n = weigh_shares(P, Hq);
  return n == 1 ? 0 : kTicketFloats + (size_t)n * P.B * P.H * P.max_kv;
}
// For every batch of no more sequences, new tokens and rows than P's: shares times blocks are 512 at most, of 256 keys each.
size_t paged_weights_bound(const Paged& P, int Hq) {
  const size_t most = (size_t)P.max_q * (Hq / P.H) / (4 * kWeighRows);
  return kTicketFloats + (most < 2 ? 0 : std::min<size_t>(512 * kWeighKeys, most * P.B * P.H * P.max_kv));
}

template <typename T, int D, int MODE>
static hipError_t launch_weights(const PagedAttnArgs& A, hipStream_t st) {
  const Paged& P = A.P;
  const Which w = which_kernels(P, A.Hq);
  const int shares = weigh_shares(P, A.Hq);
  if (w.chunk) {
    const int blocks = (P.max_kv + kWeighKeys - 1) / kWeighKeys;
    k_weigh_chunk<T, D, MODE><<<dim3(blocks * shares, P.H, P.B), 256, 0, st>>>(A, w.few, shares);
    if (shares > 1) k_weigh_join<<<dim3((P.max_kv + 255) / 256, P.H, P.B), 256, 0, st>>>(A, w.few, shares);
  }
  if (w.step) {
    // as many keys per wave as still give a workgroup for every place on the chip
    const long long want = (long long)P.B * P.H * P.max_kv / (4 * 1024);
    const int keys = (int)std::min<long long>(kWeighStepKeys, std::max(64ll, (want + 31) / 32 * 32));
    k_weigh_step<T, D, MODE><<<dim3((P.max_kv + 4 * keys - 1) / (4 * keys), P.H, P.B), 256, 0, st>>>(A, keys);
  }
  return hipGetLastError();
}

hipError_t launch_paged_weights(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  return dispatch(dtype, D, mode_of(A.S), [&](auto t, auto d, auto m) {
    return launch_weights<typename decltype(t)::type, decltype(d)::value, decltype(m)::value>(A, st);
  });
}

}  // namespace arkv
