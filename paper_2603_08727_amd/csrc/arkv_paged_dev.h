// What the paged operators' host side and kernels share.
#pragma once
#include <hip/hip_runtime.h>

#include "arkv_paged.h"

namespace arkv {

int hip_failure(hipError_t e, const char* what);   // keeps the text for arkv_last_hip_error, returns ARKV_EHIP

// Pages and sequences as the kernels take them.
struct Paged {
  void *k, *v;
  int32_t* pos;
  float* weight;
  const int32_t *cu_q, *kv_len, *table;
  int n_pages, lg_page, H, B, N, max_q, max_kv, width;
};

struct Rows { const void* p; int64_t ts, hs; };

struct Scores { float scale, cap; const float* slopes; const int32_t *q_pos, *prefix; };

// One sequence, cut to what the launch was announced: nothing behind these numbers reaches outside the arrays.
struct Seq { int q0, nq, kv; };
__host__ __device__ inline Seq clamp_seq(int a, int e, int kv, int N, int max_q, int max_kv) {
  Seq s;
  s.q0 = a < 0 ? 0 : (a > N ? N : a);
  e = e > N ? N : e;
  s.nq = e > s.q0 ? e - s.q0 : 0;
  if (s.nq > max_q) s.nq = max_q;
  s.kv = kv < 0 ? 0 : (kv > max_kv ? max_kv : kv);
  return s;
}

// Row of [n_pages][H][page] of the slot at offset `off` of page id `page`, -1: no such page.
__host__ __device__ inline int page_row(int page, int n_pages, int H, int h, int lg_page, int off) {
  return (unsigned)page < (unsigned)n_pages ? ((page * H + h) << lg_page) + off : -1;
}
__host__ __device__ inline int slot_row(const int32_t* table_row, int n_pages, int H, int h, int lg_page, int len, int slot) {
  if ((unsigned)slot >= (unsigned)len) return -1;
  return page_row(table_row[slot >> lg_page], n_pages, H, h, lg_page, slot & ((1 << lg_page) - 1));
}

// The front of a workspace holds the tickets of k_paged_attn and k_evict_select, zero between calls; nothing else is kept there.
constexpr int kJoinUnits = 1024, kTicketWords = 16;                // (a ticket has a cache line of its own)
constexpr size_t kTicketFloats = (size_t)kJoinUnits * kTicketWords;

// A launch takes fewer than 2^32 work-items in x.
constexpr long long kMostWorkgroups = (1ll << 32) / 256 - 1;       // of 256

struct AppendArgs {
  Paged P;
  Rows q, k, v;
  void* q_out;
  const int32_t* positions;
  const double* freq;
  int Hq, half, adjacent, n_axes;
  uint8_t axis[64];
};
hipError_t launch_paged_append(int dtype, int D, const AppendArgs& A, hipStream_t st);

struct PagedAttnArgs {
  Paged P;
  Scores S;
  Rows q;
  void* out;
  float* lse;          // attention: written (or null); weights: read
  int Hq, G;
  float decay;
  const float* carried;
  float* ws;
};
// Floats of workspace: _floats: of this batch, _bound: of any that is no larger.
size_t paged_attention_floats(const Paged& P, int D, int Hq);
size_t paged_attention_bound(const Paged& P, int D, int Hq);
size_t paged_weights_floats(const Paged& P, int Hq);
size_t paged_weights_bound(const Paged& P, int Hq);
long long paged_attention_workgroups(const Paged& P, int D, int Hq);   // of its largest launch
hipError_t launch_paged_attention(int dtype, int D, const PagedAttnArgs& A, hipStream_t st);
hipError_t launch_paged_weights(int dtype, int D, const PagedAttnArgs& A, hipStream_t st);

struct EvictArgs {
  Paged P;
  const int32_t *keep, *dst_table;
  int32_t *kept, *new_len;
  int max_keep, sink, recent, dst_width;
  float* ws;           // null: none given
};
size_t paged_evict_floats(const Paged& P);
size_t paged_evict_bound(const Paged& P);
bool paged_evict_needs_workspace(const Paged& P, int D, int max_keep);
hipError_t launch_paged_evict(int D, const EvictArgs& A, hipStream_t st);

}  // namespace arkv
