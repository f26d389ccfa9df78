// Host side of include/arkv_paged.h: argument checks and launches.  Everything the kernels index by is either checked
// here or cut to the announced bounds in the kernel (clamp_seq, page_row).
#include <math.h>

#include <algorithm>

#include "arkv_paged_dev.h"

using namespace arkv;


static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// whether n words from p and m words from q share one
static bool overlap(const int32_t* p, size_t n, const int32_t* q, size_t m) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return a < b ? b - a < 4 * n : a - b < 4 * m;
}

static int check(const arkv_pages* p, const arkv_page_batch* b, Paged& P) {
  if (!p || !b || !p->k || !p->v || !p->pos || !b->cu_q || !b->kv_len || !b->table) return ARKV_EINVAL;
  if (p->n_pages < 1 || p->n_kv_heads < 1 || p->head_dim < 1 || p->page_size < 1) return ARKV_EINVAL;
  if (b->batch < 1 || b->n_tokens < 0 || b->max_q < 0 || b->max_kv < 0 || b->table_width < 1) return ARKV_EINVAL;
  if ((p->page_size & (p->page_size - 1)) || !aligned16(p->k) || !aligned16(p->v) || !aligned16(p->pos) || !aligned16(p->weight)) return ARKV_EINVAL;
  if (p->dtype != ARKV_DTYPE_BF16 && p->dtype != ARKV_DTYPE_FP16) return ARKV_EUNSUPPORTED;
  if ((p->head_dim != 64 && p->head_dim != 128) || p->page_size < 16 || p->page_size > 1024) return ARKV_EUNSUPPORTED;
  if ((int64_t)p->n_pages * p->n_kv_heads >= (int64_t)(1u << 31) / p->page_size) return ARKV_EUNSUPPORTED;
  if (b->batch > 65535 || p->n_kv_heads > 65535 || b->n_tokens > (1 << 28)) return ARKV_EUNSUPPORTED;
  if ((int64_t)b->max_kv > (int64_t)b->table_width * p->page_size || b->max_q > b->n_tokens) return ARKV_EINVAL;
  // (what the kernels count in 32 bits; how many workgroups a launch may have is checked where they are known)
  const int64_t units = (int64_t)b->batch * p->n_kv_heads;
  if (b->max_kv > (1 << 28) || units > (1 << 20) || units * b->max_kv > (1ll << 40)) return ARKV_EUNSUPPORTED;
  P.k = p->k; P.v = p->v; P.pos = p->pos; P.weight = p->weight;
  P.cu_q = b->cu_q; P.kv_len = b->kv_len; P.table = b->table;
  P.n_pages = p->n_pages; P.H = p->n_kv_heads; P.B = b->batch; P.N = b->n_tokens;
  P.max_q = b->max_q; P.max_kv = b->max_kv; P.width = b->table_width;
  P.lg_page = 0;
  while ((1 << P.lg_page) < p->page_size) ++P.lg_page;
  return ARKV_OK;
}

// (n: how many there are; arrays of none may have no address)
static int check_rows(const arkv_rows* r, int n, Rows& out) {
  if (!r || (!r->p && n) || !aligned16(r->p) || r->token_stride < 0 || r->head_stride < 0 || r->token_stride % 8 || r->head_stride % 8)
    return ARKV_EINVAL;
  out = {r->p, r->token_stride, r->head_stride};
  return ARKV_OK;
}

static int check_heads(int n_q_heads, int H, int n_tokens, int& G) {
  if (n_q_heads < 1 || n_q_heads % H) return ARKV_EINVAL;
  G = n_q_heads / H;
  return G > 16 || (int64_t)n_q_heads * n_tokens >= (1ll << 31) ? ARKV_EUNSUPPORTED : ARKV_OK;
}

// One size for all calls, so that a workspace serves every one of them: what this batch's need ...
static size_t workspace_bytes(const Paged& P, int D, int Hq) {
  return 4 * std::max({paged_attention_floats(P, D, Hq), paged_weights_floats(P, Hq), paged_evict_floats(P)});
}
// ... and what no smaller batch's exceed.
static size_t workspace_bound(const Paged& P, int D, int Hq) {
  return std::max(workspace_bytes(P, D, Hq), 4 * std::max({paged_attention_bound(P, D, Hq), paged_weights_bound(P, Hq), paged_evict_bound(P)}));
}

static int check_scores(const arkv_scores* s, Scores& out) {
  if (!s || !isfinite(s->scale) || !isfinite(s->cap) || s->cap < 0 || (s->slopes && !s->q_pos)) return ARKV_EINVAL;
  out = {s->scale, s->cap, s->slopes, s->q_pos, s->prefix};
  return ARKV_OK;
}

#define TRY(expr) do { const int rc_ = (expr); if (rc_ != ARKV_OK) return rc_; } while (0)
#define LAUNCH(expr) do { const hipError_t e_ = (expr); return e_ == hipSuccess ? ARKV_OK : hip_failure(e_, #expr); } while (0)

extern "C" {

int arkv_paged_append(const arkv_pages* pages, const arkv_page_batch* batch, const arkv_rotary* rotary, int32_t n_q_heads,
                      const arkv_rows* q, const arkv_rows* k, const arkv_rows* v, const int32_t* positions, void* q_out,
                      void* hip_stream) {
  AppendArgs A = {};
  TRY(check(pages, batch, A.P));
  if (!rotary || (!positions && A.P.N) || (!q != !q_out && A.P.N)) return ARKV_EINVAL;
  if (rotary->rot_dim < 0 || rotary->rot_dim % 16 || rotary->rot_dim > pages->head_dim || rotary->n_axes < 1 || rotary->n_axes > 4 ||
      (rotary->adjacent != 0 && rotary->adjacent != 1) || (rotary->rot_dim && !rotary->freq))
    return ARKV_EINVAL;
  for (int i = 0; i < rotary->rot_dim / 2; ++i) {
    if (rotary->axis[i] >= rotary->n_axes) return ARKV_EINVAL;
    A.axis[i] = rotary->axis[i];
  }
  TRY(check_rows(k, A.P.N, A.k));
  TRY(check_rows(v, A.P.N, A.v));
  if (q) {
    if (n_q_heads < 1 || !aligned16(q_out)) return ARKV_EINVAL;
    TRY(check_rows(q, A.P.N, A.q));
    if (n_q_heads > 65535) return ARKV_EUNSUPPORTED;
    // in place, every row has to lie where it is stored: other rows are still to be read
    const int64_t d = pages->head_dim;
    if (q->p && q->p == q_out && ((A.P.N > 1 && q->token_stride != n_q_heads * d) || (n_q_heads > 1 && q->head_stride != d))) return ARKV_EINVAL;
    A.Hq = n_q_heads;
  }
  A.q_out = q_out; A.positions = positions;
  A.freq = rotary->rot_dim ? rotary->freq : (const double*)pages->k;   // (read in any case, a branch would cost a round trip)
  A.half = rotary->rot_dim / 2; A.adjacent = rotary->adjacent; A.n_axes = rotary->n_axes;
  if (!A.P.N) return ARKV_OK;
  if (A.P.N > 4 * kMostWorkgroups) return ARKV_EUNSUPPORTED;       // (four tokens a workgroup)
  LAUNCH(launch_paged_append(pages->dtype, pages->head_dim, A, (hipStream_t)hip_stream));
}

int arkv_paged_workspace(const arkv_pages* pages, const arkv_page_batch* batch, int32_t n_q_heads, size_t* bytes) {
  Paged P;
  int G;
  if (!bytes) return ARKV_EINVAL;
  TRY(check(pages, batch, P));
  TRY(check_heads(n_q_heads, P.H, P.N, G));
  *bytes = workspace_bound(P, pages->head_dim, n_q_heads);
  return ARKV_OK;
}

static int attn_args(const arkv_pages* pages, const arkv_page_batch* batch, const arkv_scores* scores, int32_t n_q_heads,
                     const arkv_rows* q, void* workspace, size_t bytes, PagedAttnArgs& A) {
  TRY(check(pages, batch, A.P));
  TRY(check_heads(n_q_heads, A.P.H, A.P.N, A.G));
  TRY(check_scores(scores, A.S));
  TRY(check_rows(q, A.P.N, A.q));
  A.Hq = n_q_heads;
  const size_t need = workspace_bytes(A.P, pages->head_dim, n_q_heads);
  if (need && (!workspace || !aligned16(workspace) || bytes < need)) return ARKV_EINVAL;
  A.ws = (float*)workspace;
  return ARKV_OK;
}

int arkv_paged_attention(const arkv_pages* pages, const arkv_page_batch* batch, const arkv_scores* scores,
                         int32_t n_q_heads, const arkv_rows* q, void* out, float* lse, void* workspace, size_t bytes,
                         void* hip_stream) {
  PagedAttnArgs A = {};
  TRY(attn_args(pages, batch, scores, n_q_heads, q, workspace, bytes, A));
  if ((!out && A.P.N) || !aligned16(out)) return ARKV_EINVAL;
  A.out = out; A.lse = lse;
  if (!A.P.N || !A.P.max_q) return ARKV_OK;
  if (paged_attention_workgroups(A.P, pages->head_dim, n_q_heads) > kMostWorkgroups) return ARKV_EUNSUPPORTED;
  LAUNCH(launch_paged_attention(pages->dtype, pages->head_dim, A, (hipStream_t)hip_stream));
}

int arkv_paged_weights(const arkv_pages* pages, const arkv_page_batch* batch, const arkv_scores* scores,
                       int32_t n_q_heads, const arkv_rows* q, const float* lse, float decay, const float* carried,
                       void* workspace, size_t bytes, void* hip_stream) {
  PagedAttnArgs A = {};
  TRY(attn_args(pages, batch, scores, n_q_heads, q, workspace, bytes, A));
  if ((!lse && A.P.N) || !pages->weight || !isfinite(decay)) return ARKV_EINVAL;
  A.lse = const_cast<float*>(lse); A.decay = decay; A.carried = carried ? carried : pages->weight;
  if (!A.P.max_kv) return ARKV_OK;
  LAUNCH(launch_paged_weights(pages->dtype, pages->head_dim, A, (hipStream_t)hip_stream));
}

int arkv_paged_evict(const arkv_pages* pages, const arkv_page_batch* batch, const int32_t* keep, int32_t max_keep,
                     int32_t sink, int32_t recent, const int32_t* dst_table, int32_t dst_width, int32_t* kept,
                     int32_t* new_len, void* workspace, size_t bytes, void* hip_stream) {
  EvictArgs A = {};
  TRY(check(pages, batch, A.P));
  if (!keep || !dst_table || !kept || !new_len || !pages->weight || sink < 0 || recent < 0 || dst_width < 1 || max_keep < 1 ||
      (int64_t)max_keep > (int64_t)dst_width * pages->page_size)
    return ARKV_EINVAL;
  if (workspace || paged_evict_needs_workspace(A.P, pages->head_dim, max_keep)) {
    if (!workspace || !aligned16(workspace) || bytes < 4 * paged_evict_floats(A.P)) return ARKV_EINVAL;
  }
  // Workgroups read lengths and tables while others have written their results.
  const size_t B = A.P.B, n_kept = B * A.P.H * max_keep;
  struct { const int32_t* p; size_t n; } in[] = {{A.P.kv_len, B}, {keep, B}, {A.P.table, B * A.P.width}, {dst_table, B * dst_width}};
  for (const auto& i : in)
    if (overlap(kept, n_kept, i.p, i.n) || overlap(new_len, B, i.p, i.n)) return ARKV_EINVAL;
  if (overlap(kept, n_kept, new_len, B)) return ARKV_EINVAL;
  A.ws = (float*)workspace;
  A.keep = keep; A.dst_table = dst_table; A.kept = kept; A.new_len = new_len;
  A.max_keep = max_keep; A.sink = sink; A.recent = recent; A.dst_width = dst_width;
  LAUNCH(launch_paged_evict(pages->head_dim, A, (hipStream_t)hip_stream));
}

int arkv_debug_paged_row(const int32_t* table_row, int32_t table_width, int32_t n_pages, int32_t page_size,
                         int32_t n_kv_heads, int32_t kv_head, int32_t len, int32_t slot, int64_t* row) {
  if (!table_row || !row || table_width < 1 || n_pages < 1 || n_kv_heads < 1 || kv_head < 0 || kv_head >= n_kv_heads || len < 0)
    return ARKV_EINVAL;
  if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) || (int64_t)len > (int64_t)table_width * page_size)
    return ARKV_EINVAL;
  int lg = 0;
  while ((1 << lg) < page_size) ++lg;
  *row = slot_row(table_row, n_pages, n_kv_heads, kv_head, lg, len, slot);
  return ARKV_OK;
}

}  // extern "C"
