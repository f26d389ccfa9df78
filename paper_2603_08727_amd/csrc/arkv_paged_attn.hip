// Attention over 16-bit pages, every new token seeing all slots up to its own: its builds, and the sizes of workspaces and launches.
#include <iterator>

#include "arkv_paged_attn.h"

namespace arkv {

// Rows of partial results that suffice for every batch of no more sequences, tokens, new tokens and rows than P's: fewer of them
// may be cut finer, so this bounds part_rows over all such batches.  With u units and want workgroups wanted, a cut whose pieces are
// neither the shortest nor the longest allowed has at most ceil(want / u) of them, and u times that is below want + u.
static size_t part_rows_bound(const Paged& P, int D, int Hq) {
  auto parts = [](long long n, long long piece) { return (n + piece - 1) / piece; };
  const long long kv = P.max_kv, units = (long long)P.B * P.H, rows = (long long)P.N * (Hq / P.H);
  long long n = 0, step = 0;
  if (kv > 128)
    n = step = kStepRows * std::min(units * parts(kv, 128), std::max({256 + units, units * parts(kv, kStepMaxPiece), std::min(units, 15ll) * parts(kv, kStepMaxPiece / 2)}));
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
  if ((long long)P.max_q * (Hq / P.H) > kStepRows) {
    const long long sequences = std::min<long long>(P.B, rows);
    // groups of kStepRows rows, of which no more than kGroupWorkgroups are wanted with their pieces, which are of 128 keys at least
    const long long groups = (rows / kStepRows + sequences) * P.H;
    if (kv > 128) n = std::max(n, kStepRows * std::min(groups * parts(kv, 128), kGroupWorkgroups + std::min<long long>(groups, kJoinUnits)));
    // blocks whose pieces may be halved: of 256 keys at least
    if (kv > 256) n = std::max(n, step + kChunkRows * std::min<long long>(kJoinBlocks, (rows / kChunkRows + sequences) * P.H * parts(kv, 256)));
  }
  return (size_t)n;
}

size_t paged_attention_floats(const Paged& P, const Sight& V, int D, int Hq) {
  size_t chunk0;
  const Cut c = cut_of(P, V, D, Hq);
  const size_t rows = part_rows(P, Hq, c, chunk0);
  return kTicketFloats + rows * (D + 2) + (c.chunk_spread ? 2 + 4 * (size_t)c.blocks * P.H : 0);
}
size_t paged_attention_bound(const Paged& P, int D, int Hq) {
  return kTicketFloats + part_rows_bound(P, D, Hq) * (D + 2) + ((long long)P.max_q * (Hq / P.H) > kStepRows && P.max_kv > 256 ? 2 + 4 * kJoinBlocks : 0);
}

long long paged_attention_workgroups(const Paged& P, const Sight& V, int D, int Hq) {
  const Launches l = launches_of(P, Hq, cut_of(P, V, D, Hq));
  return std::max(l.chunk + l.step, l.merge);
}

void paged_attention_cut(const Paged& P, const Scores& S, const Sight& V, int D, int Hq, int32_t* cut) {
  const Cut c = cut_of(P, V, D, Hq);
  const int G = Hq / P.H;
  const auto seq = [&](int b) { return clamp_seq(P.cu_q[b], P.cu_q[b + 1], P.kv_len[b], P.N, P.max_q, P.max_kv); };
  const auto prefix = [&](int b) { return S.prefix ? S.prefix[b] : 0; };
  const int length = !c.places ? c.chunk_piece : chosen_piece(c, [&](auto f) {
    int x = 0;
    for (int b = 0; b < P.B; ++b) {
      const Load l = load_of(P, V, seq(b), prefix(b), G, c.w.few);
      x += f(l.blocks, l.tiles);
    }
    return x;
  });
  int step = 1, chunk = 1;
  long long chunks = 0;
  for (int b = 0; b < P.B; ++b) {
    const Seq s = seq(b);
    const int R = s.nq * G, blocks = row_blocks<kChunkRows>(s.nq, G, c.w.few);
    const auto pieces = [&](int r0, int rows, int piece) {
      return std::max(1, (Keys<true>(V, s, prefix(b), r0 / G, (std::min(R, r0 + rows) - 1) / G).end + piece - 1) / piece);
    };
    if (c.w.chunk)
      for (int i = 0; i < blocks; ++i) {
        const int n = pieces(i * kChunkRows, kChunkRows, length);
        chunk = std::max(chunk, n);
        chunks += (long long)n * P.H;
      }
    if (c.w.step && (c.groups || R <= kStepRows))
      for (int r0 = 0; r0 < R; r0 += kStepRows) step = std::max(step, pieces(r0, kStepRows, c.step_piece));
  }
  const int joined = chunk == 1 ? 0 : c.chunk_joined ? 1 : c.chunk_spread ? 2 : 3;
  const int32_t got[] = {(c.w.chunk ? 1 : 0) | (c.w.step ? 2 : 0), c.groups, c.step_piece, step, length, chunk, joined, (int32_t)std::min(chunks, 1ll << 30), c.places};
  std::copy(std::begin(got), std::end(got), cut);
}

hipError_t launch_paged_attention(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  return dispatch(dtype, D, mode_of(A.S), [&](auto t, auto d, auto m) {
    return launch_attention<typename decltype(t)::type, decltype(d)::value, decltype(m)::value, 16, false>(A, st);
  });
}

}  // namespace arkv
