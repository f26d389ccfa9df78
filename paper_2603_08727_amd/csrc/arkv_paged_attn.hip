// Attention over 16-bit pages, every new token seeing all slots up to its own: its builds, and the sizes of workspaces and launches.
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

hipError_t launch_paged_attention(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  return dispatch(dtype, D, mode_of(A.S), [&](auto t, auto d, auto m) {
    return launch_attention<typename decltype(t)::type, decltype(d)::value, decltype(m)::value, 16, false>(A, st);
  });
}

}  // namespace arkv
