// Attention over 16-bit pages under a window, or of drafted trees: its builds.
#include "arkv_paged_attn.h"

namespace arkv {

hipError_t launch_paged_attention_sight(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  return dispatch(dtype, D, mode_of(A.S), [&](auto t, auto d, auto m) {
    return launch_attention<typename decltype(t)::type, decltype(d)::value, decltype(m)::value, 16, true>(A, st);
  });
}

}  // namespace arkv
