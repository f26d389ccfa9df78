// Attention over pages of 4-bit rows: its builds.
#include "arkv_paged_attn.h"

namespace arkv {

hipError_t launch_packed_attention4(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  return dispatch(dtype, D, mode_of(A.S), [&](auto t, auto d, auto m) {
    return launch_attention<typename decltype(t)::type, decltype(d)::value, decltype(m)::value, 4, true>(A, st);
  });
}

}  // namespace arkv
