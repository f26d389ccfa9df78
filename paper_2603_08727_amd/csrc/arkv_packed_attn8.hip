// Attention over pages of 8-bit rows: its builds.
#include "arkv_paged_attn.h"

namespace arkv {

hipError_t launch_packed_attention8(int dtype, int D, const PagedAttnArgs& A, hipStream_t st) {
  return dispatch(dtype, D, mode_of(A.S), [&](auto t, auto d, auto m) {
    return launch_attention<typename decltype(t)::type, decltype(d)::value, decltype(m)::value, 8, true>(A, st);
  });
}

}  // namespace arkv
