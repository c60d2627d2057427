// Attention of chunks of prompts over the paged cache: kernels in pprefill_kernel.h.
#include "pprefill_kernel.h"

namespace sna {

bool chunks_fit_a_launch(const PagedAttnArgs& a) {
  return fits_a_launch(chunk_blocks(a), 64 * a.waves) && (a.splits == 1 || fits_a_launch(a.s.T, 256));
}
hipError_t launch_paged_chunks(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t s) { return launch_chunks<false>(a, dtype, head_dim, s); }

}  // namespace sna
