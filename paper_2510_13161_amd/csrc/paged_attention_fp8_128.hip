// The paged attention kernels of head dim 128 over 8-bit pages (a source of their own: they build side by side).
#include "paged_attention.h"

namespace msd {
void launch_paged_fp8_128(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s) {
  launch_tiles<128, true>(a, topo, grid, s);
}
}  // namespace msd
