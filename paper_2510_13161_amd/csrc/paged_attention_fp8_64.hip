// The paged attention kernels of head dim 64 over 8-bit pages (a source of their own: they build side by side).
#include "paged_attention.h"

namespace msd {
void launch_paged_fp8_64(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s) {
  launch_tiles<64, true>(a, topo, grid, s);
}
}  // namespace msd
