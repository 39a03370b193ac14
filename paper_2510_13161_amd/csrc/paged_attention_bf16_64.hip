// The paged attention kernels of head dim 64 over bf16 pages (a source of their own: they build side by side).
#include "paged_attention.h"

namespace msd {
void launch_paged_bf16_64(const PagedAttnArgs& a, const Topo& topo, dim3 grid, hipStream_t s) {
  launch_tiles<64, false>(a, topo, grid, s);
}
}  // namespace msd
