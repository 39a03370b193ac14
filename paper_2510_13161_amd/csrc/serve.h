// Host checks that the serving entry points share.
#pragma once
#include "kernels.h"
#include "msd.h"

namespace msd {

// Sets msd_last_error()'s text and returns s.
msd_status report(msd_status s, const char* msg) noexcept;

// Block topology from parents (null: a chain): false unless parent[0] = -1 and
// 0 <= parent[i] < i.
inline bool topo_from(const int32_t* parent, int n, Topo* t) {
  t->n_slots = n;
  t->max_depth = 0;
  for (int i = 0; i < kMaxSlots; ++i) {
    t->anc[i] = 0;
    t->depth[i] = 0;
    t->parent[i] = -1;
  }
  for (int i = 0; i < n; ++i) {
    const int p = parent ? parent[i] : i - 1;
    if (i == 0 ? p != -1 : (p < 0 || p >= i)) return false;
    t->parent[i] = p;
    t->depth[i] = i == 0 ? 0 : t->depth[p] + 1;
    t->anc[i] = (i == 0 ? 0ull : t->anc[p]) | (1ull << i);
    if (t->depth[i] > t->max_depth) t->max_depth = t->depth[i];
  }
  return true;
}

// Host checks of a paged cache, and its kernels' view of it.
msd_status check_cache(const msd_paged_kv* kv, PagedView* v) noexcept;
// Launches a (its cache, layer, block and queries filled in) with the partial
// results in ws.
msd_status run_paged_attention(const msd_paged_kv* kv, PagedAttnArgs a, const Topo& topo, void* ws, size_t ws_bytes,
                               hipStream_t stream) noexcept;

}  // namespace msd
