// C ABI of the serving operators (include/msd.h): the paged cache's append,
// commit and attention, and sampling. Argument checks and launches; every call
// is asynchronous on the caller's stream and allocates nothing.
#include <algorithm>
#include <cmath>

#include "serve.h"

using namespace msd;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0; }

msd_status hip_fail(hipError_t e) { return e == hipSuccess ? MSD_OK : report(MSD_ERR_HIP, hipGetErrorString(e)); }

msd_status check_rope(const msd_rope* r, const PagedView& kv, RopeView* v) {
  *v = RopeView{nullptr, 0, 0};
  if (!r) return MSD_OK;
  if (!r->table) return report(MSD_ERR_INVALID_ARG, "null rotation table");
  if (((uintptr_t)r->table & 7u) != 0) return report(MSD_ERR_INVALID_ARG, "rotation table must be 8-byte aligned");
  if (r->layout != MSD_ROPE_HALF && r->layout != MSD_ROPE_INTERLEAVED)
    return report(MSD_ERR_INVALID_ARG, "unknown rotation layout");
  if (r->rotary_dim < 16 || r->rotary_dim > kv.head_dim || r->rotary_dim % 16)
    return report(MSD_ERR_SHAPE, "rotary_dim must be a multiple of 16, at most head_dim");
  if (r->positions < kv.capacity)
    return report(MSD_ERR_CAPACITY, "the rotation table is shorter than max_pages * page_size");
  *v = RopeView{reinterpret_cast<const float2*>(r->table), r->rotary_dim, r->layout == MSD_ROPE_INTERLEAVED};
  return MSD_OK;
}

msd_status fill_append(const msd_paged_kv* kv, const msd_kv_rows* rows, const msd_rope* rope, AppendArgs* a) {
  *a = AppendArgs{};
  msd_status st = check_cache(kv, &a->kv);
  if (st != MSD_OK) return st;
  if (!rows || !rows->k || !rows->v) return report(MSD_ERR_INVALID_ARG, "null rows");
  if (!aligned16(rows->k) || !aligned16(rows->v)) return report(MSD_ERR_INVALID_ARG, "rows must be 16-byte aligned");
  if (!stride_ok(rows->layer_stride) || !stride_ok(rows->seq_stride) || !stride_ok(rows->row_stride) ||
      !stride_ok(rows->head_stride))
    return report(MSD_ERR_SHAPE, "row strides must be >= 0 and multiples of 8 elements");
  if (rows->n_layers < 1 || rows->layer < 0 || rows->layer > kv->n_layers - rows->n_layers)
    return report(MSD_ERR_SHAPE, "layers outside the cache");
  if (rows->batch < 1 || rows->batch > kv->batch_cap) return report(MSD_ERR_SHAPE, "batch must lie in [1, batch_cap]");
  if (rows->n_rows < 1 || rows->n_rows > a->kv.capacity)
    return report(MSD_ERR_CAPACITY, "n_rows must lie in [1, max_pages * page_size]");
  st = check_rope(rope, a->kv, &a->rope);
  if (st != MSD_OK) return st;
  a->k = static_cast<const uint16_t*>(rows->k);
  a->v = static_cast<const uint16_t*>(rows->v);
  a->layer_stride = rows->layer_stride;
  a->seq_stride = rows->seq_stride;
  a->row_stride = rows->row_stride;
  a->head_stride = rows->head_stride;
  a->layer = rows->layer;
  a->n_layers = rows->n_layers;
  a->batch = rows->batch;
  a->n_rows = rows->n_rows;
  a->count = rows->count;
  // the grid: blocks and heads, sequences, layers
  if (a->batch > 65535 || a->n_layers > 65535 ||
      (int64_t)((a->n_rows + 14) / 16 + 1) * a->kv.heads > (int64_t)1 << 24)
    return report(MSD_ERR_SHAPE, "too many rows for one call");
  return MSD_OK;
}

// Launch shape of an attention call (8-bit pages, 8 kv heads, head dim 128 unless said;
// attention and joining kernel).
//
// Query tiles: groups of tiles read the keys again, so few groups of many tiles where
// the keys are many; but a tile costs a workgroup 3.1 us of its own (queries, own
// keys, joining the waves) beside 2.2 + 0.2 a tile for each round of 8 blocks (fitted to chains and
// trees at 100 to 30000). The count with the least of that is taken. A chain of 9 slots,
// 5 heads a kv head, at 100: 16.8 us with 3 tiles a workgroup, 10.1 with one; at 6000
// 27.2 and 20.5; at 30000 37.3 and 39.3; 8 sequences at 4000 35 and 47.7, 16 at 300
// (2 tiles) 16.8 and 22.3; a tree of
// 25 slots at 8000 33.0 with 3, 29.4 with 2, 30.7 with one.
//
// Workgroups: where the sequences alone fill fewer than the device holds at once and a
// sequence can have more blocks than two for each wave, chunks are planned on the
// device over that many workgroups and joined by a second kernel. 14 blocks, one token:
// 11.5 in one workgroup, 13.7 split; 29 blocks 15.4 and 14.8, of a chain 25.8 and 20.9.
// 16 sequences at 512 to 8192: over 256 workgroups 42.3, over 512 47.6 (chains 61.9 and
// 71.4); at head dim 64 (two fit a compute unit) 32.6 and 29.0.
constexpr int64_t kPagedWgs = 512;      // workgroups of one query tile at head dim 64
constexpr int64_t kPagedWgsMany = 256;  // others
constexpr int64_t kPagedAlone = 16;     // blocks that one workgroup takes without a split
struct PagedShape {
  int q_per_wg, groups, wgs;
};
PagedShape paged_shape(const msd_paged_kv* kv, int32_t batch, int32_t n_slots, int32_t n_heads, int64_t blocks) {
  const int32_t heads = kv->n_kv_heads;
  const bool light = kv->head_dim == 64;
  const int tiles = (n_heads / heads * n_slots + 15) / 16;
  PagedShape s;
  const int most = paged_max_tiles(kv->format == MSD_KV_FP8, kv->head_dim);
  const int64_t rounds = (blocks + 7) / 8;
  // 10 ns of a workgroup of q tiles: its chunk's rounds, those of all its turns on a full device
  auto cost = [&](int q) {
    const int64_t fit = kPagedWgsMany;  // two on a compute unit take turns
    const int64_t all = (int64_t)batch * heads * ((tiles + q - 1) / q), chunks = std::max<int64_t>(1, fit / all);
    return ((rounds + chunks - 1) / chunks * (225 + 22 * q) + 315 * q) * ((all + fit - 1) / fit);
  };
  int q = std::min(tiles, most);
  for (int fewer = q - 1; fewer >= 1; --fewer)
    if (cost(fewer) < cost(q)) q = fewer;
  s.groups = (tiles + q - 1) / q;
  s.q_per_wg = (tiles + s.groups - 1) / s.groups;
  const int64_t share = (s.q_per_wg == 1 && light ? kPagedWgs : kPagedWgsMany) / ((int64_t)heads * s.groups);
  // (the plan counts all sequences' blocks in 32 bits)
  s.wgs = blocks <= kPagedAlone || share <= batch || batch > kPagedPlanBatch || blocks * batch > INT32_MAX
              ? 0
              : (int)std::min<int64_t>(share, batch * ((blocks + 7) / 8));
  return s;
}
size_t paged_partials(const PagedShape& s, int32_t heads, int32_t hd) {
  return (size_t)s.wgs * heads * s.groups * s.q_per_wg * 16 * (hd + 2) * sizeof(float);
}
constexpr size_t kPagedPlanBytes = (kPagedPlanBatch + 4) * sizeof(int32_t);

}  // namespace

namespace msd {

msd_status check_cache(const msd_paged_kv* kv, PagedView* v) noexcept {
  if (!kv) return report(MSD_ERR_INVALID_ARG, "null paged cache");
  if (!kv->k || !kv->v || !kv->page_table || !kv->len || !kv->status)
    return report(MSD_ERR_INVALID_ARG, "null paged cache field");
  if (kv->format != MSD_KV_BF16 && kv->format != MSD_KV_FP8)
    return report(MSD_ERR_UNSUPPORTED, "unknown paged cache format");
  if (kv->format == MSD_KV_FP8 && (!kv->k_scale || !kv->v_scale))
    return report(MSD_ERR_INVALID_ARG, "8-bit pages need k_scale and v_scale");
  if (!aligned16(kv->k) || !aligned16(kv->v)) return report(MSD_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if (kv->head_dim != 64 && kv->head_dim != 128) return report(MSD_ERR_SHAPE, "head_dim must be 64 or 128");
  int shift = 4;
  while (shift <= 8 && (1 << shift) != kv->page_size) ++shift;
  if (shift > 8) return report(MSD_ERR_SHAPE, "page_size must be 16, 32, 64, 128 or 256");
  if (kv->n_layers < 1 || kv->n_pages < 1 || kv->n_kv_heads < 1 || kv->batch_cap < 1 || kv->max_pages < 1)
    return report(MSD_ERR_SHAPE, "paged cache sizes must be >= 1");
  const int64_t cap = (int64_t)kv->max_pages * kv->page_size;
  if (cap > (int64_t)1 << 30) return report(MSD_ERR_CAPACITY, "max_pages * page_size above 2^30");
  *v = PagedView{kv->k, kv->v, kv->k_scale, kv->v_scale, kv->page_table, kv->len, kv->status,
                 kv->n_pages, kv->n_kv_heads, shift, kv->head_dim, kv->max_pages, cap};
  return MSD_OK;
}

msd_status run_paged_attention(const msd_paged_kv* kv, PagedAttnArgs a, const Topo& topo, void* ws, size_t ws_bytes,
                               hipStream_t stream) noexcept {
  // blocks that a sequence can have: of its whole capacity, or of the sinks and the window
  int64_t blocks = (a.kv.capacity + 31) / 32;
  if (a.window > 0)
    blocks = std::min(blocks, ((int64_t)a.sinks + 31) / 32 + ((int64_t)a.window + a.n_slots + 30) / 32 + 1);
  if (a.k_new) blocks += (a.n_slots + 31) / 32;
  const PagedShape sh = paged_shape(kv, a.batch, a.n_slots, a.n_heads, blocks);
  a.q_per_wg = sh.q_per_wg;
  a.groups = sh.groups;
  a.wgs = sh.wgs;
  const size_t rows = (size_t)sh.wgs * kv->n_kv_heads * sh.groups * sh.q_per_wg * 16;
  a.plan = static_cast<int32_t*>(ws);
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + kPagedPlanBytes);
  a.part_ml = a.part_o + rows * kv->head_dim;
  if (kPagedPlanBytes + paged_partials(sh, kv->n_kv_heads, kv->head_dim) > ws_bytes)
    return report(MSD_ERR_WORKSPACE, "workspace too small");
  return hip_fail(launch_paged_attention(kv->format == MSD_KV_FP8, a, topo, stream));
}

}  // namespace msd

extern "C" {

msd_status msd_paged_append(const msd_paged_kv* kv, const msd_kv_rows* rows, const msd_rope* rope,
                            hipStream_t stream) {
  AppendArgs a;
  const msd_status st = fill_append(kv, rows, rope, &a);
  if (st != MSD_OK) return st;
  return hip_fail(launch_paged_append(kv->format == MSD_KV_FP8, a, stream));
}

msd_status msd_paged_commit(const msd_paged_kv* kv, const msd_kv_rows* rows, const msd_rope* rope,
                            const int32_t* acc_len, const int32_t* path, hipStream_t stream) {
  AppendArgs a;
  const msd_status st = fill_append(kv, rows, rope, &a);
  if (st != MSD_OK) return st;
  if (!acc_len || !path) return report(MSD_ERR_INVALID_ARG, "null acc_len or path");
  if (rows->count) return report(MSD_ERR_INVALID_ARG, "a commit takes its counts from acc_len: count must be NULL");
  if (rows->n_rows > kMaxSlots) return report(MSD_ERR_SHAPE, "a block has at most 64 slots");
  if (rows->layer != 0 || rows->n_layers != kv->n_layers)
    return report(MSD_ERR_SHAPE, "a commit covers all layers of the cache");
  a.acc_len = acc_len;
  a.path = path;
  const hipError_t e = launch_paged_append(kv->format == MSD_KV_FP8, a, stream);
  return hip_fail(e != hipSuccess ? e : launch_paged_advance(a, stream));
}

size_t msd_paged_attention_workspace_bytes(const msd_paged_kv* kv, int32_t batch, int32_t n_slots,
                                           int32_t n_heads) {
  if (!kv || batch < 1 || n_slots < 1 || n_heads < 1 || kv->n_kv_heads < 1) return 0;
  // The most that any smaller call uses: kPagedWgs workgroups of one tile, or
  // kPagedWgsMany of up to 3.
  const size_t tiles = ((size_t)((n_heads + kv->n_kv_heads - 1) / kv->n_kv_heads) * n_slots + 15) / 16;
  const size_t most = tiles == 1 ? (size_t)kPagedWgs
                                 : std::max((size_t)kPagedWgs, (size_t)kPagedWgsMany * std::min<size_t>(tiles, 3));
  return kPagedPlanBytes + most * 16 * (kv->head_dim + 2) * sizeof(float);
}

msd_status msd_paged_attention(const msd_paged_kv* kv, int32_t layer, const msd_paged_attn* at, void* ws,
                               size_t ws_bytes, hipStream_t stream) {
  PagedAttnArgs a{};
  msd_status st = check_cache(kv, &a.kv);
  if (st != MSD_OK) return st;
  if (!at || !at->q || !at->out) return report(MSD_ERR_INVALID_ARG, "null query or output");
  if ((at->k_new == nullptr) != (at->v_new == nullptr))
    return report(MSD_ERR_INVALID_ARG, "k_new and v_new go together");
  if (layer < 0 || layer >= kv->n_layers) return report(MSD_ERR_SHAPE, "layer outside the cache");
  if (!aligned16(at->q) || !aligned16(at->out) || !aligned16(at->k_new) || !aligned16(at->v_new))
    return report(MSD_ERR_INVALID_ARG, "rows must be 16-byte aligned");
  if (!stride_ok(at->q_seq) || !stride_ok(at->q_row) || !stride_ok(at->q_head) || !stride_ok(at->out_seq) ||
      !stride_ok(at->out_row) || !stride_ok(at->out_head) || !stride_ok(at->new_seq) || !stride_ok(at->new_row) ||
      !stride_ok(at->new_head))
    return report(MSD_ERR_SHAPE, "strides must be >= 0 and multiples of 8 elements");
  if (at->batch < 1 || at->batch > kv->batch_cap || at->batch > 65535)
    return report(MSD_ERR_SHAPE, "batch must lie in [1, min(batch_cap, 65535)]");
  if (at->n_slots < 1 || at->n_slots > kMaxSlots) return report(MSD_ERR_SHAPE, "n_slots must lie in [1, 64]");
  if (at->n_heads < 1 || at->n_heads % kv->n_kv_heads)
    return report(MSD_ERR_SHAPE, "n_heads must be a multiple of n_kv_heads");
  if (at->n_heads > 65536) return report(MSD_ERR_SHAPE, "n_heads above 65536");
  if (!std::isfinite(at->scale)) return report(MSD_ERR_INVALID_ARG, "scale must be finite");
  if (at->window < 0 || at->sinks < 0) return report(MSD_ERR_INVALID_ARG, "window and sinks must be >= 0");
  if (!at->k_new && at->parent) return report(MSD_ERR_UNSUPPORTED, "a tree needs its keys in k_new and v_new");
  if (a.kv.capacity < at->n_slots) return report(MSD_ERR_CAPACITY, "max_pages * page_size below n_slots");
  Topo topo;
  if (!topo_from(at->parent, at->n_slots, &topo))
    return report(MSD_ERR_SHAPE, "parent[0] must be -1 and parent[i] lie in [0, i)");
  st = check_rope(at->rope, a.kv, &a.rope);
  if (st != MSD_OK) return st;
  if (!ws || !aligned16(ws) ||
      ws_bytes < msd_paged_attention_workspace_bytes(kv, at->batch, at->n_slots, at->n_heads))
    return report(MSD_ERR_WORKSPACE, "workspace NULL, unaligned or too small");
  a.layer = layer;
  a.q = static_cast<const uint16_t*>(at->q);
  a.q_seq = at->q_seq;
  a.q_row = at->q_row;
  a.q_head = at->q_head;
  a.out = static_cast<uint16_t*>(at->out);
  a.out_seq = at->out_seq;
  a.out_row = at->out_row;
  a.out_head = at->out_head;
  a.k_new = static_cast<const uint16_t*>(at->k_new);
  a.v_new = static_cast<const uint16_t*>(at->v_new);
  a.new_seq = at->new_seq;
  a.new_row = at->new_row;
  a.new_head = at->new_head;
  a.count = at->count;
  a.scale = at->scale;
  a.batch = at->batch;
  a.n_slots = at->n_slots;
  a.n_heads = at->n_heads;
  a.window = at->window;
  a.sinks = at->sinks;
  return run_paged_attention(kv, a, topo, ws, ws_bytes, stream);
}

size_t msd_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1) return 0;
  return sample_ws_bytes(rows, vocab);
}

msd_status msd_sample(const float* logits, int64_t row_stride, int32_t rows, int32_t vocab,
                      const msd_sample_params* params, const float* u, int32_t* tok, float* logp,
                      int32_t* kept, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!logits || !u || !tok) return report(MSD_ERR_INVALID_ARG, "null logits, u or tok");
  if (rows < 1 || rows > 65535) return report(MSD_ERR_SHAPE, "rows must lie in [1, 65535]");
  if (vocab < 1 || vocab > 1048576) return report(MSD_ERR_SHAPE, "vocab must lie in [1, 1048576]");
  if (row_stride < vocab) return report(MSD_ERR_SHAPE, "row_stride below vocab");
  if (!ws || !aligned16(ws) || ws_bytes < msd_sample_workspace_bytes(rows, vocab))
    return report(MSD_ERR_WORKSPACE, "workspace NULL, unaligned or too small");
  SampleArgs a{};
  a.logits = logits;
  a.row_stride = row_stride;
  a.rows = rows;
  a.vocab = vocab;
  if (params) {
    a.temperature = params->temperature;
    a.top_k = params->top_k;
    a.top_p = params->top_p;
    a.min_p = params->min_p;
  }
  a.u = u;
  a.tok = tok;
  a.logp = logp;
  a.kept = kept;
  a.ws = ws;
  return hip_fail(launch_sample(a, stream));
}

}  // extern "C"
