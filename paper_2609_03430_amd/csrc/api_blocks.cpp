// C ABI: rows of every head read at once, and block-sparse decode attention.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>
#include <vector>

#include "cache.h"
#include "ra_internal.h"
#include "randattn.h"

using ra::SeqMeta;
using ra::host::Plan;

namespace {

bool sparse_supported(const ra_config& c) {
  return c.dtype != RA_F32 && c.layout != RA_LAYOUT_HOLE_FILL;
}

size_t list_bytes(const ra_config& c, int32_t n_blocks) {
  const size_t per_head = static_cast<size_t>(std::min(n_blocks, ra::kMaxBlocks));
  const size_t n = static_cast<size_t>(c.max_seqs) * c.num_kv_heads * per_head * sizeof(int32_t);
  return (n + 255) / 256 * 256;
}

// Scores of the candidates, which the attention's partials follow in the same place.
size_t scores_bytes(const ra_config& c) {
  return static_cast<size_t>(c.max_seqs) * c.num_kv_heads * ra::kMaxBlocks * sizeof(uint32_t);
}

}  // namespace

extern "C" {

ra_status ra_export_rows(ra_cache* c, int32_t seq, void* dev_k, void* dev_v, int64_t out_elems,
                         void* stream) {
  if (!c || seq < 0 || seq >= c->cfg.max_seqs) return RA_ERR_INVALID_ARG;
  if (c->graph) return RA_ERR_STATE;   // needs the host mirror (ra_graph_mode)
  if (c->step_open()) return RA_ERR_STATE;
  const SeqMeta& M = c->mirror[seq];
  if (!M.active) return RA_ERR_STATE;
  if (out_elems < static_cast<int64_t>(M.len) * c->cfg.num_layers * c->cfg.num_kv_heads *
                      ra::kHeadDim)
    return RA_ERR_CAPACITY;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const ra_status fl = ra::host::flush_pending(c, s);
  if (fl != RA_OK) return fl;
  RA_LAUNCH(ra::launch_export_rows(c->shape(), M, seq, M.len, c->kpool, c->vpool, dev_k, dev_v, s));
  return RA_OK;
}

size_t ra_sparse_bytes(const ra_config* c, int64_t pool_rows) {
  if (ra_config_check(c) != RA_OK || !sparse_supported(*c) || pool_rows <= 0 ||
      pool_rows % ra::kBlockRows != 0 || pool_rows > (int64_t(1) << 40))
    return 0;
  return static_cast<size_t>(
      ra::host::round_up(pool_rows / ra::kBlockRows * (ra::kBoundsBytes + 1), 256));
}

size_t ra_sparse_workspace_bytes(const ra_config* c, int32_t n_blocks) {
  if (ra_config_check(c) != RA_OK || !sparse_supported(*c) || n_blocks < 0) return 0;
  return list_bytes(*c, n_blocks) + std::max(ra_workspace_bytes(c), scores_bytes(*c));
}

ra_status ra_sparse_attach(ra_cache* c, void* bounds, size_t bounds_bytes, void* stream) {
  if (!c) return RA_ERR_INVALID_ARG;
  if (!sparse_supported(c->cfg)) return RA_ERR_UNSUPPORTED;
  if (bounds && (bounds_bytes < ra_sparse_bytes(&c->cfg, c->pool_rows) ||
                 (reinterpret_cast<uintptr_t>(bounds) & 15u) != 0))
    return RA_ERR_INVALID_ARG;
  if (c->graph || c->step_open()) return RA_ERR_STATE;
  const ra_status fl = ra::host::flush_pending(c, static_cast<hipStream_t>(stream));
  if (fl != RA_OK) return fl;
  try {
    std::vector<int32_t> built(
        bounds ? static_cast<size_t>(c->cfg.num_layers) * c->cfg.max_seqs : 0, 0);
    std::vector<uint8_t> layers(c->cfg.num_layers, 0);
    c->ranges.reserve(c->cfg.max_seqs);
    c->stale_layers.reserve(c->cfg.num_layers);
    c->bounds_built.swap(built);
    c->sparse_layers.swap(layers);
  } catch (const std::bad_alloc&) {
    return RA_ERR_CAPACITY;
  }
  c->bounds = static_cast<int8_t*>(bounds);
  return RA_OK;
}

ra_status ra_sparse_attention(ra_cache* c, int32_t layer, int32_t n_blocks, int32_t recent_rows,
                              const void* q, const void* k_new, const void* v_new, void* out,
                              void* workspace, size_t workspace_bytes, void* stream) {
  if (n_blocks < 0 || recent_rows < 0) return RA_ERR_INVALID_ARG;
  const ra_status st = ra::host::check_decode(c, layer, q, k_new, v_new, out);
  if (st != RA_OK) return st;
  if (!sparse_supported(c->cfg)) return RA_ERR_UNSUPPORTED;
  if (!c->bounds || c->graph) return RA_ERR_STATE;   // (graph mode: bounds follow the mirror)
  if (!workspace || workspace_bytes < ra_sparse_workspace_bytes(&c->cfg, n_blocks) ||
      (reinterpret_cast<uintptr_t>(workspace) & 15u) != 0)
    return RA_ERR_INVALID_ARG;
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  // what to rebuild is decided here: a replay would not decide it again
  // (nor may the null stream be used while another is captured)
  hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
  const hipError_t asked = hipStreamIsCapturing(hs, &capturing);
  if (asked != hipSuccess) (void)hipGetLastError();   // (the next launch must not report it)
  if (asked == hipErrorStreamCaptureImplicit) return RA_ERR_STATE;
  if (asked != hipSuccess) return ra::host::hip_fail(asked);
  if (capturing != hipStreamCaptureStatusNone) return RA_ERR_STATE;
  // the attended rows of the longest step, and the slots that choose their blocks
  std::vector<ra::BoundsRange>& ranges = c->ranges;
  ranges.clear();
  int most = 0, n_active = 0, candidates = 0;
  bool stale = false;
  const auto built = [&](int l, int s) -> int32_t& {
    return c->bounds_built[static_cast<size_t>(l) * c->cfg.max_seqs + s];
  };
  for (int s = c->slot_lo; s < c->slot_hi; ++s) {
    const SeqMeta& M = c->mirror[s];
    if (!M.active) continue;
    ++n_active;
    most = std::max(most, ra::attended_blocks(M.len, recent_rows, n_blocks));
    const int cand = ra::candidate_blocks(M.len, recent_rows);
    if (cand <= n_blocks) continue;
    candidates = std::max(candidates, cand);
    if (n_blocks == 0) continue;      // none is chosen: no bounds
    stale = stale || built(layer, s) < cand;
    ranges.push_back(ra::BoundsRange{s, cand, cand});
  }
  if (candidates > ra::kMaxBlocks) return RA_ERR_UNSUPPORTED;
  const ra_status grown = ra::host::grow_for_step(c, hs);
  if (grown != RA_OK) return grown;
  ra::Shape sh = c->shape();
  sh.order = c->refresh_order();
  c->sparse_layers[layer] = 1;
  if (stale) {
    // one launch for every layer that sparse steps are made of: rows change in all
    // layers at once (36 layers of a request of 2,100 rows, one launch each: 4.8 us
    // each)
    std::vector<int>& layers = c->stale_layers;
    layers.clear();
    for (int l = 0; l < c->cfg.num_layers; ++l) {
      bool any = false;
      for (ra::BoundsRange& r : ranges) {
        any = any || (c->sparse_layers[l] && built(l, r.slot) < r.to);
        if (c->sparse_layers[l]) r.from = std::min(r.from, built(l, r.slot));
      }
      if (any) layers.push_back(l);
    }
    ranges.erase(std::remove_if(ranges.begin(), ranges.end(),
                                [](const ra::BoundsRange& r) { return r.from >= r.to; }),
                 ranges.end());
    RA_LAUNCH(ra::launch_block_bounds(sh, c->meta, c->kpool, c->bounds, c->pool_rows,
                                      layers.data(), static_cast<int>(layers.size()),
                                      ranges.data(), static_cast<int>(ranges.size()), hs));
    for (const int l : layers)
      for (const ra::BoundsRange& r : ranges) built(l, r.slot) = std::max(built(l, r.slot), r.to);
  }
  int32_t* list = static_cast<int32_t*>(workspace);
  void* scratch = static_cast<char*>(workspace) + list_bytes(c->cfg, n_blocks);
  ra::BlockChoice choice;
  choice.list = list;
  choice.stride = n_blocks;      // (more than kMaxBlocks: no head chooses)
  choice.n_blocks = n_blocks;
  choice.recent = recent_rows;
  choice.bounds = c->bounds;
  choice.units = c->bounds + c->pool_rows / ra::kBlockRows * ra::kBoundsBytes;
  if (candidates > 0 && n_blocks > 0)
    RA_LAUNCH(ra::launch_choose_blocks(sh, c->meta, q, layer, c->slot_hi, choice,
                                       static_cast<uint32_t*>(scratch), ra::kMaxBlocks,
                                       c->arrivals, candidates, hs));
  c->appended[layer] = 1;
  ++c->n_appended;
  if (n_active == 0) return RA_OK;
  const Plan plan = ra::host::plan_blocks(c, int64_t(most) * ra::kBlockRows,
                                          n_active * c->cfg.num_kv_heads);
  const size_t items = static_cast<size_t>(c->cfg.max_seqs) * c->cfg.num_kv_heads * ra::kMaxSplits;
  ra::AttnLaunch a{};
  a.meta = c->meta;
  a.kpool = c->kpool;
  a.vpool = c->vpool;
  a.pos = c->pos;
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.out = out;
  a.ws_o = static_cast<float*>(scratch);
  a.ws_ml = a.ws_o + items * c->G * ra::kHeadDim;
  a.split_stride = ra::kMaxSplits;
  a.layer = layer;
  a.max_seqs = c->slot_hi;
  a.split_keys = plan.launch_keys();
  a.max_splits = plan.launch_splits();
  a.waves = plan.launch_waves();
  a.arrivals = c->arrivals;
  const hipError_t e = ra::launch_block_attention(sh, a, choice, hs);
  if (e != hipSuccess) {
    c->appended[layer] = 0;
    --c->n_appended;
    return ra::host::hip_fail(e);
  }
  return RA_OK;
}

}  // extern "C"
