// C ABI: rotary positions, decode attention under a score rule, and accumulated weights.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cache.h"
#include "ra_internal.h"
#include "randattn.h"

using ra::SeqMeta;
using ra::host::Plan;

namespace {

constexpr ra::WeightHooks kWeightHooks{ra::launch_weight_event, ra::launch_set_weights};

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

bool weights_supported(const ra_config& c) { return c.layout != RA_LAYOUT_HOLE_FILL; }

// Rows that a head's scores take: those of its region, or of a full block table.
int64_t paged_rows(const ra_config& c) {
  const int64_t held = c.budget_mode == RA_BUDGET_TOTAL
                           ? static_cast<int64_t>(c.budget_k)
                           : static_cast<int64_t>(c.max_prompt_len) + c.budget_k;
  return ra::host::round_up(held + c.recent_r + c.evict_every, c.page_rows);
}

size_t stats_floats(const ra_config& c) {
  return static_cast<size_t>(
      ra::host::round_up(static_cast<int64_t>(c.max_seqs) * c.num_q_heads * 2, 64));
}

// The split partials, then the queries' statistics, then the scores.
size_t weighed_bytes(const ra_config& c, int64_t rows) {
  return (ra_workspace_bytes(&c) + 255) / 256 * 256 +
         (stats_floats(c) + static_cast<size_t>(c.max_seqs) * c.num_q_heads * rows) * sizeof(float);
}

// Quarter turns per position of every pair (at most 2 / pi: base > 1, factor >= 1), or an error.
ra_status rotary_turns(const ra_rotary* p, ra::RotaryLaunch& out) {
  if (!p || p->dims < 2 || p->dims > ra::kHeadDim || p->dims % 2 != 0 ||
      !(std::isfinite(p->base) && p->base > 1.0) ||
      (p->pairs != RA_PAIRS_HALVES && p->pairs != RA_PAIRS_ADJACENT) ||
      p->scaling < RA_ROTARY_PLAIN || p->scaling > RA_ROTARY_CHANNELS ||
      !std::isfinite(p->magnitude) || p->magnitude < 0.0)
    return RA_ERR_INVALID_ARG;
  if (p->scaling != RA_ROTARY_PLAIN && !(std::isfinite(p->factor) && p->factor >= 1.0))
    return RA_ERR_INVALID_ARG;
  const bool bands = p->scaling == RA_ROTARY_ROTATIONS || p->scaling == RA_ROTARY_CHANNELS;
  if (bands && !(p->original_len > 0 && std::isfinite(p->high) && p->low > 0.0 && p->high > p->low))
    return RA_ERR_INVALID_ARG;
  const double pi2 = 6.283185307179586476925286766559;
  // the pair that makes `turns` turns over the original context
  const auto pair_of = [&](double turns) {
    return p->dims * std::log(p->original_len / (pi2 * turns)) / (2.0 * std::log(p->base));
  };
  double first = 0.0, last = 0.0;
  if (p->scaling == RA_ROTARY_CHANNELS) {
    first = std::max(std::floor(pair_of(p->high)), 0.0);
    last = std::min(std::ceil(pair_of(p->low)), p->dims - 1.0);
  }
  out.half = p->dims / 2;
  out.adjacent = p->pairs == RA_PAIRS_ADJACENT;
  out.magnitude = p->magnitude == 0.0 ? 1.f : static_cast<float>(p->magnitude);
  // base^(-2i / dims) as a product of two powers: 16 of them, not 64 (a microsecond a call)
  double high[8], low[8];
  for (int i = 0; i < 8; ++i) {
    high[i] = 8 * i < out.half ? std::pow(p->base, -16.0 * i / p->dims) : 0.0;
    low[i] = i < out.half ? std::pow(p->base, -2.0 * i / p->dims) : 0.0;
  }
  for (int i = 0; i < ra::kHeadDim / 2; ++i) {
    const double f = high[i / 8] * low[i % 8];
    double own = 1.0;    // share of the pair's own frequency, the rest divided by factor
    if (p->scaling == RA_ROTARY_LINEAR) {
      own = 0.0;
    } else if (p->scaling == RA_ROTARY_ROTATIONS) {
      own = (p->original_len * f / pi2 - p->low) / (p->high - p->low);
    } else if (p->scaling == RA_ROTARY_CHANNELS) {
      own = 1.0 - (i - first) / std::max(last - first, 0.001);
    }
    own = std::min(1.0, std::max(0.0, own));
    const double scaled = p->scaling == RA_ROTARY_PLAIN ? f : f * (own + (1.0 - own) / p->factor);
    out.quarters[i] = i < out.half ? scaled / (pi2 / 4) : 0.0;
  }
  return RA_OK;
}

// plan_blocks, but for two kinds of launches (microseconds per layer in a captured step,
// plan_blocks and this):
//   few fp32 rows, twice as long as those it was measured with: 64 keys to a workgroup up to
//     1,300 keys, for up to 16 heads 160 beyond, while there is a CU for each, and no more than
//     512 (2 heads of 200 rows 13.3 and 10.5, of 500 15.0 and 11.9, of 5,000 25.6 and 21.8; 8
//     heads of 600 17.4 and 13.8, of 1,200 18.5 and 16.4, of 2,200 19.6 and 18.2, with 64 keys
//     26.5, of 5,000 26.1 and 22.0, of 9,000 35.0 and 30.3; but 64 heads of 600, 640 workgroups,
//     20.4 and 35.3, 32 of 1,000 19.6 and, with 128 keys, 30.3);
//   129 to 256 ragged heads, of which it makes one item each: six, so that the CUs of the short
//     ones share the long ones' work (bf16, 160 heads of 300 to 9,000 rows 199 and 95, 256 of
//     them 217 and 142, 192 of 4,500 to 9,000 226 and 148, of 200 to 3,000 69 and 43; e4m3, 192
//     of 300 to 9,000 100 and 55, of 200 to 3,000 42 and 29; four items within 15% of it).
Plan biased_plan(const ra_cache* c, int64_t keys_max, int64_t keys_mean, int heads) {
  Plan p = ra::host::plan_blocks(c, keys_max, heads);
  if (c->cfg.attn_split > 0) return p;
  const auto items = [&](int64_t keys) { return (keys_max + keys - 1) / keys; };
  int64_t keys = p.split_keys;
  if (c->cfg.dtype == RA_F32 && keys_max <= 1300 && items(64) * heads <= 256)
    keys = 64;
  else if (c->cfg.dtype == RA_F32 && heads <= 16 && items(160) * heads <= 256 &&
           items(160) <= ra::kMaxSplits)
    keys = 160;
  else if (c->cfg.dtype == RA_F32 && items(512) * heads <= 256 && items(512) <= ra::kMaxSplits)
    keys = std::min<int64_t>(keys, 512);
  else if (heads > 128 && heads <= 256 && keys_max >= 1536 && 8 * keys_mean < 7 * keys_max)
    keys = ra::host::round_up((keys_max + 5) / 6, ra::kBlockRows);
  p.split_keys = static_cast<int>(keys);
  p.max_splits = p.partials = static_cast<int>(items(keys));
  return p;
}

}  // namespace

extern "C" {

ra_status ra_rotate_step(const ra_cache* c, const ra_rotary* rotary, const void* q,
                         const void* k_new, void* q_out, void* k_out, void* stream) {
  if (!c || (!q && !k_new) || (q && !q_out) || (k_new && !k_out) || misaligned(q) ||
      misaligned(k_new) || misaligned(q_out) || misaligned(k_out))
    return RA_ERR_INVALID_ARG;
  ra::RotaryLaunch r;
  const ra_status st = rotary_turns(rotary, r);
  if (st != RA_OK) return st;
  if (c->slot_hi <= c->slot_lo) return RA_OK;
  RA_LAUNCH(ra::launch_rotate_step(c->meta, c->slot_hi, c->cfg.dtype, c->cfg.num_q_heads,
                                   c->cfg.num_kv_heads, r, q, k_new, q_out, k_out,
                                   static_cast<hipStream_t>(stream)));
  return RA_OK;
}

ra_status ra_rotate_rows(const ra_rotary* rotary, int32_t dtype, const void* x, void* out,
                         int64_t heads, int32_t rows, int32_t first_position,
                         const int32_t* dev_positions, void* stream) {
  if ((dtype != RA_F32 && dtype != RA_BF16) || heads < 0 || rows < 0 ||
      heads > (int64_t(1) << 31) || misaligned(x) || misaligned(out) ||
      (!dev_positions &&
       (first_position < 0 || static_cast<int64_t>(first_position) + rows - 1 > INT32_MAX)))
    return RA_ERR_INVALID_ARG;
  ra::RotaryLaunch r;
  const ra_status st = rotary_turns(rotary, r);
  if (st != RA_OK) return st;
  if (heads == 0 || rows == 0) return RA_OK;
  if (!x || !out) return RA_ERR_INVALID_ARG;
  RA_LAUNCH(ra::launch_rotate_rows(dtype, r, x, out, heads, rows, first_position, dev_positions,
                                   static_cast<hipStream_t>(stream)));
  return RA_OK;
}

ra_status ra_biased_attention(ra_cache* c, int32_t layer, const ra_score_rule* rule, const void* q,
                              const void* k_new, const void* v_new, void* out, void* workspace,
                              size_t workspace_bytes, void* stream) {
  // (factors whose quotients and products are normal numbers)
  const auto usable = [](float x) { return x == 0.f || (x >= 0x1p-40f && x <= 0x1p40f); };
  if (!rule || !usable(rule->scale) || !usable(rule->cap) || rule->window < 0 || rule->prefix < 0)
    return RA_ERR_INVALID_ARG;
  const ra_status st = ra::host::check_decode(c, layer, q, k_new, v_new, out);
  if (st != RA_OK) return st;
  // the longest step's blocks; in graph mode those of any step to come
  const bool ordered = c->cfg.layout != RA_LAYOUT_HOLE_FILL;
  const int window = ordered ? rule->window : 0;
  int most = 0, n_active = 0;
  int64_t blocks_all = 0;
  int64_t score_rows = c->is_paged() ? paged_rows(c->cfg) : ra::kRegionAlign;
  for (int s = c->slot_lo; s < c->slot_hi; ++s) {
    const SeqMeta& M = c->mirror[s];
    if (!M.active) continue;
    ++n_active;
    if (!c->is_paged()) score_rows = std::max<int64_t>(score_rows, M.cap);
    int64_t blocks = ra::window_blocks(M.len, window, rule->prefix).n;
    if (c->graph) {
      blocks = M.cap / ra::kBlockRows;
      if (window > 0)
        blocks = std::min<int64_t>(
            blocks, int64_t(window) / ra::kBlockRows + 2 + rule->prefix / ra::kBlockRows + 1);
    }
    most = std::max(most, static_cast<int>(blocks));
    blocks_all += blocks;
  }
  if (c->weights && score_rows > ra::kMaxScoreRows) return RA_ERR_UNSUPPORTED;
  const size_t need =
      c->weights ? weighed_bytes(c->cfg, score_rows) : ra_workspace_bytes(&c->cfg);
  if (!workspace || workspace_bytes < need || misaligned(workspace)) return RA_ERR_INVALID_ARG;
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  // the rows of deferred events move first, as this attention moves none: every layer's at
  // once, or where layers of this step have moved theirs (each while it attended) this one's
  if (c->n_appended == 0) {
    const ra_status fl = ra::host::flush_pending(c, hs);
    if (fl != RA_OK) return fl;
  } else if (c->any_pending()) {
    RA_LAUNCH(ra::launch_flush_layer(c->shape(), c->meta, c->kpool, c->vpool, c->drops,
                                     c->cfg.evict_every, layer, c->slot_lo, c->slot_hi, hs));
  }
  const ra_status grown = ra::host::grow_for_step(c, hs);
  if (grown != RA_OK) return grown;
  ra::Shape sh = c->shape();
  if (!c->graph) sh.order = c->refresh_order();
  c->appended[layer] = 1;
  ++c->n_appended;
  c->biased_step = true;
  if (n_active == 0) return RA_OK;
  const Plan plan =
      biased_plan(c, int64_t(most) * ra::kBlockRows, blocks_all * ra::kBlockRows / n_active,
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
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = a.ws_o + items * c->G * ra::kHeadDim;
  a.split_stride = ra::kMaxSplits;
  a.layer = layer;
  a.max_seqs = c->slot_hi;
  a.split_keys = plan.launch_keys();
  a.max_splits = plan.launch_splits();
  a.waves = plan.launch_waves();
  a.arrivals = c->arrivals;
  ra::BiasLaunch b;
  b.scale = rule->scale == 0.f ? 1.0 / std::sqrt(double(ra::kHeadDim)) : rule->scale;
  b.cap = rule->cap;
  b.slopes = rule->dev_slopes;
  b.window = rule->window;
  b.prefix = rule->prefix;
  b.ordered = ordered;
  b.rows = static_cast<int>(std::min<int64_t>(int64_t(most) * ra::kBlockRows, INT32_MAX));
  b.heads = n_active * c->cfg.num_kv_heads;
  ra::score_units(b);
  if (c->weights) {
    b.weights = c->weights;
    b.stats = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                       (ra_workspace_bytes(&c->cfg) + 255) / 256 * 256);
    b.scores = b.stats + stats_floats(c->cfg);
    b.score_stride = score_rows;
  }
  const hipError_t e = ra::launch_biased_attention(sh, a, b, hs);
  if (e != hipSuccess) {
    c->appended[layer] = 0;
    --c->n_appended;
    return ra::host::hip_fail(e);
  }
  return RA_OK;
}

size_t ra_weights_bytes(const ra_config* c, int64_t pool_rows) {
  if (ra_config_check(c) != RA_OK || !weights_supported(*c) || pool_rows <= 0 ||
      pool_rows % ra::kRegionAlign != 0 || pool_rows > (int64_t(1) << 40))
    return 0;
  return static_cast<size_t>(pool_rows) * sizeof(float);
}

size_t ra_weights_workspace_bytes(const ra_config* c, int32_t max_prompt_len) {
  if (ra_config_check(c) != RA_OK || !weights_supported(*c) || max_prompt_len < 0) return 0;
  const int64_t rows =
      c->layout == RA_LAYOUT_PAGED ? paged_rows(*c) : ra_region_rows(c, max_prompt_len);
  return rows < 0 ? 0 : weighed_bytes(*c, std::max<int64_t>(rows, ra::kRegionAlign));
}

ra_status ra_weights_attach(ra_cache* c, float* dev_weights, size_t weights_bytes) {
  if (!c) return RA_ERR_INVALID_ARG;
  if (!weights_supported(c->cfg)) return RA_ERR_UNSUPPORTED;
  if (dev_weights && (weights_bytes < ra_weights_bytes(&c->cfg, c->pool_rows) ||
                      misaligned(dev_weights)))
    return RA_ERR_INVALID_ARG;
  if (c->graph || c->step_open() || c->slot_hi > c->slot_lo) return RA_ERR_STATE;
  c->weights = dev_weights;
  c->weight_hooks = dev_weights ? &kWeightHooks : nullptr;
  return RA_OK;
}

// A slot whose weights or positions may be read or written now.
static ra_status check_weighed(const ra_cache* c, int32_t seq) {
  if (!c || seq < 0 || seq >= c->cfg.max_seqs) return RA_ERR_INVALID_ARG;
  if (!c->weights || c->graph || c->step_open() || !c->mirror[seq].active) return RA_ERR_STATE;
  return RA_OK;
}

ra_status ra_write_weights(ra_cache* c, int32_t seq, const float* dev_weights, void* stream) {
  const ra_status st = check_weighed(c, seq);
  if (st != RA_OK) return st;
  const SeqMeta& M = c->mirror[seq];
  if (!dev_weights && M.len > 0) return RA_ERR_INVALID_ARG;   // NULL only if empty
  RA_LAUNCH(ra::launch_set_weights(c->shape(), M, seq, 0, M.len, dev_weights, c->weights,
                                   static_cast<hipStream_t>(stream)));
  return RA_OK;
}

ra_status ra_export_weights(ra_cache* c, int32_t seq, float* dev_out, int64_t out_elems,
                            void* stream) {
  const ra_status st = check_weighed(c, seq);
  if (st != RA_OK) return st;
  const SeqMeta& M = c->mirror[seq];
  if (!dev_out && M.len > 0) return RA_ERR_INVALID_ARG;   // nothing to copy: may be NULL
  if (out_elems < static_cast<int64_t>(M.len) * c->cfg.num_layers * c->cfg.num_kv_heads)
    return RA_ERR_CAPACITY;
  RA_LAUNCH(ra::launch_export_weights(c->shape(), M, seq, M.len, c->weights, dev_out,
                                      static_cast<hipStream_t>(stream)));
  return RA_OK;
}

ra_status ra_write_positions(ra_cache* c, int32_t seq, const int32_t* dev_positions, void* stream) {
  const ra_status st = check_weighed(c, seq);
  if (st != RA_OK) return st;
  const SeqMeta& M = c->mirror[seq];
  if (!dev_positions && M.len > 0) return RA_ERR_INVALID_ARG;   // NULL only if empty
  RA_LAUNCH(ra::launch_write_rows(c->shape(), M, seq, M.len, nullptr, nullptr, dev_positions,
                                  c->kpool, c->vpool, c->pos, static_cast<hipStream_t>(stream)));
  return RA_OK;
}

}  // extern "C"
