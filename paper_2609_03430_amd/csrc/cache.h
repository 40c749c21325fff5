// The host side of a cache, shared by the sources of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <map>
#include <vector>

#include "ra_internal.h"
#include "randattn.h"

namespace ra {
namespace host {

// Records a failed HIP call for ra_last_hip_error.
ra_status hip_fail(hipError_t e);

#define RA_LAUNCH(expr)                                   \
  do {                                                    \
    const hipError_t e_ = (expr);                         \
    if (e_ != hipSuccess) return ra::host::hip_fail(e_);  \
  } while (0)

inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Attention launch plan (plan_for): work items of split_keys keys, `waves`
// wavefronts each; group_waves > 0: items of one wavefront, group_waves
// consecutive items of a head to a workgroup.
struct Plan {
  int split_keys = 0, max_splits = 0, waves = 1, wide_regs = 0;
  int group_waves = 0;
  int short_runs = 0;   // every item is at most 64 keys: the latency build
  // an event of every sequence may leave its row moves to the next step's
  // attention, one workgroup per head (attn_bf16_move_kernel)
  bool whole = false;
  // partial slots per head that the no-alloc entry point's limit counts (at
  // least the workgroups of a head)
  int partials = 0;

  int launch_waves() const { return group_waves ? group_waves : waves; }
  int launch_keys() const { return group_waves ? group_waves * split_keys : split_keys; }
  int launch_splits() const {
    return group_waves ? (max_splits + group_waves - 1) / group_waves : max_splits;
  }
};

// Launch plan of attention over blocks of rows.
Plan plan_blocks(const ra_cache* c, int64_t keys_max, int heads);

// Host checks shared by the attention entry points; nothing is launched.
ra_status check_decode(const ra_cache* c, int32_t layer, const void* q, const void* k_new,
                       const void* v_new, const void* out);
// Paged layout: pages for the rows this step appends (the first layer of the step).
// RA_ERR_CAPACITY, nothing changed, if the host has no memory for their entries.
ra_status grow_for_step(ra_cache* c, hipStream_t s);
// Moves the key/value rows of every sequence whose last event deferred them (their
// positions are already compacted); a call that reads or writes rows, or plans
// another event, runs this first.
ra_status flush_pending(ra_cache* c, hipStream_t s);

}  // namespace host
}  // namespace ra

struct ra_cache {
  ra_config cfg{};
  int G = 0;
  size_t elem = 0;
  void* kpool = nullptr;
  void* vpool = nullptr;
  int32_t* pos = nullptr;
  int64_t pool_rows = 0;
  ra::SeqMeta* meta = nullptr;
  std::vector<ra::SeqMeta> mirror;       // host copy of the device metadata
  std::map<int64_t, int64_t> free_rows;  // first-fit free list: base -> rows
  std::vector<uint8_t> appended;         // layers appended in the open step
  int n_appended = 0;
  int slot_lo = 0, slot_hi = 0;          // range covering the active slots
  // paged layout
  ra::Paging pg{};                       // device tables and page geometry
  int page_rows = 0;
  int64_t n_groups = 0;                  // page groups in the pool
  std::vector<int32_t> free_groups;      // stack: the next group is back()
  std::vector<std::vector<int32_t>> groups;   // per slot: its table, in order
  // deferred row moves (see ra_end_step)
  int32_t* drops = nullptr;              // drop lists of the last events
  int32_t* arrivals = nullptr;           // split arrival counters, event sync words
  // graph mode (see ra_graph_mode): launches that depend on no host state
  bool graph = false;
  ra::host::Plan graph_plan;
  int graph_candidates = 0;              // bound on any event's candidate slots
  void* scratch = nullptr;               // device address of the no-alloc partials

  // block-sparse attention (ra_sparse_attach): the bounds of the blocks' keys, and
  // per layer and slot how many leading blocks of a head they are current for
  int8_t* bounds = nullptr;
  std::vector<int32_t> bounds_built;
  std::vector<uint8_t> sparse_layers;    // layers that sparse steps were made of
  std::vector<ra::BoundsRange> ranges;   // a step's own, room for every slot and layer
  std::vector<int> stale_layers;         //   set aside when bounds are attached

  // accumulated attention weights (ra_weights_attach): a float per pool row
  float* weights = nullptr;
  const ra::WeightHooks* weight_hooks = nullptr;
  bool biased_step = false;              // the last attention launch carries no row moves

  ra::Shape shape() const {
    ra::Shape sh{cfg.num_layers, cfg.num_q_heads, cfg.num_kv_heads, G,
                 cfg.recent_r, cfg.evict_every, cfg.dtype, cfg.layout,
                 cfg.policy, std::max(1, cfg.policy_block), pg};
    if (cfg.dtype == RA_E4M3) {
      sh.k_scale = static_cast<uint8_t*>(kpool) + pool_rows * ra::kHeadDim;
      sh.v_scale = static_cast<uint8_t*>(vpool) + pool_rows * ra::kHeadDim;
    }
    return sh;
  }
  // attention over blocks: the active slots, the longest first (see refresh_order)
  ra::SlotOrder order;
  bool order_stale = true;               // the active slots changed
  bool order_sorted = false;             // sorted by the lengths of this step

  // Brings `order` up to date, at the first launch of a step that asks for it (not
  // the first layer: launches that take no order may come before), and returns it where
  // the caches are ragged: heads that start last should be short (microseconds per step,
  // slots as they come and the longest first: 1,280 heads of 1,000 to 9,000 e4m3 rows 338
  // and 299, 480 paged ones of 300 to 4,100 76 and 68).  Lengths hardly change their
  // order between steps, so an insertion sort goes over them once.
  const ra::SlotOrder* refresh_order() {
    if (n_appended == 0 || order_stale || !order_sorted) {
      if (order_stale) {
        order.n = 0;
        int active = 0;
        for (int s = slot_lo; s < slot_hi; ++s) {
          if (!mirror[s].active) continue;
          if (++active <= ra::kOrderMax) order.slot[order.n++] = static_cast<uint16_t>(s);
        }
        if (active > ra::kOrderMax) order.n = 0;   // too many for a launch's arguments
        order_stale = false;
      }
      for (int i = 1; i < order.n; ++i) {
        const uint16_t s = order.slot[i];
        int j = i;
        for (; j > 0 && mirror[order.slot[j - 1]].len < mirror[s].len; --j)
          order.slot[j] = order.slot[j - 1];
        order.slot[j] = s;
      }
      order_sorted = true;
    }
    if (order.n < 2) return nullptr;
    const int longest = mirror[order.slot[0]].len, shortest = mirror[order.slot[order.n - 1]].len;
    return 8 * (longest - shortest) > longest ? &order : nullptr;
  }
  // Rows of slot `s` from row `from` on change: their blocks' bounds are stale.
  void rows_change(int s, int from) {
    if (!bounds) return;
    for (int l = 0; l < cfg.num_layers; ++l) {
      int32_t& n = bounds_built[static_cast<size_t>(l) * cfg.max_seqs + s];
      n = std::min(n, from / ra::kBlockRows);
    }
  }
  bool is_paged() const { return cfg.layout == RA_LAYOUT_PAGED; }
  bool any_pending() const {
    for (int s = slot_lo; s < slot_hi; ++s)
      if (mirror[s].active && mirror[s].due == ra::kDueMovePending) return true;
    return false;
  }
  int64_t pages_for(int64_t rows) const { return (rows + page_rows - 1) / page_rows; }
  // paged: whether `rows` rows fit the block table of one sequence (rows
  // pile up past lp + k_keep + r + R only under the external policy)
  bool fits_table(int64_t rows) const { return pages_for(rows) <= pg.pages_per_seq; }
  // paged: page groups slot `s` must add to hold `rows` rows
  int64_t groups_short(int s, int64_t rows) const {
    return std::max<int64_t>(0, pages_for(rows) - static_cast<int64_t>(groups[s].size()));
  }
  // paged: take groups from the free list until slot `s` holds `rows` rows;
  // the new table entries are appended to `out` (the caller checked that
  // enough groups are free)
  void grow(int s, int64_t rows, std::vector<ra::TableEntry>& out) {
    while (static_cast<int64_t>(groups[s].size()) < pages_for(rows)) {
      const int32_t g = free_groups.back();
      free_groups.pop_back();
      out.push_back(ra::TableEntry{s, static_cast<int32_t>(groups[s].size()), g});
      groups[s].push_back(g);
    }
    mirror[s].cap = static_cast<int32_t>(groups[s].size()) * page_rows;
  }
  // paged: return the groups past the first pages_for(rows) to the free list
  void shrink(int s, int64_t rows) {
    while (static_cast<int64_t>(groups[s].size()) > pages_for(rows)) {
      free_groups.push_back(groups[s].back());
      groups[s].pop_back();
    }
    mirror[s].cap = static_cast<int32_t>(groups[s].size()) * page_rows;
  }
  bool step_open() const { return n_appended != 0; }
  void update_range() {
    order_stale = true;
    slot_lo = 0;
    slot_hi = 0;
    bool any = false;
    for (int s = 0; s < cfg.max_seqs; ++s) {
      if (!mirror[s].active) continue;
      if (!any) slot_lo = s;
      slot_hi = s + 1;
      any = true;
    }
  }
  // slots the selection examines per head (see evict.hip)
  int span(const ra::SeqMeta& M) const {
    return M.plan_len - M.prompt_len - (cfg.layout == RA_LAYOUT_HOLE_FILL ? 0 : cfg.recent_r);
  }
  int max_candidates_due() const {
    int mx = 0;
    for (int s = slot_lo; s < slot_hi; ++s)
      if (mirror[s].active && mirror[s].due) mx = std::max(mx, span(mirror[s]));
    return mx;
  }
};
