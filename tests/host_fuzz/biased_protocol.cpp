// Random calls on a cache whose steps go through ra_biased_attention, mixed with plain ones,
// with and without accumulated weights (test infrastructure): api.cpp and api_biased.cpp with
// the stand-ins of stub_launchers.cpp and, here, of the launches that api_biased.cpp makes.
//
// Checked, against the slot records as the device would hold them (in graph mode the mirror
// stands still while they advance): a launch's items cover every block that a head may attend
// to, within the partials' slots; partials, statistics and scores fit the workspace given, and
// a head's attended rows its scores; deferred row moves of a layer run once, before or in its
// attention; with weights attached every row gets a weight when it comes to be (a prompt's, a
// fast forward's), events go by weight, and nothing else compacts rows.
//
// Usage: biased_protocol SEED DTYPE LAYOUT WEIGHTS OPS
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include <hip/hip_runtime.h>

#include "ra_internal.h"
#include "randattn.h"

extern "C" void stub_configure(int64_t pool_rows, int64_t n_groups, int max_seqs, int page_rows);

namespace {

constexpr int L = 3, Hkv = 2, G = 3, kSlots = 3;
ra_cache* g_cache = nullptr;
char* g_ws = nullptr;
size_t g_ws_bytes = 0;
float* g_weights = nullptr;
int g_attends = 0, g_events = 0, g_flushed = 0;
int g_weighed_rows[kSlots];             // rows that have a weight, at least

[[noreturn]] void fail(const char* what, long long a, long long b) {
  std::fprintf(stderr, "check failed: %s (%lld, %lld)\n", what, a, b);
  std::abort();
}

}  // namespace

namespace ra {

hipError_t launch_biased_attention(const Shape& sh, const AttnLaunch& a, const BiasLaunch& b,
                                   hipStream_t) {
  if (a.max_splits < 1 || a.max_splits > kMaxSplits || a.split_keys < kBlockRows ||
      a.split_keys % kBlockRows != 0 || a.split_stride < a.max_splits)
    fail("plan", a.max_splits, a.split_keys);
  if (b.ordered != (sh.layout != 1)) fail("order", b.ordered, sh.layout);
  for (int s = 0; s < kSlots; ++s) {
    const SeqMeta& M = a.meta[s];
    if (!M.active) continue;
    if (s >= a.max_seqs) fail("slot beyond the launch", s, a.max_seqs);
    if (M.len + 1 > M.cap && sh.layout != 2) fail("append past the region", M.len, M.cap);
    const WindowBlocks w = window_blocks(M.len, b.ordered ? b.window : 0, b.prefix);
    if (static_cast<int64_t>(a.max_splits) * a.split_keys < int64_t(w.n) * kBlockRows)
      fail("blocks past the splits", w.n, a.max_splits * a.split_keys);
    // blocks that may hold a row in sight are all among the attended ones
    const int last = M.len / kBlockRows;
    if ((w.n - 1 < w.head ? w.n - 1 : w.n - 1 + w.shift) != last) fail("the new row's block", w.n, last);
    for (int j = 0; b.ordered && b.window > 0 && j <= M.len; ++j) {
      if (M.len - j >= b.window && j >= b.prefix) continue;
      const int blk = j / kBlockRows;
      if (blk >= w.head && blk < w.head + w.shift) fail("a row in sight left out", j, M.len);
    }
    if (b.weights) {
      if (b.weights != g_weights) fail("weights", 0, 0);
      if (int64_t(w.n) * kBlockRows > b.score_stride) fail("scores", w.n, b.score_stride);
      if (g_weighed_rows[s] < M.len) fail("rows without a weight", g_weighed_rows[s], M.len);
      if (a.layer == L - 1) g_weighed_rows[s] = M.len + 1;
    }
  }
  const char* end = reinterpret_cast<const char*>(
      b.weights ? b.scores + int64_t(kSlots) * sh.Hq * b.score_stride
                : a.ws_ml + int64_t(kSlots) * sh.Hkv * kMaxSplits * sh.G * 2);
  if (reinterpret_cast<const char*>(a.ws_o) < g_ws || end > g_ws + g_ws_bytes)
    fail("workspace", end - g_ws, g_ws_bytes);
  if (b.weights) {
    if (reinterpret_cast<const char*>(b.stats) <
            reinterpret_cast<const char*>(a.ws_ml + int64_t(kSlots) * sh.Hkv * kMaxSplits * sh.G * 2) ||
        b.stats + 2 * kSlots * sh.Hq > b.scores || reinterpret_cast<uintptr_t>(b.scores) % 16)
      fail("statistics", 0, 0);
  }
  ++g_attends;
  return hipSuccess;
}

hipError_t launch_weight_event(const Shape& sh, const SeqMeta* meta, void*, void*, int32_t*,
                               float* weights, int slot_lo, int slot_hi, int max_candidates, bool,
                               hipStream_t) {
  if (weights != g_weights) fail("event's weights", 0, 0);
  for (int s = slot_lo; s < slot_hi; ++s) {
    const SeqMeta& M = meta[s];
    if (!M.active || !M.due) continue;
    const int cand = M.plan_len - M.prompt_len - sh.r;
    if (cand > max_candidates || max_candidates > kMaxCandidates) fail("candidates", cand, max_candidates);
    if (M.plan_len - M.len > kMaxEvery) fail("drops", M.plan_len, M.len);
    ++g_events;
  }
  return hipSuccess;
}

hipError_t launch_set_weights(const Shape& sh, const SeqMeta& M, int slot, int from, int to,
                              const float*, float* weights, hipStream_t) {
  if (weights != g_weights || from < 0 || from > to) fail("set weights", from, to);
  if (to > M.cap && sh.layout != 2) fail("weights past the region", to, M.cap);
  if (from > g_weighed_rows[slot] && from > 0) fail("a gap before the weights", from, g_weighed_rows[slot]);
  g_weighed_rows[slot] = to;
  return hipSuccess;
}

hipError_t launch_export_weights(const Shape&, const SeqMeta& M, int slot, int len, const float*,
                                 float*, hipStream_t) {
  if (len != M.len || g_weighed_rows[slot] < len) fail("export", len, M.len);
  return hipSuccess;
}

hipError_t launch_flush_layer(const Shape& sh, const SeqMeta*, void*, void*, const int32_t* drops,
                              int stride, int layer, int lo, int hi, hipStream_t) {
  if (sh.dtype != 1 || sh.layout != 0 || !drops || stride != sh.every || layer < 1 || layer >= L ||
      lo < 0 || hi > kSlots)
    fail("flush of a layer", layer, stride);
  ++g_flushed;
  return hipSuccess;
}

hipError_t launch_rotate_step(const SeqMeta*, int max_seqs, int, int, int, const RotaryLaunch& r,
                              const void*, const void*, void*, void*, hipStream_t) {
  if (max_seqs < 1 || max_seqs > kSlots || r.half < 1 || r.half > 64) fail("rotate", max_seqs, r.half);
  for (int i = 0; i < r.half; ++i)
    if (!(r.quarters[i] > 0.0 && r.quarters[i] < 0.64)) fail("turns", i, r.half);
  return hipSuccess;
}

hipError_t launch_rotate_rows(int, const RotaryLaunch&, const void*, void*, int64_t, int, int,
                              const int32_t*, hipStream_t) {
  return hipSuccess;
}

}  // namespace ra

int main(int argc, char** argv) {
  if (argc != 6) return 2;
  std::mt19937 rng(std::atoi(argv[1]));
  const auto pick = [&](int n) { return static_cast<int>(rng() % static_cast<unsigned>(n)); };
  const bool weighed = std::atoi(argv[4]) != 0;
  ra_config c{};
  c.num_layers = L;
  c.num_q_heads = G * Hkv;
  c.num_kv_heads = Hkv;
  c.head_dim = 128;
  c.budget_k = pick(2) ? 60 + pick(200) : 3000 + pick(3000);
  c.recent_r = pick(40);
  c.evict_every = 1 + pick(30);
  c.dtype = std::atoi(argv[2]);
  c.layout = std::atoi(argv[3]);
  c.max_seqs = kSlots;
  // one slot, a head to a work item: events defer their row moves
  const bool alone = !weighed && c.dtype == RA_BF16 && pick(2) == 0;
  if (alone) c.budget_k = pick(60);
  c.attn_split = alone ? 8192 : pick(3) ? 0 : 32 * (1 + pick(40));
  c.policy_block = 1;
  c.page_rows = 32 << pick(3);
  c.max_prompt_len = 300;
  const int64_t group = static_cast<int64_t>(L) * Hkv * c.page_rows;
  const int64_t rows = (ra_seq_rows(&c, 300) * kSlots + group - 1) / group * group;
  stub_configure(rows, rows / group, kSlots, c.page_rows);
  alignas(16) static char pool[16];                  // the stand-ins touch no row
  alignas(16) static float weights[4];
  g_weights = weights;
  std::vector<int32_t> pos(rows + 16);
  std::vector<char> meta(ra_meta_bytes(&c) + 16);
  const auto aligned = [](char* p) { return p + (16 - reinterpret_cast<uintptr_t>(p) % 16) % 16; };
  g_ws_bytes = weighed ? ra_weights_workspace_bytes(&c, 300) : ra_workspace_bytes(&c);
  std::vector<char> ws(g_ws_bytes + 16);
  g_ws = aligned(ws.data());
  int32_t* p = reinterpret_cast<int32_t*>(aligned(reinterpret_cast<char*>(pos.data())));
  if (ra_cache_create(&c, pool, pool, p, rows, aligned(meta.data()), ra_meta_bytes(&c), nullptr,
                      &g_cache) != RA_OK)
    fail("create", 0, 0);
  if (weighed && ra_weights_attach(g_cache, weights, ra_weights_bytes(&c, rows)) != RA_OK)
    fail("attach", 0, 0);
  const size_t row = 128 * 4;
  std::vector<char> q(kSlots * G * Hkv * row + 16), kv(kSlots * Hkv * row + 16),
      many(static_cast<size_t>(L) * Hkv * 7000 * row);
  char* qa = aligned(q.data());
  char* ka = aligned(kv.data());
  bool graph = false, forwarded = false;
  int steps = 0, refused = 0, mixed = 0;
  const auto info_of = [&](int s) {
    ra_seq_info i;
    if (ra_get_seq_info(g_cache, s, &i) != RA_OK) fail("info", s, 0);
    return i;
  };
  for (int op = 0, ops = std::atoi(argv[5]); op < ops; ++op) {
    const int s = alone ? 0 : pick(kSlots);
    switch (alone && pick(4) ? 11 : pick(12)) {
      case 0:
        ra_seq_begin(g_cache, s, pick(301), 1, op, many.data(), many.data(), nullptr);
        break;
      case 1:
        if (pick(3) == 0) ra_seq_end(g_cache, s, nullptr);
        break;
      case 2:
        // (a fast forward leaves its events' flags to the next step, which the stand-in of
        // another slot's event would take for events it was not given)
        if (!forwarded) ra_evict_now(g_cache, s, nullptr);
        break;
      case 3:
        forwarded = true;
        ra_seq_fast_forward(g_cache, s, pick(4) ? pick(60) : pick(7000), nullptr);
        break;
      case 4: {
        const ra_status st = ra_write_weights(g_cache, s, weights, nullptr);
        const bool ok = weighed && !graph && info_of(s).active;
        if ((st == RA_OK) != ok) fail("write weights", st, ok);
        break;
      }
      case 5: {
        const ra_status st = ra_export_weights(g_cache, s, weights, int64_t(1) << 40, nullptr);
        const bool ok = weighed && !graph && info_of(s).active;
        if ((st == RA_OK) != ok) fail("export weights", st, ok);
        break;
      }
      case 6: {
        const bool on = pick(3) == 0;
        const ra_status st = ra_graph_mode(g_cache, on, nullptr);
        if (st == RA_OK) graph = on;
        else if (c.layout != RA_LAYOUT_PAGED) fail("graph mode", st, on);
        if (st == RA_OK && !on)
          for (int i = 0; i < kSlots; ++i)
            if (info_of(i).active) g_weighed_rows[i] = std::max(g_weighed_rows[i], info_of(i).len);
        break;
      }
      case 7: {
        ra_rotary r{};
        r.base = 2.0 + pick(100000);
        r.dims = 2 + 2 * pick(64);
        r.scaling = pick(4);
        r.factor = 1.0 + pick(30);
        r.low = 1.0;
        r.high = 1.5 + pick(30);
        r.original_len = 1 + pick(9000);
        if (ra_rotate_step(g_cache, &r, qa, ka, qa, ka, nullptr) != RA_OK) fail("rotate", op, 0);
        break;
      }
      default: {
        // a step; a refusal of its first layer (no room) leaves it unopened
        bool open = true;
        int kinds = 0;
        for (int l = 0; l < L && open; ++l) {
          ra_score_rule rule{};
          rule.window = pick(2) ? 0 : 1 + pick(pick(2) ? 100 : 7000);
          rule.prefix = pick(2) ? 0 : pick(300);
          rule.cap = pick(2) ? 0.f : 20.f;
          const bool plain = !weighed && pick(3) == 0;
          const bool pending = info_of(0).move_pending || info_of(1).move_pending ||
                               info_of(2).move_pending;
          const int before = g_flushed;
          kinds |= plain ? 1 : 2;
          const ra_status st =
              plain ? ra_decode_attention(g_cache, l, qa, ka, ka, qa, g_ws, g_ws_bytes, nullptr)
                    : ra_biased_attention(g_cache, l, &rule, qa, ka, ka, qa, g_ws, g_ws_bytes, nullptr);
          if (st == RA_OK) {
            if (!plain && pending && l > 0 && g_flushed != before + 1) fail("a layer's moves", l, op);
            if (!plain && l == 0 && (info_of(0).move_pending || info_of(1).move_pending ||
                                     info_of(2).move_pending))
              fail("moves left pending", op, 0);
            continue;
          }
          if (l > 0 || st != RA_ERR_CAPACITY) fail("step", st, l);
          open = false;
          ++refused;
        }
        if (!open) break;
        if (weighed && ra_export_weights(g_cache, s, weights, 1 << 30, nullptr) != RA_ERR_STATE &&
            info_of(s).active)
          fail("export inside a step", op, 0);
        if (ra_end_step(g_cache, nullptr, nullptr) != RA_OK) fail("end of a step", op, 0);
        ++steps;
        forwarded = false;
        mixed += kinds == 3;
        break;
      }
    }
  }
  ra_cache_destroy(g_cache);
  std::printf("{\"steps\": %d, \"attends\": %d, \"events\": %d, \"flushed\": %d, \"refused\": %d, "
              "\"mixed\": %d}\n", steps, g_attends, g_events, g_flushed, refused, mixed);
  return 0;
}
