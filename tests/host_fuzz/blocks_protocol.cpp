// Random calls on a cache whose steps mix dense and block-sparse attention (test
// infrastructure): api.cpp and api_blocks.cpp with the stand-ins of
// stub_launchers.cpp and, here, of the launches that api_blocks.cpp makes.
//
// Checked: whenever a sparse step chooses among the blocks of a head, the bounds of
// every candidate were computed from the rows that the head holds now (each change
// of a slot's rows starts a new version of the rows from where it may reach); bounds
// are only computed of whole blocks of cached rows; the lists, scores and partials
// fit the workspace; no launch follows a refusal.
//
// Usage: blocks_protocol SEED DTYPE LAYOUT OPS
#include <cstdio>
#include <cstdlib>
#include <new>
#include <random>
#include <vector>

#include <hip/hip_runtime.h>

#include "ra_internal.h"
#include "randattn.h"

extern "C" void stub_configure(int64_t pool_rows, int64_t n_groups, int max_seqs, int page_rows);

namespace {

constexpr int L = 2, Hkv = 2, kSlots = 3, kRowsMax = 4096;
int64_t g_version = 1;
int64_t g_rows[kSlots][kRowsMax];                  // version of each row of a slot
int64_t g_bounds[L][kSlots][kRowsMax / 32];        // version a block's bounds are of
ra_cache* g_cache = nullptr;
bool g_capturing = false, g_implicit = false, g_no_memory = false;
int g_hip_error = 0;                               // what hipGetLastError would report
int g_launches = 0, g_bounds_built = 0, g_checked = 0;
char* g_ws = nullptr;
size_t g_ws_bytes = 0;
int8_t* g_buf = nullptr;
size_t g_buf_bytes = 0;

[[noreturn]] void fail(const char* what, long long a, long long b) {
  std::fprintf(stderr, "check failed: %s (%lld, %lld)\n", what, a, b);
  std::abort();
}

ra_seq_info info_of(int s) {
  ra_seq_info i;
  if (ra_get_seq_info(g_cache, s, &i) != RA_OK) fail("info", s, 0);
  return i;
}

void rows_change(int s, int from) {
  ++g_version;
  for (int r = from; r < kRowsMax; ++r) g_rows[s][r] = g_version;
}

void check_candidates(int layer, int recent, int n_blocks) {
  for (int s = 0; n_blocks > 0 && s < kSlots; ++s) {
    const ra_seq_info i = info_of(s);
    if (!i.active) continue;
    const int cand = ra::candidate_blocks(i.len, recent);
    if (cand <= n_blocks) continue;
    for (int b = 0; b < cand; ++b) {
      ++g_checked;
      for (int r = 32 * b; r < 32 * b + 32; ++r)
        if (g_rows[s][r] > g_bounds[layer][s][b]) fail("stale bounds", s, b);
    }
  }
}

}  // namespace

// host memory that runs out while g_no_memory is set
void* operator new(size_t n) {
  void* p = g_no_memory ? nullptr : std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void* operator new(size_t n, const std::nothrow_t&) noexcept { return std::malloc(n ? n : 1); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

extern "C" hipError_t hipGetLastError() {
  const int e = g_hip_error;
  g_hip_error = 0;
  return static_cast<hipError_t>(e);
}

extern "C" hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* out) {
  if (g_implicit) {                                  // another stream is captured
    g_hip_error = hipErrorStreamCaptureImplicit;
    return hipErrorStreamCaptureImplicit;
  }
  *out = g_capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}

namespace ra {

hipError_t launch_export_rows(const Shape&, const SeqMeta&, int, int, const void*, const void*,
                              void*, void*, hipStream_t) {
  ++g_launches;
  return hipSuccess;
}

hipError_t launch_block_bounds(const Shape&, const SeqMeta*, const void*, int8_t* bounds,
                               int64_t pool_rows, const int* layers, int n_layers,
                               const BoundsRange* r, int n, hipStream_t) {
  ++g_launches;
  if (n_layers < 1 || n < 1) fail("empty launch", n_layers, n);
  if (bounds != g_buf || pool_rows / 32 * (kBoundsBytes + 1) > static_cast<int64_t>(g_buf_bytes))
    fail("bounds buffer", pool_rows, static_cast<long long>(g_buf_bytes));
  for (int i = 0; i < n; ++i) {
    const ra_seq_info s = info_of(r[i].slot);
    if (!s.active || r[i].from >= r[i].to || r[i].from < 0 || 32 * r[i].to > s.len)
      fail("range", r[i].from, r[i].to);
    for (int l = 0; l < n_layers; ++l) {
      if (layers[l] < 0 || layers[l] >= L) fail("layer", layers[l], L);
      for (int b = r[i].from; b < r[i].to; ++b, ++g_bounds_built)
        g_bounds[layers[l]][r[i].slot][b] = g_version;
    }
  }
  return hipSuccess;
}

hipError_t launch_choose_blocks(const Shape&, const SeqMeta*, const void*, int layer, int max_seqs,
                                const BlockChoice& ch, uint32_t* scores, int stride, int*,
                                int max_candidates, hipStream_t) {
  ++g_launches;
  check_candidates(layer, ch.recent, ch.n_blocks);
  if (max_candidates > stride) fail("scores", max_candidates, stride);
  if (reinterpret_cast<char*>(scores + static_cast<size_t>(max_seqs) * Hkv * stride) >
      g_ws + g_ws_bytes)
    fail("scores past the workspace", max_seqs, stride);
  return hipSuccess;
}

hipError_t launch_block_attention(const Shape& sh, const AttnLaunch& a, const BlockChoice& ch,
                                  hipStream_t) {
  ++g_launches;
  check_candidates(a.layer, ch.recent, ch.n_blocks);
  if (ch.bounds != g_buf) fail("bounds", 0, 0);
  const size_t heads = static_cast<size_t>(a.max_seqs) * sh.Hkv;
  if (reinterpret_cast<char*>(ch.list + heads * ch.stride) > reinterpret_cast<char*>(a.ws_o) ||
      reinterpret_cast<char*>(a.ws_ml + heads * a.split_stride * sh.G * 2) > g_ws + g_ws_bytes)
    fail("workspace", static_cast<long long>(heads), ch.stride);
  if (a.max_splits > a.split_stride || a.split_keys % 32) fail("splits", a.max_splits, a.split_keys);
  for (int s = 0; s < kSlots; ++s) {
    const ra_seq_info i = info_of(s);
    if (i.active && ra::attended_blocks(i.len, ch.recent, ch.n_blocks) * 32 >
                        a.split_keys * a.max_splits)
      fail("rows past the splits", s, i.len);
  }
  return hipSuccess;
}

}  // namespace ra

int main(int argc, char** argv) {
  if (argc != 5) return 2;
  std::mt19937 rng(std::atoi(argv[1]));
  const auto pick = [&](int n) { return static_cast<int>(rng() % static_cast<unsigned>(n)); };
  ra_config c{};
  c.num_layers = L;
  c.num_q_heads = 2 * Hkv;
  c.num_kv_heads = Hkv;
  c.head_dim = 128;
  c.budget_k = 100 + pick(200);
  c.recent_r = pick(40);
  c.evict_every = 1 + pick(30);
  c.dtype = std::atoi(argv[2]);
  c.layout = std::atoi(argv[3]);
  c.max_seqs = kSlots;
  c.policy_block = 1;
  c.page_rows = 32 << pick(3);
  c.max_prompt_len = 300;
  const int64_t group = static_cast<int64_t>(L) * Hkv * c.page_rows;
  const int64_t rows = (ra_seq_rows(&c, 300) * kSlots + group - 1) / group * group;
  stub_configure(rows, rows / group, kSlots, c.page_rows);
  alignas(16) static char pool[16];                  // the stand-ins touch no row
  std::vector<int32_t> pos(rows + 16);
  std::vector<char> meta(ra_meta_bytes(&c) + 16);
  const auto aligned = [](char* p) { return p + (16 - reinterpret_cast<uintptr_t>(p) % 16) % 16; };
  std::vector<char> bounds(ra_sparse_bytes(&c, rows) + 16);
  g_buf_bytes = ra_sparse_bytes(&c, rows);
  g_buf = reinterpret_cast<int8_t*>(aligned(bounds.data()));
  const int most = 6;
  std::vector<char> ws(ra_sparse_workspace_bytes(&c, most) + 16);
  g_ws = aligned(ws.data());
  g_ws_bytes = ra_sparse_workspace_bytes(&c, most);
  int32_t* p = reinterpret_cast<int32_t*>(aligned(reinterpret_cast<char*>(pos.data())));
  if (ra_cache_create(&c, pool, pool, p, rows, aligned(meta.data()), ra_meta_bytes(&c), nullptr,
                      &g_cache) != RA_OK)
    fail("create", 0, 0);
  const size_t row = 128 * 4;
  std::vector<char> q(kSlots * 2 * Hkv * row), kv(kSlots * Hkv * row),
      many(static_cast<size_t>(L) * Hkv * kRowsMax * row);
  bool attached = false, graph = false;
  int sparse = 0, refused = 0;
  for (int op = 0, ops = std::atoi(argv[4]); op < ops; ++op) {
    const int s = pick(kSlots);
    ra_status st = RA_OK;
    switch (pick(14)) {
      case 0: {
        const int n = pick(301);
        st = ra_seq_begin(g_cache, s, n, 1, op, many.data(), many.data(), nullptr);
        if (st == RA_OK) rows_change(s, 0);
        break;
      }
      case 1:
        if (pick(3) == 0) ra_seq_end(g_cache, s, nullptr);
        break;
      case 2: {
        const ra_seq_info i = info_of(s);
        if (ra_evict_now(g_cache, s, nullptr) == RA_OK && info_of(s).event != i.event)
          rows_change(s, i.prompt_len);
        break;
      }
      case 3: {
        const int n = pick(60);
        const ra_seq_info i = info_of(s);
        if (ra_seq_fast_forward(g_cache, s, n, nullptr) == RA_OK) rows_change(s, i.prompt_len);
        break;
      }
      case 4:
        if (ra_write_rows(g_cache, s, many.data(), many.data(), nullptr) == RA_OK) rows_change(s, 0);
        break;
      case 5: {
        const bool detach = pick(6) == 0;
        g_no_memory = pick(4) == 0;
        st = ra_sparse_attach(g_cache, detach ? nullptr : g_buf, g_buf_bytes, nullptr);
        const bool tried = g_no_memory && !graph;
        g_no_memory = false;
        if (tried) {
          if (st != RA_ERR_CAPACITY) fail("attach without memory", st, detach);
          break;                                     // what was attached stays
        }
        if (st != (graph ? RA_ERR_STATE : RA_OK)) fail("attach", st, graph);
        if (st == RA_OK) {
          attached = !detach;
          for (auto& layer : g_bounds)
            for (auto& slot : layer)
              for (int64_t& b : slot) b = 0;
        }
        break;
      }
      case 6:
        ra_export_rows(g_cache, s, many.data(), nullptr, int64_t(L) * Hkv * kRowsMax * 128, nullptr);
        break;
      case 7: {
        const bool on = pick(3) == 0;
        st = ra_graph_mode(g_cache, on, nullptr);
        if (st == RA_OK) {
          if (graph && !on)
            for (int i = 0; i < kSlots; ++i)
              if (info_of(i).active) rows_change(i, info_of(i).prompt_len);
          graph = on;
        } else if (c.layout != RA_LAYOUT_PAGED) {
          fail("graph mode", st, on);
        }
        break;
      }
      default: {                                     // a step
        const int n_blocks = pick(most + 1), recent = pick(80);
        bool open = false;
        for (int l = 0; l < L; ++l) {
          const bool want = pick(3) != 0;
          const int mark = g_launches;
          g_capturing = pick(20) == 0;
          g_implicit = pick(20) == 0;
          g_no_memory = c.layout != RA_LAYOUT_PAGED;   // (new pages extend the tables)
          st = want ? ra_sparse_attention(g_cache, l, n_blocks, recent, q.data(), kv.data(),
                                          kv.data(), q.data(), g_ws, g_ws_bytes, nullptr)
                    : RA_ERR_STATE;
          const bool may = attached && !graph && !g_capturing && !g_implicit;
          g_capturing = g_implicit = g_no_memory = false;
          if (hipGetLastError() != hipSuccess) fail("an error is left behind", l, st);
          if (want && st != RA_OK) {
            if (st == RA_ERR_STATE ? may : st != RA_ERR_CAPACITY) fail("sparse", st, may);
            if (g_launches != mark) fail("launched and refused", st, l);
            ++refused;
          }
          if (want && st == RA_OK && !may) fail("sparse step allowed", attached, graph);
          sparse += st == RA_OK;
          if (st == RA_ERR_STATE)
            st = ra_decode_attention(g_cache, l, q.data(), kv.data(), kv.data(), q.data(), g_ws,
                                     g_ws_bytes, nullptr);
          if (st == RA_ERR_CAPACITY && !open) break;
          if (st != RA_OK) fail("step", st, l);
          open = true;
        }
        if (!open) break;
        ra_seq_info was[kSlots];
        for (int i = 0; i < kSlots; ++i) was[i] = info_of(i);
        int32_t n = 0;
        if (ra_end_step(g_cache, nullptr, &n) != RA_OK) fail("end", 0, 0);
        for (int i = 0; i < kSlots; ++i)
          if (was[i].active && info_of(i).event != was[i].event) rows_change(i, was[i].prompt_len);
      }
    }
  }
  ra_cache_destroy(g_cache);
  std::printf("{\"sparse\":%d,\"built\":%d,\"checked\":%d,\"refused\":%d}\n", sparse, g_bounds_built,
              g_checked, refused);
  return 0;
}
